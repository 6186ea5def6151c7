// cache_attend_tree.cu -- e2_cache_attend_tree from 17 rows of a request and KV head on.
//
// A block takes 128 rows (nodes times the query heads of a KV head) and walks over tiles of 64
// keys.  A warp copies them, eight dequantise a tile (fp16, one rounding: 2^-11 of a value), one issues
// S = q K^T, one O += P V, four make the weights, a thread a row.  Queries, weights and O are in tensor memory:
// a tile's keys and values are all that the products read from shared memory.  Up to 64 rows lie in it twice (TWICE), the
// first ones with the weights of a tile's first 32 keys and zeros, the others with those of the last, so that all eight warps
// have weights to make; their sums are joined at the end.  A warp that has no rows makes none.
// Even and odd tiles have weights' warps, maxima and sums of their own, joined at the end.
// Bound by a tile's instructions (65 to 69% of issue slots) and the waits between its steps (copied, unpacked, scored,
// weighed, summed: 100 to 400 cycles each, three to five tiles on their way); half the unpacking would give 5%, half the
// weights 0 to 4, half of either product 2.  Measured, us (128 elements, bf16): 8 requests x 8 KV heads x 56 rows x 65,536
// keys 265 (1,080 cycles a tile; the cache alone 89 at the memory's rate), 2 x 8 x 1,024 rows x 16,384 keys 151 (907 TFLOP/s,
// 48% of the tensor cores' measured rate), 8 x 8 x 128 rows x 2,304 keys 24, of which 6 before the first product and 4 after
// the last; 13 x 3 x 77 rows, window 128, 9.6; 8 x 8 x 16 rows, window 128 of 65,000 keys, 11.4.
// On the way: one set of weights' warps 400 for the first, copies by 16 keys 360, by one warp 320, eight warps that unpack
// 315, a barrier polled by one lane for its warp twice as long, copies of one tile after the other 304, both widths of
// weights in one kernel 284, sixteen warps that unpack 274, four copies of the code for the rows' end 270 (and 2.5 us of
// 14 of a small call that has to fetch them).
// Elements of eight lie in the order that unpacking leaves (0, 4, 1, 5, 2, 6, 3, 7) in q, K and V,
// and are put right in the output.  Weights go to fp16 times 2^7 (2^-11 each; fp16 outputs take the
// rounding's rest in a second product).  A weight of 0 does not stop a NaN among the values, so
// values whose scale or minimum is not finite are held back as zeros, and rows that do see their
// keys are made NaN.
//
// Every wait ends: one that takes too long marks the block as failed, which then frees
// its tensor memory and writes NaN.
#include "cache_attend.cuh"
#include "ops_tensor.cuh"

namespace e2ops {
namespace {

constexpr int kKeys = 64, kStages = 5, kRawStages = 6, kScores = 3;
// Warps by fours, one on each scheduler: products and copies, two sets for weights, three to unpack; and the
// registers they split a block's 768 x 80 into.
constexpr int kThreads = 768, kUnpackSets = 3;
constexpr int kBarriers = 2 * kStages + 3 * kScores + 1 + 2 * kRawStages;
constexpr uint32_t kColumns = 512, kSums = 192, kQueries = 448;       // tensor memory: scores [3][64], sums [2][128], queries

template <int D> struct TreeShared {
    static constexpr int kBlocks = D / 64;                   // of 64 elements: 128-byte rows
    static constexpr int kTile = kBlocks * kKeys * 128;      // a tile's keys, or values
    // A tile as it is cached: keys' codes, values' codes, keys' scales, values' scales; 16 keys' parts of them.
    static constexpr int kCodes = 16 * (D / 2), kScales = 16 * (D / E2_CACHE_GROUP) * 4;
    static constexpr int kRaw = 8 * (kCodes + kScales);
    static constexpr int kBytes = kStages * 2 * kTile + kRawStages * kRaw + 1024;
};

// Rows of a block: 64 that lie there twice, or 128.
template <bool TWICE> constexpr int kRowsOf = TWICE ? kTreeRows / 2 : kTreeRows;

// So many rows, and the tiles of keys that they see, of this split's.
struct Span {
    Slab slab;
    int hi, first, n;
    __device__ Span(const AttendParams &p, const Rows &rows, const Tree &tree, int64_t block, int at_once) : slab(rows, block * at_once)
    {
        const int last = (int)min((int64_t)at_once, slab.left) - 1;
        // (32 bits: lengths stop 64 short of 2^31)
        const int lo = p.window > 0 ? (int)max((int64_t)tree.base - p.window + 1, (int64_t)0) : 0;
        hi = (int)max(min(min(slab.pos(last) + 1, (int64_t)p.table_cols << p.page_shift), (int64_t)0x7fffffc0), (int64_t)0);
        const int tile_lo = lo / kKeys, tiles = hi > lo ? (hi + kKeys - 1) / kKeys - tile_lo : 0;
        const int per = (tiles + p.splits - 1) / p.splits;
        first = (int)min((int64_t)tile_lo + (int64_t)blockIdx.z * per, (int64_t)tile_lo + tiles);
        n = min(first + per, tile_lo + tiles) - first;
    }
};

// What a block shares.
template <int D> struct Shared {
    uint8_t *stages, *raw;
    uint32_t full, empty, scored, weighed, summed, asked;    // barriers; scored, weighed, summed [kScores]
    uint32_t copied, taken;                                  // [raw stage]
    uint8_t (*raw_there)[4];                                 // [raw stage]
    uint8_t (*there)[4];                                     // [stage]: whether each 16 keys are there
    uint16_t (*bad)[D / E2_CACHE_GROUP][4];                  // [stage][group]: keys whose values are not finite
    float *states;                                           // [row]: an odd tiles' maximum, sum of weights, spoilt groups
    volatile int *failed;
    uint32_t memory;
};

__device__ __forceinline__ bool warp_wait(uint32_t at, uint32_t parity, int lane)
{
    return __all_sync(~0u, barrier_wait(at, parity));
}

__device__ __forceinline__ bool finite(uint32_t dm) { return (dm & 0x7c00u) != 0x7c00u && (dm & 0x7c000000u) != 0x7c000000u; }

// A warp: S = q K^T of each tile.
template <int D> __device__ __forceinline__ void score(const Shared<D> &m, int n, int lane)
{
    using Sh = TreeShared<D>;
    const uint32_t kind = product_kind(kKeys);
    const uint64_t keys0 = operand(smem_addr(m.stages));
    bool ok = warp_wait(m.asked, 0, lane);
    int stage = 0, phase = 0, place = 0, used = 1;
    for (int j = 0; j < n && ok; ++j) {
        ok = warp_wait(m.full + 8 * stage, phase, lane);
        // (the weights in this place have been used)
        if (ok) ok = warp_wait(m.summed + 8 * place, used, lane);
        if (!ok) break;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        if (elected()) {
            // (addresses in 16 bytes: a block of 64 elements, then 16 of them; queries in columns of two elements)
            const uint64_t b = keys0 + stage * (2 * Sh::kTile / 16);
#pragma unroll
            for (int k = 0; k < D / 16; ++k)
                issue_product(m.memory + place * 64, m.memory + kQueries + 8 * k, b + k / 4 * (kKeys * 8) + 2 * (k % 4), kind, k > 0);
            commit_products(m.scored + 8 * place);
        }
        __syncwarp();
        if (++place == kScores) place = 0, used ^= 1;
        if (++stage == kStages) stage = 0, phase ^= 1;
    }
    if (!ok) *m.failed = 1;
}

// A warp: O += P V of each tile.
template <int D, bool kRest> __device__ __forceinline__ void sum_up(const Shared<D> &m, int n, int lane)
{
    using Sh = TreeShared<D>;
    const uint32_t kind = product_kind(D, true);
    const uint64_t values0 = operand(smem_addr(m.stages) + Sh::kTile, kKeys * 128);
    bool ok = true;
    int stage = 0, place = 0, phase = 0;
    for (int j = 0; j < n && ok; ++j) {
        ok = warp_wait(m.weighed + 8 * place, phase, lane);
        if (!ok) break;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        if (elected()) {
            const uint32_t weights = m.memory + place * 64, sums = m.memory + kSums + (j & 1) * 128;
            const uint64_t b = values0 + stage * (2 * Sh::kTile / 16);
#pragma unroll
            for (int k = 0; k < kKeys / 16; ++k) issue_product(sums, weights + 8 * k, b + k * 128, kind, j > 1 || k > 0);
            if (kRest) {
#pragma unroll
                for (int k = 0; k < kKeys / 16; ++k) issue_product(sums, weights + 32 + 8 * k, b + k * 128, kind, true);
            }
            commit_products(m.summed + 8 * place);
            commit_products(m.empty + 8 * stage);
        }
        __syncwarp();
        if (++place == kScores) place = 0, phase ^= 1;
        if (++stage == kStages) stage = 0;
    }
    if (!ok) *m.failed = 1;
}

// Pairs of 32-bit numbers.
__device__ __forceinline__ uint64_t two_of(float a, float b)
{
    uint64_t d;
    asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(a), "f"(b));
    return d;
}
__device__ __forceinline__ void halves_of(uint64_t x, float &a, float &b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(x)); }
__device__ __forceinline__ uint64_t multiply_add(uint64_t a, uint64_t b, uint64_t c)
{
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ uint64_t add(uint64_t a, uint64_t b)
{
    uint64_t d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ float largest_of(float a, float b, float c)
{
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}

// Four warps: weights of even tiles (set 0) or odd ones, a thread a row; then the rows' outputs, by set 0.
template <class T, int D, bool TWICE>
__device__ __forceinline__ void weights(const AttendParams &p, const Span &span, const Shared<D> &m, const Tree &tree, int64_t skipped,
                                        int kv, int set, int quarter, int lane, bool join)
{
    constexpr int GR = D / E2_CACHE_GROUP;
    constexpr bool kRest = std::is_same<T, __half>::value;
    // (up to 64 rows lie there twice: the first ones have a tile's first 32 keys, the others the last)
    const Slab &slab = span.slab;
    const int row = 32 * (TWICE ? quarter % 2 : quarter) + lane, keys_part = TWICE ? quarter / 2 : 0;
    const bool live = slab.live(row), some = slab.live(row - lane);
    const int64_t token = slab.token(row);
    const int head = slab.head(kv, row);
    const uint32_t lanes = (uint32_t)(32 * quarter) << 16;
    if (set == 0 && some) {
        // the queries, to fp16 times a power of two each (and the scale's sign)
        const uint4 *src = reinterpret_cast<const uint4 *>(static_cast<const T *>(p.q) + (live ? token * p.q_stride + head * D : 0));
        uint4 q[D / 8];
        unsigned largest = 0;
#pragma unroll
        for (int o = 0; o < D / 8; ++o) {
            q[o] = live ? src[o] : uint4{0, 0, 0, 0};
            largest = max(largest, octet_largest(q[o]));
        }
        const int power = power_for<T>(largest);
        const float f = p.scale < 0 ? -power_of_two(power) : power_of_two(power);
#pragma unroll
        for (int o = 0; o < D / 8; o += 4) {
            uint32_t w[16];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const uint4 v = octet_in_order<T>(q[o + k], f);
                w[4 * k] = v.x, w[4 * k + 1] = v.y, w[4 * k + 2] = v.z, w[4 * k + 3] = v.w;
            }
            store_columns(m.memory + lanes + kQueries + 4 * o, w);
        }
        asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
        // (of a query that is not finite every score is infinite or NaN, and its softmax NaN)
        m.states[row * 4 + 3] = not_finite<T>(largest) ? NAN : fabsf(p.scale) * 1.4426950408889634f * power_of_two(-power);
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncwarp();
    if (set == 0 && lane == 0) barrier_arrive(m.asked);
    // keys before the tree up to pos, from `from` on; and those of the node's way
    const int64_t node = skipped + slab.pos(row) - slab.first_pos;
    // (a row of nobody sees as much as others, so that its warp need not look)
    const int pos = tree.base - 1;
    int from = 0;
    const uint64_t way = live ? tree.way(min(node, (int64_t)E2_MAX_DRAFT - 1), from) : 0;
    asm volatile("bar.sync 1, 256;" ::: "memory");
    const float scale = !some ? 0.0f : live && node >= E2_MAX_DRAFT ? NAN : m.states[row * 4 + 3];
    float top = -INFINITY, sum = 0;
    unsigned spoilt = 0;                                     // bit j: this row sees a value of group j that is not finite
    bool ok = true;
    // whether a tile's sums are there, and all before it (products run in their order)
    auto summed = [&](int j) { return warp_wait(m.summed + 8 * (j % kScores), j / kScores & 1, lane); };
    const uint32_t sums = m.memory + lanes + kSums + set * 128;
    // a set's tiles: all 64 keys of each, or this warp's 32 of them
    constexpr int kMine = TWICE ? 32 : 64;
    using Bits = typename std::conditional<TWICE, uint32_t, unsigned long long>::type;
    int stage = set, next_place = set, next_phase = 0;
    for (int j = set; j < span.n; j += 2) {
        const int key0 = (span.first + j) * kKeys + 32 * keys_part, place = next_place;
        const uint32_t at = m.memory + lanes + place * 64;
        ok = warp_wait(m.scored + 8 * place, next_phase, lane);
        if (!ok) break;
        next_place += 2;
        if (next_place >= kScores) next_place -= kScores, next_phase ^= 1;
        if (!some) {
            if (lane == 0) barrier_arrive(m.weighed + 8 * place);
            continue;
        }
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        uint32_t half[kMine / 32][32];
#pragma unroll
        for (int i = 0; i < kMine / 32; ++i) load_columns(half[i], at + 32 * (keys_part + i));
        const uint32_t all_there = TWICE ? 0x0101u : 0x01010101u;
        const uint32_t present = *reinterpret_cast<const volatile uint32_t *>(m.there[stage]) >> (16 * keys_part) & all_there;
        Bits spoils[GR];
#pragma unroll
        for (int i = 0; i < GR; ++i) spoils[i] = *reinterpret_cast<const volatile Bits *>(&m.bad[stage][i][2 * keys_part]);
        stage = stage + 2 >= kStages ? stage + 2 - kStages : stage + 2;
#pragma unroll
        for (int i = 0; i < kMine / 32; ++i) loaded(half[i]);
        float *s = reinterpret_cast<float *>(half);
        // keys this row sees, of these
        Bits seen = ~(Bits)0;
        const bool whole = __all_sync(~0u, from <= key0 && key0 + kMine - 1 <= pos) && present == all_there;
        if (!whole) {
            const int lowest = from - key0, highest = pos - key0, shift = tree.base - key0;
            seen = highest < 0 ? 0 : highest >= kMine - 1 ? ~(Bits)0 : ((Bits)2 << highest) - 1;
            if (lowest > 0) seen &= lowest > kMine - 1 ? 0 : ~(Bits)0 << lowest;
            seen |= (Bits)(shift >= 0 ? (shift > 63 ? 0 : way << shift) : (shift < -63 ? 0 : way >> -shift));
#pragma unroll
            for (int w = 0; w < kMine / 16; ++w)
                if (!(present >> (8 * w) & 1)) seen &= ~((Bits)0xffff << (16 * w));
            // (the table's end, which may be before the tree's)
            if (key0 + kMine > span.hi) seen &= span.hi > key0 ? ((Bits)1 << (span.hi - key0)) - 1 : 0;
#pragma unroll
            for (int k = 0; k < kMine; ++k)
                if (!(seen >> k & 1)) s[k] = -INFINITY;
        }
#pragma unroll
        for (int i = 0; i < GR; ++i)
            if (spoils[i] & seen) spoilt |= 1u << i;
        float part[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) part[k] = fmaxf(s[k], s[k + 4]);
#pragma unroll
        for (int k = 8; k < kMine; k += 8)
#pragma unroll
            for (int i = 0; i < 4; ++i) part[i] = largest_of(part[i], s[k + i], s[k + i + 4]);
        float most = fmaxf(largest_of(part[0], part[1], part[2]), part[3]);
        most = most == -INFINITY ? most : most * scale;  // (hidden is -inf whatever the scale, 0 too)
        const bool renew = most > top + 8.0f || (top == -INFINITY && most > -INFINITY);
        if (__any_sync(~0u, renew)) {
            const float is = fmaxf(top, most), back = top == is ? 1.0f : power2(top - is);
            top = is;
            sum *= back;
            if (j > 1) {
                ok = summed(j - 2);
                if (!ok) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll
                for (int c = 0; c < D; c += 16) {
                    uint32_t v[16];
                    load_columns(v, sums + c);
                    loaded(v);
#pragma unroll
                    for (int k = 0; k < 16; ++k) v[k] = __float_as_uint(__uint_as_float(v[k]) * back);
                    store_columns(sums + c, v);
                }
            }
        }
        const float base = top == -INFINITY ? 0.0f : top - 7.0f;
        // (two at a time where there is nothing to it but arithmetic)
        const uint64_t scales = two_of(scale, scale), bases = two_of(-base, -base);
        uint64_t sums2 = two_of(0, 0);
        const uint32_t to = at + 16 * keys_part;
        auto weigh = [&](auto masked) {
#pragma unroll
            for (int c = 0; c < kMine / 16; ++c) {
                uint32_t w[8], rest[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    float a, b;
                    halves_of(multiply_add(two_of(s[16 * c + 2 * k], s[16 * c + 2 * k + 1]), scales, bases), a, b);
                    a = power2(a), b = power2(b);
                    if (masked.value) {
                        if (!(seen >> (16 * c + 2 * k) & 1)) a = 0;
                        if (!(seen >> (16 * c + 2 * k + 1) & 1)) b = 0;
                    }
                    sums2 = add(sums2, two_of(a, b));
                    w[k] = pack_half(a, b);
                    if (kRest) {
                        const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&w[k]));
                        rest[k] = pack_half(a - f.x, b - f.y);
                    }
                }
                store_columns(to + 8 * c, w);
                if (kRest) store_columns(to + 32 + 8 * c, rest);
            }
        };
        if (whole) weigh(std::false_type{});
        else weigh(std::true_type{});
        if (TWICE) {
            // (of the other keys the row's other place has the weights)
            const uint32_t zeros[16] = {}, others = at + 16 * (1 - keys_part);
            store_columns(others, zeros);
            if (kRest) store_columns(others + 32, zeros);
        }
        float even, odd;
        halves_of(sums2, even, odd);
        sum += even + odd;
        asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        __syncwarp();
        if (lane == 0) barrier_arrive(m.weighed + 8 * place);
    }
    if (ok && span.n > 1) ok = summed(span.n - 2);
    if (ok && span.n > 0) ok = summed(span.n - 1);
    if (!ok) *m.failed = 1;
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    // both sets' sums, brought to the joint maximum; then those of a row's two places, by way of the tiles' place
    // (all products have run)
    auto part_place = [&](int r, int o) { return reinterpret_cast<float4 *>(m.stages + r * D * 4 + ((o & ~7) | ((o ^ r) & 7)) * 16); };
    float *other = m.states + (32 * quarter + lane) * 4;
    if (set == 1) other[0] = top, other[1] = sum, other[2] = __uint_as_float(spoilt);
    asm volatile("bar.sync 1, 256;" ::: "memory");
    if (set == 1) return;
    const bool lost = !ok || *m.failed;
    const float nan = __int_as_float(0x7fc00000);
    // (what saw nothing has no maximum, or what saw NaN; a NaN among others is in the sum, and stays whatever they weigh)
    auto factor = [](float top, float sum, float best) { return sum == 0 || sum != sum ? sum : power2(top - best); };
    auto join_sums = [](float a, float fa, float b, float fb) { return (fa == 0 ? 0.0f : a * fa) + (fb == 0 ? 0.0f : b * fb); };
    const float best = fmaxf(top, other[0]);
    const float f0 = span.n < 1 ? 0.0f : factor(top, sum, best), f1 = span.n < 2 ? 0.0f : factor(other[0], other[1], best);
    sum = join_sums(sum, f0, other[1], f1);
    spoilt |= __float_as_uint(other[2]);
    top = best;
    // elements c and on, 0, 4, 1, 5, 2, 6, 3, 7 of each eight put right
    auto both_sets = [&](int c, float (&x)[32]) {
        auto take = [&](uint32_t from, float f) {
            uint32_t v[32];
            load_columns(v, from + c);
            loaded(v);
#pragma unroll
            for (int k = 0; k < 32; ++k) {
                float &to = x[k / 8 * 8 + k % 8 / 2 + k % 2 * 4];
                to = f == 0 ? to : __fmaf_rn(__uint_as_float(v[k]), f, to);
            }
        };
        if (span.n > 0) take(sums, f0);
        if (span.n > 1) take(sums + 128, f1);
    };
    float g0 = 1, g1 = 0;
    if (TWICE) {
        if (keys_part && some) {
            other[0] = top, other[1] = sum, other[2] = __uint_as_float(spoilt);
#pragma unroll 1
            for (int c = 0; c < D; c += 32) {
                float x[32] = {};
                both_sets(c, x);
#pragma unroll
                for (int k = 0; k < 8; ++k) *part_place(kTreeRows / 2 + row, c / 4 + k) = make_float4(x[4 * k], x[4 * k + 1], x[4 * k + 2], x[4 * k + 3]);
            }
        }
        asm volatile("bar.sync 2, 128;" ::: "memory");
        if (!keys_part && some) {
            const float *theirs = other + kTreeRows / 2 * 4;
            const float most = fmaxf(top, theirs[0]);
            g0 = factor(top, sum, most), g1 = factor(theirs[0], theirs[1], most);
            sum = join_sums(sum, g0, theirs[1], g1);
            spoilt |= __float_as_uint(theirs[2]);
            top = most;
        }
    }
    const bool any = some && !keys_part;
    const float inverse = sum > 0 ? 1.0f / sum : 0.0f;
    // rows as whole lines, a lane an octet, by way of the tiles' place (all products have run)
    constexpr int kOctets = D / 8, kAtOnce = 32 / kOctets, kLoads = 32 / kAtOnce;
    auto place = [&](int r, int o) {
        return reinterpret_cast<uint4 *>(m.stages + o / 8 * kTreeRows * 128 + r * 128 + ((o % 8) ^ (r & 7)) * 16);
    };
    if (any) {
        // (one copy of the code: where it runs once, fetching it is what it costs)
#pragma unroll (TWICE ? 1 : 2)
        for (int c = 0; c < D; c += 32) {
            float x[32] = {};
            both_sets(c, x);
            if (TWICE) {
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const float4 four = *part_place(kTreeRows / 2 + row, c / 4 + k);
                    const float theirs[4] = {four.x, four.y, four.z, four.w};
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[4 * k + i] = join_sums(x[4 * k + i], g0, theirs[i], g1);
                }
            }
            const bool none = lost || (spoilt >> (c / E2_CACHE_GROUP) & 1);
            if (p.splits == 1) {
#pragma unroll
                for (int o = 0; o < 4; ++o) {
                    float y[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) y[k] = none ? nan : sum > 0 ? x[8 * o + k] * inverse : sum;
                    *place(row, c / 8 + o) = pack8<T>(y);
                }
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    *part_place(row, c / 4 + k) = none ? make_float4(nan, nan, nan, nan)
                                                       : make_float4(x[4 * k], x[4 * k + 1], x[4 * k + 2], x[4 * k + 3]);
            }
            __syncwarp();
        }
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    if (p.splits == 1 && any) {
        const int64_t mine = live ? token * p.out_stride + head * D : -1;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int r = i * kAtOnce + lane / kOctets, o = lane % kOctets;
            const int64_t at = __shfl_sync(~0u, mine, r);
            if (at >= 0) reinterpret_cast<uint4 *>(static_cast<T *>(p.out) + at)[o] = *place(row - lane + r, o);
        }
    } else if (join) {
        if (!keys_part) other[0] = top, other[1] = lost ? nan : sum;
    } else if (any) {
        const int64_t mine = live ? ((token * p.q_heads + head) * p.splits + blockIdx.z) * (D + 2) : -1;
        if (live) p.parts[mine + D] = top, p.parts[mine + D + 1] = lost ? nan : sum;
#pragma unroll 4
        for (int r = 0; r < 32; ++r) {
            const int64_t at = __shfl_sync(~0u, mine, r);
            // (8 bytes: rows of parts lie D + 2 apart)
            if (at >= 0 && lane < D / 4) {
                const float4 v = *part_place(row - lane + r, lane);
                reinterpret_cast<float2 *>(p.parts + at)[2 * lane] = make_float2(v.x, v.y);
                reinterpret_cast<float2 *>(p.parts + at)[2 * lane + 1] = make_float2(v.z, v.w);
            }
        }
    }
}

// Eight warps: the parts of a cluster's blocks, in their order.  Block `rank` has every splits-th row.
template <class T, int D, bool TWICE>
__device__ __forceinline__ void join_parts(const AttendParams &p, const Slab &slab, const Shared<D> &m, int kv, int warp, int lane)
{
    const int rank = blockIdx.z;
    for (int r = warp * p.splits + rank; r < kRowsOf<TWICE> && slab.live(r); r += 8 * p.splits) {
        const uint32_t state = smem_addr(m.states + r * 4), part = smem_addr(m.stages + r * D * 4 + ((lane & ~7) | ((lane ^ r) & 7)) * 16);
        float tops[kTreeCluster], weights[kTreeCluster], best = -INFINITY;
        float4 x[kTreeCluster];
#pragma unroll
        for (int k = 0; k < kTreeCluster; ++k) {
            const int peer = min(k, p.splits - 1);
            tops[k] = peer_load(peer_addr(state, peer)), weights[k] = peer_load(peer_addr(state, peer) + 4);
            if (lane < D / 4) x[k] = peer_load4(peer_addr(part, peer));
            best = fmaxf(best, tops[k]);
        }
        float total = 0, y[4] = {};
#pragma unroll
        for (int k = 0; k < kTreeCluster; ++k) {
            // (a part without a maximum saw nothing, or NaN; NaN stays whatever its part weighs)
            const float f = tops[k] == -INFINITY ? (weights[k] == 0 ? 0.0f : weights[k]) : power2(tops[k] - best);
            if (k < p.splits) {
                total = __fmaf_rn(weights[k], f, total);
                const float v[4] = {x[k].x, x[k].y, x[k].z, x[k].w};
#pragma unroll
                for (int i = 0; i < 4; ++i) y[i] = __fmaf_rn(v[i], f, y[i]);
            }
        }
        if (lane < D / 4) {
            T out[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) out[i] = from_float<T>(total > 0 ? y[i] / total : total);
            *reinterpret_cast<uint2 *>(static_cast<T *>(p.out) + slab.token(r) * p.out_stride + slab.head(kv, r) * D + 4 * lane) =
                *reinterpret_cast<const uint2 *>(out);
        }
    }
}

// A tile's runs of keys that lie side by side: one, or two or four where pages are smaller.
__device__ __forceinline__ int runs_of(const AttendParams &p) { return p.page_shift >= 6 ? 1 : 64 >> p.page_shift; }

// A warp for keys (which 0) and one for values: tiles as they are cached, kRawStages ahead, two at a time: what such a warp
// needs for a tile, one instruction after the other, is what bounds a tile.  So one lane, which the compiler knows to be one, asks
// for all copies, and pages are looked up for 32 runs at a time, a lane each, and 32 ahead.
template <int D, int RUNS>
__device__ __forceinline__ void copy_runs(const AttendParams &p, const Span &span, const Shared<D> &m, int request, int kv, int which, int lane)
{
    using Sh = TreeShared<D>;
    constexpr int GR = D / E2_CACHE_GROUP, kRun = kKeys / RUNS;
    constexpr uint32_t kCodeBytes = kRun * (D / 2), kScaleBytes = kRun * (GR * 4);
    static_assert(kRawStages % 2 == 0 && kCodeBytes == 8 * kScaleBytes, "tiles by twos; a run's scales an eighth of its codes");
    const int page_mask = (1 << p.page_shift) - 1;
    const int32_t *table = p.table + request * p.table_stride;
    const uint8_t *codes = p.codes[which], *scales = reinterpret_cast<const uint8_t *>(p.scales[which]);
    const uint32_t to_codes = smem_addr(m.raw) + which * 4 * Sh::kCodes, to_scales = smem_addr(m.raw) + 8 * Sh::kCodes + which * 4 * Sh::kScales;
    auto key_of = [&](int run) { return (int64_t)span.first * kKeys + (int64_t)run * kRun; };
    // (what is loaded here is not touched before its turn)
    auto look_up = [&](int run) { return table[min(key_of(run), (int64_t)span.hi - 1) >> p.page_shift]; };
    // a run's place among the codes, in bytes; -1 where it is not there
    auto place_of = [&](int run, int page) {
        const int64_t key = key_of(run);
        if (key >= span.hi || page < 0 || page >= p.pages) return (int64_t)-1;
        return ((((int64_t)page * p.kv_heads + kv) << p.page_shift) + (key & page_mask)) * (D / 2);
    };
    auto bring = [](uint32_t to, const uint8_t *from, uint32_t bytes, uint32_t barrier) {
        asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(to), "l"(from), "r"(bytes),
                     "r"(barrier)
                     : "memory");
    };
    bool ok = true;
    int issued = 0;
    if (span.n > 0) {
        int64_t places = place_of(lane, look_up(lane));
        int next = look_up(32 + lane), stage = 0, phase = 1;
        for (int run = 0; issued < span.n; run += 2 * RUNS) {
            const bool two = issued + 1 < span.n;
            ok = warp_wait(m.taken + 8 * (stage + (two ? lane % 2 : 0)), phase, lane);
            if (!ok) break;
            int64_t at[2 * RUNS];
#pragma unroll
            for (int i = 0; i < 2 * RUNS; ++i) at[i] = __shfl_sync(~0u, places, run % 32 + i);
            if (elected()) {
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    if (t && !two) break;
                    const uint32_t barrier = m.copied + 8 * (stage + t);
                    uint32_t bytes = 0, there = 0;
#pragma unroll
                    for (int w = 0; w < RUNS; ++w) {
                        bytes += at[t * RUNS + w] < 0 ? 0 : kCodeBytes + kScaleBytes;
                        there |= at[t * RUNS + w] < 0 ? 0 : (RUNS == 1 ? 0x01010101u : RUNS == 2 ? 0x0101u << (16 * w) : 1u << (8 * w));
                    }
                    if (which == 0) *reinterpret_cast<uint32_t *>(m.raw_there[stage + t]) = there;
                    barrier_expect(barrier, bytes);
#pragma unroll
                    for (int w = 0; w < RUNS; ++w) {
                        const int64_t from = at[t * RUNS + w];
                        if (from < 0) continue;
                        bring(to_codes + (stage + t) * Sh::kRaw + w * kCodeBytes, codes + from, kCodeBytes, barrier);
                        bring(to_scales + (stage + t) * Sh::kRaw + w * kScaleBytes, scales + from / 8, kScaleBytes, barrier);
                    }
                }
            }
            __syncwarp();
            issued += two ? 2 : 1;
            if ((run + 2 * RUNS) % 32 == 0) {
                places = place_of(run + 2 * RUNS + lane, next);
                next = look_up(run + 2 * RUNS + 32 + lane);
            }
            stage += 2;
            if (stage == kRawStages) stage = 0, phase ^= 1;
        }
    }
    // (no copy is on its way any more when the block ends: all have been taken, or have come)
    for (int j = max(issued - kRawStages, 0); j < issued; ++j) {
        if (ok) ok = warp_wait(m.taken + 8 * (j % kRawStages), j / kRawStages & 1, lane);
        if (!ok) barrier_wait(m.copied + 8 * (j % kRawStages), j / kRawStages & 1);
    }
    if (!ok) *m.failed = 1;
}
template <int D> __device__ __forceinline__ void copy(const AttendParams &p, const Span &span, const Shared<D> &m, int request, int kv, int which, int lane)
{
    if (runs_of(p) == 1) copy_runs<D, 1>(p, span, m, request, kv, which, lane);
    else if (runs_of(p) == 2) copy_runs<D, 2>(p, span, m, request, kv, which, lane);
    else copy_runs<D, 4>(p, span, m, request, kv, which, lane);
}

// Warp w of four of a set, which has every third tile: 16 of its 64 keys, and values, dequantised.  A lane
// has 32 elements of one key, or of two keys eight apart; so that eight lanes write 128 bytes of different
// banks those of a key's second half write their words in another order.
template <int D> __device__ __forceinline__ void unpack(const Span &span, const Shared<D> &m, int set, int w, int lane)
{
    using Sh = TreeShared<D>;
    constexpr int GR = D / E2_CACHE_GROUP, kParts = D / 32, kItems = kParts / 2;
    const int key = lane / kParts, part = lane % kParts, half = part / 2;
    const uint32_t raw0 = smem_addr(m.raw) + w * Sh::kCodes + lane * 16;
    const uint32_t scales0 = smem_addr(m.raw) + 8 * Sh::kCodes + w * Sh::kScales + (key * GR + half) * 4;
    const int row = 16 * w + key;
    const uint32_t to0 = smem_addr(m.stages) + half * kKeys * 128 + row * 128;
    const uint32_t chunk = (uint32_t)((part % 2 * 4) ^ (row & 7) ^ (2 * half)) * 16;
    bool ok = true;
    int stage = set, phase = 1, raw = set, raw_phase = 0;
    for (int j = set; j < span.n; j += kUnpackSets) {
        ok = warp_wait(m.copied + 8 * raw, raw_phase, lane);
        if (!ok) break;
        uint4 four[2][kItems];
        uint32_t dm[2][kItems];
#pragma unroll
        for (int which = 0; which < 2; ++which)
#pragma unroll
            for (int i = 0; i < kItems; ++i) {
                asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                             : "=r"(four[which][i].x), "=r"(four[which][i].y), "=r"(four[which][i].z), "=r"(four[which][i].w)
                             : "r"(raw0 + raw * Sh::kRaw + which * 4 * Sh::kCodes + i * 512)
                             : "memory");
                asm volatile("ld.shared.u32 %0, [%1];"
                             : "=r"(dm[which][i])
                             : "r"(scales0 + raw * Sh::kRaw + which * 4 * Sh::kScales + i * 8 * GR * 4)
                             : "memory");
            }
        const bool present = *reinterpret_cast<const volatile uint8_t *>(&m.raw_there[raw][w]);
        // (15 |d| + |m| is within fp16's range where |d| is at most 2,048 and |m| below 32,768)
        uint32_t magnitudes = 0;
#pragma unroll
        for (int which = 0; which < 2; ++which)
#pragma unroll
            for (int i = 0; i < kItems; ++i) magnitudes = __vmaxu2(magnitudes, dm[which][i] & 0x7fff7fffu);
        const bool easy = present && (magnitudes & 0xffffu) <= 0x6800u && magnitudes >> 16 < 0x7800u;
        const bool plain = __all_sync(~0u, easy);
        __syncwarp();
        if (lane == 0) barrier_arrive(m.taken + 8 * raw);
        raw += kUnpackSets;
        if (raw >= kRawStages) raw -= kRawStages, raw_phase ^= 1;
        ok = warp_wait(m.empty + 8 * stage, phase, lane);
        if (!ok) break;
        // values' groups that are not finite: bit key
        unsigned bad[GR] = {};
        if (!plain) {
            unsigned votes[kItems];
#pragma unroll
            for (int i = 0; i < kItems; ++i) votes[i] = __ballot_sync(~0u, present && !finite(dm[1][i]));
            for (int k = 0; k < 16; ++k)
#pragma unroll
                for (int g = 0; g < GR; ++g)
                    bad[g] |= (votes[kItems == 1 ? 0 : k / 8] >> (k % (32 / kParts) * kParts + 2 * g) & 1) << k;
        }
        if (lane == 0) {
#pragma unroll
            for (int g = 0; g < GR; ++g) m.bad[stage][g][w] = (uint16_t)bad[g];
            m.there[stage][w] = present;
        }
        const uint32_t to = to0 + stage * 2 * Sh::kTile;
        auto all = [&](auto limit) {
#pragma unroll
            for (int which = 0; which < 2; ++which)
#pragma unroll
                for (int i = 0; i < kItems; ++i) {
                    uint32_t both = dm[which][i];
                    if (limit.value) {
                        // keys are NaN then, values 0; what is not there is 0
                        if (!finite(both)) both = which ? 0u : 0x7e000000u;
                        if (!present) both = 0;
                    }
                    const __half2 h = *reinterpret_cast<const __half2 *>(&both);
                    const __half2 d = __low2half2(h), mn = __high2half2(h);
                    // (half: the third word first)
                    const uint4 &f = four[which][i];
                    const uint32_t words[4] = {half ? f.z : f.x, half ? f.w : f.y, half ? f.x : f.z, half ? f.y : f.w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint4 v = unpack_word<limit.value>(words[e], d, mn);
                        asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(to + which * Sh::kTile + (chunk ^ e * 16) + i * 8 * 128),
                                     "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w)
                                     : "memory");
                    }
                }
        };
        if (plain) all(std::false_type{});
        else all(std::true_type{});
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) barrier_arrive(m.full + 8 * stage);
        stage += kUnpackSets;
        if (stage >= kStages) stage -= kStages, phase ^= 1;
    }
    // (nothing is to arrive at a barrier any more: the last use of each stage)
    for (int j = max(span.n - kStages, 0); j < span.n && ok; ++j) ok = warp_wait(m.empty + 8 * (j % kStages), j / kStages & 1, lane);
    if (!ok) *m.failed = 1;
}

template <class T, int D, bool TWICE> __global__ void __launch_bounds__(kThreads, 1) tree_kernel(const AttendParams p)
{
    using Sh = TreeShared<D>;
    extern __shared__ uint8_t dynamic[];
    __shared__ __align__(8) uint64_t barriers[kBarriers];
    __shared__ __align__(4) uint8_t there[kStages][4], raw_there[kRawStages][4];
    __shared__ __align__(8) uint16_t bad[kStages][D / E2_CACHE_GROUP][4];
    __shared__ uint32_t tensor_memory;
    __shared__ int failed;
    __shared__ float states[kTreeRows * 4];
    __shared__ uint64_t ways[E2_MAX_DRAFT];
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const int request = blockIdx.x / p.kv_heads, kv = blockIdx.x % p.kv_heads;
    wait_before();
    allow_next();
    const Rows rows(p, request);
    constexpr int kRows = kRowsOf<TWICE>;
    const int64_t blocks = (rows.count + kRows - 1) / kRows;
    if (blocks <= blockIdx.y) return;
    const Tree tree(p, rows, ways);
    if (warp == 1) Tree::load(p, request, ways);
    Shared<D> m;
    m.stages = dynamic + (1024 - smem_addr(dynamic) % 1024) % 1024;               // (swizzled tiles start on 1024 bytes)
    m.raw = m.stages + kStages * 2 * Sh::kTile;
    m.full = smem_addr(barriers);
    m.empty = m.full + 8 * kStages;
    m.scored = m.empty + 8 * kStages;
    m.weighed = m.scored + 8 * kScores;
    m.summed = m.weighed + 8 * kScores;
    m.asked = m.summed + 8 * kScores;
    m.copied = m.asked + 8;
    m.taken = m.copied + 8 * kRawStages;
    m.raw_there = raw_there;
    m.there = there;
    m.bad = bad;
    m.states = states;
    m.failed = &failed;
    auto set_barriers = [&] {
        for (int i = 0; i < kStages; ++i) barrier_init(m.full + 8 * i, 4), barrier_init(m.empty + 8 * i, 1);
        for (int i = 0; i < kScores; ++i) barrier_init(m.scored + 8 * i, 1), barrier_init(m.weighed + 8 * i, 4), barrier_init(m.summed + 8 * i, 1);
        barrier_init(m.asked, 4);
        for (int i = 0; i < kRawStages; ++i) barrier_init(m.copied + 8 * i, 2), barrier_init(m.taken + 8 * i, 4);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    };
    if (threadIdx.x == 0) {
        set_barriers();
        failed = 0;
    }
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&tensor_memory)), "r"(kColumns)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    m.memory = *reinterpret_cast<volatile uint32_t *>(&tensor_memory);

    // Blocks of rows; one each, where the launch knew how many.  Between two everyone meets and the
    // barriers start again.
    auto meet = [&](bool more) {
        asm volatile("bar.sync 0, %0;" ::"n"(kThreads) : "memory");
        if (more) {
            if (threadIdx.x == 0) {
                for (int i = 0; i < kBarriers; ++i) asm volatile("mbarrier.inval.shared::cta.b64 [%0];" ::"r"(m.full + 8 * i) : "memory");
                set_barriers();
            }
            asm volatile("bar.sync 0, %0;" ::"n"(kThreads) : "memory");
        }
    };
    // Parts of a cluster's blocks are joined between two barriers of it.
    const bool join = p.splits > 1 && !p.parts;
    if (warp < 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
        for (int64_t block = blockIdx.y; block < blocks; block += gridDim.y) {
            const Span span(p, rows, tree, block, kRows);
            if (warp == 0) score<D>(m, span.n, lane);
            else if (warp == 1) sum_up<D, std::is_same<T, __half>::value>(m, span.n, lane);
            else copy<D>(p, span, m, request, kv, warp - 2, lane);
            __syncwarp();
            if (join) cluster_barrier(), cluster_barrier();
            meet(block + gridDim.y < blocks);
        }
        if (warp == 0)
            asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(m.memory), "r"(kColumns) : "memory");
    } else if (warp < 12) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 136;");
        for (int64_t block = blockIdx.y; block < blocks; block += gridDim.y) {
            const Span span(p, rows, tree, block, kRows);
            weights<T, D, TWICE>(p, span, m, tree, rows.skipped, kv, (warp - 4) / 4, warp % 4, lane, join);
            if (join) {
                cluster_barrier();
                join_parts<T, D, TWICE>(p, span.slab, m, kv, warp - 4, lane);
                cluster_barrier();
            }
            meet(block + gridDim.y < blocks);
        }
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
        for (int64_t block = blockIdx.y; block < blocks; block += gridDim.y) {
            unpack<D>(Span(p, rows, tree, block, kRows), m, (warp - 12) / 4, warp % 4, lane);
            if (join) cluster_barrier(), cluster_barrier();
            meet(block + gridDim.y < blocks);
        }
    }
}

template <class T, int D, bool TWICE> int launch_as(const AttendParams &p, int blocks, int pairs, int dev, cudaStream_t s)
{
    static std::atomic<uint64_t> ready{0};                   // devices that have the attribute set
    auto kernel = tree_kernel<T, D, TWICE>;
    const int smem = TreeShared<D>::kBytes > 120 * 1024 ? TreeShared<D>::kBytes : 120 * 1024;       // (tensor memory is for one block)
    if (!(ready.load(std::memory_order_relaxed) >> dev & 1)) {
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
        if (e != cudaSuccess) return cuda_status(e);
        ready.fetch_or(1ull << dev, std::memory_order_relaxed);
    }
    cudaLaunchAttribute at[2]{};
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = at[1].val.clusterDim.y = 1, at[1].val.clusterDim.z = (unsigned)p.splits;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)pairs, (unsigned)blocks, (unsigned)p.splits);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = (size_t)smem;
    cfg.stream = s;
    cfg.attrs = at;
    cfg.numAttrs = p.splits > 1 && !p.parts ? 2 : 1;
    return cuda_status(cudaLaunchKernelEx(&cfg, kernel, p));
}

}  // namespace

int launch_tree(const AttendParams &p, int head_dim, bool half, bool few, int blocks, int pairs, int dev, cudaStream_t s)
{
    auto as = [&](auto twice) {
        constexpr bool kTwice = decltype(twice)::value;
        if (head_dim == 64)
            return half ? launch_as<__half, 64, kTwice>(p, blocks, pairs, dev, s) : launch_as<__nv_bfloat16, 64, kTwice>(p, blocks, pairs, dev, s);
        return half ? launch_as<__half, 128, kTwice>(p, blocks, pairs, dev, s) : launch_as<__nv_bfloat16, 128, kTwice>(p, blocks, pairs, dev, s);
    };
    return few ? as(std::true_type{}) : as(std::false_type{});
}

}  // namespace e2ops
