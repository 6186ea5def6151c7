// cache_attend_prompt.cu -- e2_cache_attend for prompts.
//
// A block takes 256 rows (queries times the query heads of a KV head), in two groups of
// 128 so that one group's weights are made while the other's products run, and walks over
// tiles of 64 keys.  Eight warps dequantise a tile for both (fp16, one rounding: 2^-11 of a
// value), four issue S = q K^T and O += P V of each, eight make the weights, a thread a row: scores
// come from tensor memory, weights go back into the scores' place, as the operand that P V
// reads from there.  O stays in tensor memory and is brought to a new maximum only
// when the old one is exceeded by 2^8.  Elements of eight lie in the order that unpacking
// leaves (0, 4, 1, 5, 2, 6, 3, 7) in q, K and V, and are put right in the output.
// Weights go to fp16 times 2^7 (2^-11 each; fp16 outputs take the rounding's rest in a second
// product).  A weight of 0 does not stop a NaN among the values, so values whose scale or
// minimum is not finite are held back as zeros, and rows that do see their keys are made NaN.
//
// Bound by the instructions of a tile: 2,010 cycles, of which the weights' exponentials take
// 1,024 of their unit's and the products 1,000 of the tensor cores'.  Measured (64 query heads
// over 8, 128 elements, bf16): 1,152 queries x 2,304 keys 74 us (880 TFLOP/s, 46% of the
// tensor cores' measured rate), 2,048 x 2,048 90 us, 4 x 256 x 4,096 147 us; 4,096 x 4,096 of 128
// heads 570 us (964 TFLOP/s).  The longest blocks of all heads come first.
//
// Every wait ends: one that takes too long marks the block as failed, which then frees
// its tensor memory and writes NaN.
#include "cache_attend.cuh"
#include "ops_tensor.cuh"

namespace e2ops {
namespace {

constexpr int kGroupRows = 128, kKeys = 64, kStages = 3, kRawStages = 3;
// Warps by fours, one on each scheduler: products (scores and sums of two groups), their weights,
// keys, values; and the registers they split a block's 640 x 96 into.
constexpr int kThreads = 640;
constexpr int kBarriers = 2 * kStages + 4 + 4 + 4 + 1;
constexpr uint32_t kColumns = 512, kSums = 256;             // tensor memory: scores [group][2][64], then sums [group][128]

template <int D> struct PromptShared {
    static constexpr int kBlocks = D / 64;                   // of 64 elements: 128-byte rows
    static constexpr int kQuery = kBlocks * kGroupRows * 128;                     // a group's
    static constexpr int kTile = kBlocks * kKeys * 128;                           // a tile's keys, or values
    static constexpr int kRawCodes = 16 * (D / 2), kRawScales = 16 * (D / E2_CACHE_GROUP) * 4;
    static constexpr int kRaw = kRawCodes + kRawScales;                           // a warp's 16 keys, or values, as they are cached
    static constexpr int kBytes = 2 * kQuery + kStages * 2 * kTile + 8 * kRawStages * kRaw + 1024;
};

// 256 rows, and the tiles of keys that they see, of this split's.
struct Span {
    Slab slab;
    int lo, hi, first, n;
    __device__ Span(const AttendParams &p, const Rows &rows, int64_t block) : slab(rows, block * kPromptRows)
    {
        const int last = (int)min((int64_t)kPromptRows, slab.left) - 1;
        // (32 bits: lengths stop 64 short of 2^31)
        lo = p.window > 0 ? (int)max(slab.pos(0) - p.window + 1, (int64_t)0) : 0;
        hi = (int)max(min(min(slab.pos(last) + 1, (int64_t)p.table_cols << p.page_shift), (int64_t)0x7fffffc0), (int64_t)0);
        const int tile_lo = lo / kKeys, tiles = hi > lo ? (hi + kKeys - 1) / kKeys - tile_lo : 0;
        const int per = (tiles + p.splits - 1) / p.splits;
        first = (int)min((int64_t)tile_lo + (int64_t)blockIdx.z * per, (int64_t)tile_lo + tiles);
        n = min(first + per, tile_lo + tiles) - first;
    }
};

// What a block shares.
template <int D> struct Shared {
    uint8_t *queries, *stages, *raw;
    uint32_t full, empty, scored, weighed, summed, asked;    // barriers; scored, weighed, summed [group][2]
    uint8_t (*there)[4];                                     // [stage]: whether each 16 keys are there
    uint16_t (*bad)[D / E2_CACHE_GROUP][4];                  // [stage][group]: keys whose values are not finite
    volatile int *failed;
    uint32_t memory;
};

__device__ __forceinline__ bool finite(uint32_t dm) { return (dm & 0x7c00u) != 0x7c00u && (dm & 0x7c000000u) != 0x7c000000u; }

// A warp, group g: S = q K^T of each tile.
template <int D> __device__ __forceinline__ void score(const Shared<D> &m, int n, int g)
{
    using Sh = PromptShared<D>;
    const uint32_t kind = product_kind(kKeys);
    const uint64_t query = operand(smem_addr(m.queries + g * Sh::kQuery)), keys0 = operand(smem_addr(m.stages));
    bool ok = __all_sync(~0u, barrier_wait(m.asked, 0));
    int stage = 0, phase = 0;
    for (int j = 0; j < n && ok; ++j) {
        ok = __all_sync(~0u, barrier_wait(m.full + 8 * stage, phase));
        // (the weights in this place have been used)
        if (ok && j > 1) ok = __all_sync(~0u, barrier_wait(m.summed + 8 * (2 * g + (j & 1)), (j / 2 - 1) & 1));
        if (!ok) break;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        if (elected()) {
            // (addresses in 16 bytes: a block of 64 elements, then 16 of them)
            const uint64_t b = keys0 + stage * (2 * Sh::kTile / 16);
#pragma unroll
            for (int k = 0; k < D / 16; ++k)
                issue_product(m.memory + g * 128 + (j & 1) * 64, query + k / 4 * (kGroupRows * 8) + 2 * (k % 4),
                              b + k / 4 * (kKeys * 8) + 2 * (k % 4), kind, k > 0);
            commit_products(m.scored + 8 * (2 * g + (j & 1)));
        }
        __syncwarp();
        if (++stage == kStages) stage = 0, phase ^= 1;
    }
    if (!ok) *m.failed = 1;
}

// A warp, group g: O += P V of each tile.
template <int D, bool kRest> __device__ __forceinline__ void sum_up(const Shared<D> &m, int n, int g)
{
    using Sh = PromptShared<D>;
    const uint32_t kind = product_kind(D, true), sums = m.memory + kSums + g * 128;
    const uint64_t values0 = operand(smem_addr(m.stages) + Sh::kTile, kKeys * 128);
    bool ok = true;
    int stage = 0;
    for (int j = 0; j < n && ok; ++j) {
        ok = __all_sync(~0u, barrier_wait(m.weighed + 8 * (2 * g + (j & 1)), j / 2 & 1));
        if (!ok) break;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        if (elected()) {
            const uint32_t weights = m.memory + g * 128 + (j & 1) * 64;
            const uint64_t b = values0 + stage * (2 * Sh::kTile / 16);
#pragma unroll
            for (int k = 0; k < kKeys / 16; ++k) issue_product(sums, weights + 8 * k, b + k * 128, kind, j > 0 || k > 0);
            if (kRest) {
#pragma unroll
                for (int k = 0; k < kKeys / 16; ++k) issue_product(sums, weights + 32 + 8 * k, b + k * 128, kind, true);
            }
            commit_products(m.summed + 8 * (2 * g + (j & 1)));
            commit_products(m.empty + 8 * stage);
        }
        __syncwarp();
        if (++stage == kStages) stage = 0;
    }
    if (!ok) *m.failed = 1;
}

// Four warps, group g: weights, a thread a row; then the rows' outputs.
template <class T, int D>
__device__ __forceinline__ void weights(const AttendParams &p, const Span &span, const Shared<D> &m, int kv, int g, int quarter,
                                        int lane)
{
    using Sh = PromptShared<D>;
    constexpr int GR = D / E2_CACHE_GROUP;
    constexpr bool kRest = std::is_same<T, __half>::value;
    const int r = 32 * quarter + lane;
    const int row = g * kGroupRows + r;
    const Slab &slab = span.slab;
    const bool live = slab.live(row);
    const int64_t token = slab.token(row);
    const int head = slab.head(kv, row);
    // rows as whole lines, a lane an octet: this warp's 32 rows, kAtOnce at a time; and their place in shared memory
    constexpr int kOctets = D / 8, kAtOnce = 32 / kOctets, kLoads = 32 / kAtOnce;
    auto place = [&](int r, int o) {
        return reinterpret_cast<uint4 *>(m.queries + g * Sh::kQuery + o / 8 * kGroupRows * 128 + r * 128 + ((o % 8) ^ (r & 7)) * 16);
    };
    const uint32_t lanes = (uint32_t)(32 * quarter) << 16;
    constexpr int kNotFinite = 1 << 20;
    float scale;
    {
        // the queries, to fp16 times a power of two each (and the scale's sign)
        const int64_t mine = live ? token * p.q_stride + head * D : -1;
        const int o = lane % kOctets;
        int power = 0;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            uint4 v[kLoads / 2];
#pragma unroll
            for (int i = 0; i < kLoads / 2; ++i) {
                const int64_t at = __shfl_sync(~0u, mine, (half * (kLoads / 2) + i) * kAtOnce + lane / kOctets);
                v[i] = uint4{0, 0, 0, 0};
                if (at >= 0) v[i] = reinterpret_cast<const uint4 *>(static_cast<const T *>(p.q) + at)[o];
            }
#pragma unroll
            for (int i = 0; i < kLoads / 2; ++i) {
                const int turn = half * (kLoads / 2) + i, to = 32 * quarter + turn * kAtOnce + lane / kOctets;
                unsigned top = octet_largest(v[i]);
#pragma unroll
                for (int k = 1; k < kOctets; k *= 2) top = max(top, __shfl_xor_sync(~0u, top, k));
                const int k = power_for<T>(top), theirs = __shfl_sync(~0u, not_finite<T>(top) ? kNotFinite : k, lane % kAtOnce * kOctets);
                if (lane / kAtOnce == turn) power = theirs;
                *place(to, o) = octet_in_order<T>(v[i], p.scale < 0 ? -power_of_two(k) : power_of_two(k));
            }
        }
        // (of a query that is not finite every score is infinite or NaN, and its softmax NaN)
        scale = power == kNotFinite ? NAN : fabsf(p.scale) * 1.4426950408889634f * power_of_two(-power);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) barrier_arrive(m.asked);
    }
    const int pos = row < slab.left ? (int)max(slab.pos(row), (int64_t)-1) : -1;
    const int from = row < slab.left && p.window > 0 ? (int)max(slab.pos(row) - p.window + 1, (int64_t)0) : 0;
    float top = -INFINITY, sum = 0;
    unsigned spoilt = 0;                                     // bit j: this row sees a value of group j that is not finite
    bool ok = true;
    // whether a tile's sums are there, and all before it (the products of a group run in their order)
    auto summed = [&](int j) { return (bool)__all_sync(~0u, barrier_wait(m.summed + 8 * (2 * g + (j & 1)), j / 2 & 1)); };
    int stage = 0;
    for (int j = 0; j < span.n; ++j) {
        const int key0 = (span.first + j) * kKeys;
        const uint32_t at = m.memory + lanes + g * 128 + (j & 1) * 64;
        ok = __all_sync(~0u, barrier_wait(m.scored + 8 * (2 * g + (j & 1)), j / 2 & 1));
        if (!ok) break;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        uint32_t half[2][32];
        load_columns(half[0], at);
        load_columns(half[1], at + 32);
        const uint32_t present = *reinterpret_cast<const volatile uint32_t *>(m.there[stage]);
        unsigned long long spoils[GR];
#pragma unroll
        for (int i = 0; i < GR; ++i) spoils[i] = *reinterpret_cast<const volatile unsigned long long *>(m.bad[stage][i]);
        stage = stage == kStages - 1 ? 0 : stage + 1;
        loaded(half[0]);
        loaded(half[1]);
        float *s = reinterpret_cast<float *>(half);
        // keys this row sees, of the tile's
        unsigned long long seen = ~0ull;
        const bool whole = __all_sync(~0u, from <= key0 && key0 + kKeys - 1 <= pos) && present == 0x01010101u;
        if (!whole) {
            const int lowest = from - key0, highest = pos - key0;
            seen = highest < 0 ? 0ull : highest >= 63 ? ~0ull : (2ull << highest) - 1;
            if (lowest > 0) seen &= lowest > 63 ? 0ull : ~0ull << lowest;
#pragma unroll
            for (int w = 0; w < 4; ++w)
                if (!(present >> (8 * w) & 1)) seen &= ~(0xffffull << (16 * w));
#pragma unroll
            for (int k = 0; k < kKeys; ++k)
                if (!(seen >> k & 1)) s[k] = -INFINITY;
        }
#pragma unroll
        for (int i = 0; i < GR; ++i)
            if (spoils[i] & seen) spoilt |= 1u << i;
        float most = s[0];
#pragma unroll
        for (int k = 1; k < kKeys; ++k) most = fmaxf(most, s[k]);
        most = most == -INFINITY ? most : most * scale;      // (hidden is -inf whatever the scale, 0 too)
        const bool renew = most > top + 8.0f || (top == -INFINITY && most > -INFINITY);
        if (__any_sync(~0u, renew)) {
            const float is = fmaxf(top, most), back = top == is ? 1.0f : power2(top - is);
            top = is;
            sum *= back;
            if (j > 0) {
                ok = summed(j - 1);
                if (!ok) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const uint32_t o = m.memory + lanes + kSums + g * 128;
#pragma unroll
                for (int c = 0; c < D; c += 16) {
                    uint32_t v[16];
                    load_columns(v, o + c);
                    loaded(v);
#pragma unroll
                    for (int k = 0; k < 16; ++k) v[k] = __float_as_uint(__uint_as_float(v[k]) * back);
                    store_columns(o + c, v);
                }
            }
        }
        const float base = top == -INFINITY ? 0.0f : top - 7.0f;
        auto weigh = [&](auto masked) {
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                uint32_t w[8], rest[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    float a = power2(__fmaf_rn(s[16 * c + 2 * k], scale, -base)), b = power2(__fmaf_rn(s[16 * c + 2 * k + 1], scale, -base));
                    if (masked.value) {
                        if (!(seen >> (16 * c + 2 * k) & 1)) a = 0;
                        if (!(seen >> (16 * c + 2 * k + 1) & 1)) b = 0;
                    }
                    sum += a + b;
                    w[k] = pack_half(a, b);
                    if (kRest) {
                        const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&w[k]));
                        rest[k] = pack_half(a - f.x, b - f.y);
                    }
                }
                store_columns(at + 8 * c, w);
                if (kRest) store_columns(at + 32 + 8 * c, rest);
            }
        };
        if (whole) weigh(std::false_type{});
        else weigh(std::true_type{});
        asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        __syncwarp();
        if (lane == 0) barrier_arrive(m.weighed + 8 * (2 * g + (j & 1)));
    }
    if (ok && span.n > 1) ok = summed(span.n - 2);
    if (ok && span.n > 0) ok = summed(span.n - 1);
    if (!ok) *m.failed = 1;
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const bool lost = !ok || *m.failed;
    const float nan = __int_as_float(0x7fc00000);
    const float inverse = sum > 0 ? 1.0f / sum : 0.0f;
#pragma unroll
    for (int c = 0; c < D; c += 32) {
        uint32_t v[32] = {};
        if (span.n > 0) {
            load_columns(v, m.memory + lanes + kSums + g * 128 + c);
            loaded(v);
        }
        // elements 0, 4, 1, 5, 2, 6, 3, 7
        float x[32];
#pragma unroll
        for (int k = 0; k < 32; ++k) x[k / 8 * 8 + k % 8 / 2 + k % 2 * 4] = __uint_as_float(v[k]);
        const bool none = lost || (spoilt >> (c / E2_CACHE_GROUP) & 1);
        if (p.splits == 1) {
            // (the queries' place: this group's last scores are there)
#pragma unroll
            for (int o = 0; o < 4; ++o) {
                float y[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) y[k] = none ? nan : sum > 0 ? x[8 * o + k] * inverse : sum;
                *place(r, c / 8 + o) = pack8<T>(y);
            }
        } else if (live) {
            float *to = p.parts + ((token * p.q_heads + head) * p.splits + blockIdx.z) * (D + 2);
#pragma unroll
            for (int k = 0; k < 32; ++k) to[c + k] = none ? nan : x[k];
            if (c == 0) to[D] = top, to[D + 1] = lost ? nan : sum;
        }
        __syncwarp();
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    if (p.splits == 1) {
        const int64_t mine = live ? token * p.out_stride + head * D : -1;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int from = i * kAtOnce + lane / kOctets, o = lane % kOctets;
            const int64_t at = __shfl_sync(~0u, mine, from);
            if (at >= 0) reinterpret_cast<uint4 *>(static_cast<T *>(p.out) + at)[o] = *place(32 * quarter + from, o);
        }
    }
}

// Warp w of four, for keys (which 0) or values (1): its 16 of a tile's 64, dequantised.
template <int D>
__device__ __forceinline__ void unpack(const AttendParams &p, const Span &span, const Shared<D> &m, int request, int kv, int which, int w, int lane)
{
    using Sh = PromptShared<D>;
    constexpr int GR = D / E2_CACHE_GROUP;
    const int page_mask = (1 << p.page_shift) - 1;
    const int32_t *table = p.table + request * p.table_stride;
    const uint8_t *codes = p.codes[which];
    const __half2 *scales = p.scales[which];
    uint8_t *mine = m.raw + (4 * which + w) * kRawStages * Sh::kRaw;
    auto page_of = [&](int j) {
        const int key = (span.first + j) * kKeys + 16 * w;
        return j < span.n && key < span.hi ? table[key >> p.page_shift] : -1;
    };
    int next = page_of(0);
    auto copy = [&](int j, int place) {
        const int page = next;
        next = page_of(j + 1);
        const bool in = page >= 0 && page < p.pages;
        if (j < span.n) {
            const uint32_t to = smem_addr(mine) + place * Sh::kRaw;
            const int64_t vec = ((((int64_t)(in ? page : 0) * p.kv_heads + kv) << p.page_shift) + (((span.first + j) * kKeys + 16 * w) & page_mask));
#pragma unroll
            for (int i = 0; i < D / 64; ++i) {
                const int e = i * 32 + lane;
                copy_async16(to + e * 16, codes + vec * (D / 2) + e * 16, in);
            }
            if (lane < 4 * GR)
                copy_async16(to + Sh::kRawCodes + lane * 16, reinterpret_cast<const uint8_t *>(scales + vec * GR) + lane * 16, in);
        }
        copy_commit();
        return in;
    };
    bool in0 = copy(0, 0), in1 = copy(1, 1);
    bool ok = true;
    int place = 0, stage = 0, phase = 1;
    for (int j = 0; j < span.n; ++j) {
        copy_wait<1>();
        __syncwarp();
        const bool present = in0;
        in0 = in1;
        in1 = copy(j + 2, place == 0 ? 2 : place - 1);
        const uint8_t *from = mine + place * Sh::kRaw;
        place = place == 2 ? 0 : place + 1;
        ok = __all_sync(~0u, barrier_wait(m.empty + 8 * stage, phase));
        if (!ok) break;
        // a lane looks at one scale and minimum
        const uint32_t *sc = reinterpret_cast<const uint32_t *>(from + Sh::kRawCodes);
        const uint32_t looked = sc[lane % (16 * GR)];
        const float2 range = __half22float2(*reinterpret_cast<const __half2 *>(&looked));
        const bool plain = __all_sync(~0u, __fmaf_rn(15.0f, fabsf(range.x), fabsf(range.y)) <= 65504.0f);
        if (which) {
            // values' groups that are not finite: bit key
            const unsigned mask = plain ? 0 : __ballot_sync(~0u, lane < 16 * GR && !finite(looked));
#pragma unroll
            for (int i = 0; i < GR; ++i) {
                unsigned keys = 0;
                if (mask)
                    for (int key = 0; key < 16; ++key) keys |= (mask >> (key * GR + i) & 1) << key;
                if (lane == 0) m.bad[stage][i][w] = (uint16_t)keys;
            }
        } else if (lane == 0) {
            m.there[stage][w] = present;
        }
        // four words of a key at a time
        constexpr int kFours = D / 32;
        auto all = [&](auto easy) {
#pragma unroll
            for (int i = 0; i < kFours / 2; ++i) {
                const int item = i * 32 + lane, r = 16 * w + item / kFours, word = item % kFours * 4;
                const uint4 four = reinterpret_cast<const uint4 *>(from)[item];
                const uint32_t words[4] = {four.x, four.y, four.z, four.w}, dm = sc[item / kFours * GR + word / 8];
                const __half2 both = *reinterpret_cast<const __half2 *>(&dm);
                __half2 d = __low2half2(both), mn = __high2half2(both);
                if (!easy.value && !finite(dm)) {
                    // keys are NaN then, values 0
                    d = __float2half2_rn(0.0f);
                    mn = which ? d : __float2half2_rn(__int_as_float(0x7fc00000));
                }
                uint8_t *to = m.stages + (stage * 2 + which) * Sh::kTile + word / 8 * kKeys * 128 + r * 128;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    *reinterpret_cast<uint4 *>(to + ((word % 8 + e) ^ (r & 7)) * 16) = unpack_word<!easy.value>(words[e], d, mn);
            }
        };
        if (plain) all(std::true_type{});
        else all(std::false_type{});
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) barrier_arrive(m.full + 8 * stage);
        if (++stage == kStages) stage = 0, phase ^= 1;
    }
    // (nothing is to arrive at a barrier any more)
    for (int i = 0; i < kStages && ok; ++i) {
        ok = __all_sync(~0u, barrier_wait(m.empty + 8 * stage, phase));
        if (++stage == kStages) stage = 0, phase ^= 1;
    }
    if (!ok) *m.failed = 1;
    copy_wait<0>();
}

template <class T, int D> __global__ void __launch_bounds__(kThreads, 1) prompt_kernel(const AttendParams p)
{
    using Sh = PromptShared<D>;
    extern __shared__ uint8_t dynamic[];
    __shared__ __align__(8) uint64_t barriers[kBarriers];
    __shared__ __align__(4) uint8_t there[kStages][4];
    __shared__ __align__(8) uint16_t bad[kStages][D / E2_CACHE_GROUP][4];
    __shared__ uint32_t tensor_memory;
    __shared__ int failed;
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const int request = blockIdx.x / p.kv_heads, kv = blockIdx.x % p.kv_heads;
    const Rows rows(p, request);
    const int64_t blocks = (rows.count + kPromptRows - 1) / kPromptRows;
    if (blocks <= blockIdx.y) return;
    Shared<D> m;
    m.queries = dynamic + (1024 - smem_addr(dynamic) % 1024) % 1024;              // (swizzled tiles start on 1024 bytes)
    m.stages = m.queries + 2 * Sh::kQuery;
    m.raw = m.stages + kStages * 2 * Sh::kTile;
    m.full = smem_addr(barriers);
    m.empty = m.full + 8 * kStages;
    m.scored = m.empty + 8 * kStages;
    m.weighed = m.scored + 8 * 4;
    m.summed = m.weighed + 8 * 4;
    m.asked = m.summed + 8 * 4;
    m.there = there;
    m.bad = bad;
    m.failed = &failed;
    auto set_barriers = [&] {
        for (int i = 0; i < kStages; ++i) barrier_init(m.full + 8 * i, 8), barrier_init(m.empty + 8 * i, 2);
        for (int i = 0; i < 4; ++i)
            barrier_init(m.scored + 8 * i, 1), barrier_init(m.weighed + 8 * i, 4), barrier_init(m.summed + 8 * i, 1);
        barrier_init(m.asked, 8);
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

    // Blocks of rows, the longest first; one each, where the launch knew how many.  Between
    // two everyone meets and the barriers start again.
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
    const int64_t start = blocks - 1 - blockIdx.y;
    if (warp < 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
        for (int64_t block = start; block >= 0; block -= gridDim.y) {
            const Span span(p, rows, block);
            if (warp < 2) score<D>(m, span.n, warp);
            else sum_up<D, std::is_same<T, __half>::value>(m, span.n, warp - 2);
            meet(block >= gridDim.y);
        }
        asm volatile("griddepcontrol.launch_dependents;");
        __syncwarp();
        if (warp == 0)
            asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(m.memory), "r"(kColumns) : "memory");
    } else if (warp < 12) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 136;");
        for (int64_t block = start; block >= 0; block -= gridDim.y) {
            weights<T, D>(p, Span(p, rows, block), m, kv, (warp - 4) / 4, warp % 4, lane);
            meet(block >= gridDim.y);
        }
        asm volatile("griddepcontrol.launch_dependents;");
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
        for (int64_t block = start; block >= 0; block -= gridDim.y) {
            unpack<D>(p, Span(p, rows, block), m, request, kv, (warp - 12) / 4, warp % 4, lane);
            meet(block >= gridDim.y);
        }
        asm volatile("griddepcontrol.launch_dependents;");
    }
}

template <class T, int D> int launch_as(const AttendParams &p, int blocks, int pairs, int dev, cudaStream_t s)
{
    static std::atomic<uint64_t> ready{0};                   // devices that have the attribute set
    auto kernel = prompt_kernel<T, D>;
    const int smem = PromptShared<D>::kBytes > 120 * 1024 ? PromptShared<D>::kBytes : 120 * 1024;   // (tensor memory is for one block)
    if (!(ready.load(std::memory_order_relaxed) >> dev & 1)) {
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
        if (e != cudaSuccess) return cuda_status(e);
        ready.fetch_or(1ull << dev, std::memory_order_relaxed);
    }
    kernel<<<dim3((unsigned)pairs, (unsigned)blocks, (unsigned)p.splits), kThreads, smem, s>>>(p);
    return cuda_status(cudaGetLastError());
}

}  // namespace

int launch_prompt(const AttendParams &p, int head_dim, bool half, int blocks, int pairs, int dev, cudaStream_t s)
{
    if (head_dim == 64)
        return half ? launch_as<__half, 64>(p, blocks, pairs, dev, s) : launch_as<__nv_bfloat16, 64>(p, blocks, pairs, dev, s);
    return half ? launch_as<__half, 128>(p, blocks, pairs, dev, s) : launch_as<__nv_bfloat16, 128>(p, blocks, pairs, dev, s);
}

}  // namespace e2ops
