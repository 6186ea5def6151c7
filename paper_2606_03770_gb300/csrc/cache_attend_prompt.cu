// cache_attend_prompt.cu -- e2_cache_attend for prompts.
//
// Bound by the fifth-generation tensor cores and, as much, by the exponentials.  A
// block takes 256 rows (queries times the query heads of a KV head), in two groups of
// 128 so that one group's weights are made while the other's products run, and walks over
// tiles of 64 keys.  Four warps dequantise a tile for both (fp16, one rounding: 2^-12 of a
// value), one issues S = q K^T and O += P V, eight make the weights, a thread a row: scores
// come from tensor memory, weights go back into the scores' place, as the operand that P V
// reads from there.  O stays in tensor memory and is brought to a new maximum only
// when the old one is exceeded by 2^8.  Elements of eight lie in the order that unpacking
// leaves (0, 4, 1, 5, 2, 6, 3, 7) in q, K and V, and are put right in the output.
// Weights go to fp16 times 2^7 (2^-12 each; fp16 outputs take the rounding's rest in a second
// product).  A weight of 0 does not stop a NaN among the values, so values whose scale or
// minimum is not finite are held back as zeros, and rows that do see their keys are made NaN.
//
// Every wait ends: one that takes too long marks the block as failed, which then frees
// its tensor memory and writes NaN.
#include "cache_attend.cuh"
#include "ops_tensor.cuh"

namespace e2ops {
namespace {

constexpr int kGroupRows = 128, kKeys = 64, kStages = 3, kRawStages = 3;
constexpr int kUnpackWarps = 4, kThreads = 32 * (1 + 8 + kUnpackWarps);
constexpr int kBarriers = 2 * kStages + 4 + 4 + 2 + 1;
constexpr uint32_t kColumns = 512, kSums = 256;             // tensor memory: scores [group][2][64], then sums [group][128]

template <int D> struct PromptShared {
    static constexpr int kBlocks = D / 64;                   // of 64 elements: 128-byte rows
    static constexpr int kQuery = kBlocks * kGroupRows * 128;                     // a group's
    static constexpr int kTile = kBlocks * kKeys * 128;                           // a tile's keys, or values
    static constexpr int kRawCodes = 16 * (D / 2), kRawScales = 16 * (D / E2_CACHE_GROUP) * 4;
    static constexpr int kRaw = 2 * kRawCodes + 2 * kRawScales;                   // a warp's 16 keys as they are cached
    static constexpr int kBytes = 2 * kQuery + kStages * 2 * kTile + kUnpackWarps * kRawStages * kRaw + 1024;
};

template <class T, int D> __global__ void __launch_bounds__(kThreads, 1) prompt_kernel(const AttendParams p)
{
    using Sh = PromptShared<D>;
    constexpr int GR = D / E2_CACHE_GROUP;
    constexpr bool kRest = std::is_same<T, __half>::value;
    extern __shared__ uint8_t dynamic[];
    uint8_t *smem = dynamic + (1024 - smem_addr(dynamic) % 1024) % 1024;          // (swizzled tiles start on 1024 bytes)
    __shared__ __align__(8) uint64_t barriers[kBarriers];
    __shared__ __align__(4) uint8_t there[kStages][4];      // whether each 16 keys of a stage are there
    __shared__ __align__(8) uint16_t bad[kStages][GR][4];    // keys whose values are not finite
    __shared__ uint32_t tensor_memory;
    __shared__ int failed;
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const int request = blockIdx.y / p.kv_heads, kv = blockIdx.y % p.kv_heads, split = blockIdx.z;
    const Rows rows(p, request);
    const int64_t blocks = (rows.count + kPromptRows - 1) / kPromptRows;
    if (blocks <= blockIdx.x) return;
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&tensor_memory)), "r"(kColumns)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    // (the longest first; one each, where the launch knew how many)
    for (int64_t block = blocks - 1 - blockIdx.x; block >= 0; block -= gridDim.x) {
        const int64_t row0 = block * kPromptRows, last = min(row0 + kPromptRows, rows.count) - 1;
        // the keys that some row sees, in tiles; this split's  (32 bits: lengths stop 64 short of 2^31)
        const int lo = p.window > 0 ? (int)max(rows.pos(row0) - p.window + 1, (int64_t)0) : 0;
        const int hi = (int)min(min(rows.pos(last) + 1, (int64_t)p.table_cols << p.page_shift), (int64_t)0x7fffffc0);
        const int tile_lo = lo / kKeys, tiles = hi > lo ? (hi + kKeys - 1) / kKeys - tile_lo : 0;
        const int per = (tiles + p.splits - 1) / p.splits;
        const int first = (int)min((int64_t)tile_lo + (int64_t)split * per, (int64_t)tile_lo + tiles);
        const int n = min(first + per, tile_lo + tiles) - first;

        uint8_t *queries = smem, *stages = smem + 2 * Sh::kQuery, *raw = stages + kStages * 2 * Sh::kTile;
        const uint32_t full = smem_addr(barriers), empty = full + 8 * kStages;
        const uint32_t scored = empty + 8 * kStages, weighed = scored + 8 * 4;        // [group][2]
        const uint32_t summed = weighed + 8 * 4, asked = summed + 8 * 2;              // [group]; queries there
        if (threadIdx.x == 0) {
            for (int i = 0; i < kStages; ++i) barrier_init(full + 8 * i, kUnpackWarps), barrier_init(empty + 8 * i, 1);
            for (int i = 0; i < 4; ++i) barrier_init(scored + 8 * i, 1), barrier_init(weighed + 8 * i, 4);
            for (int i = 0; i < 2; ++i) barrier_init(summed + 8 * i, 1);
            barrier_init(asked, 8);
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
            failed = 0;
        }
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        __syncthreads();
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const uint32_t memory = *reinterpret_cast<volatile uint32_t *>(&tensor_memory);

        if (warp == 0) {
            // products
            const uint32_t score_kind = product_kind(kKeys), sum_kind = product_kind(D, true);
            bool ok = __all_sync(~0u, barrier_wait(asked, 0));
            for (int j = 0; j <= n && ok; ++j) {
                if (j < n) {
                    const int stage = j % kStages;
                    ok = __all_sync(~0u, barrier_wait(full + 8 * stage, j / kStages & 1));
                    if (!ok) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    if (elected()) {
                        const uint32_t keys = smem_addr(stages) + stage * 2 * Sh::kTile;
#pragma unroll
                        for (int g = 0; g < 2; ++g) {
#pragma unroll
                            for (int k = 0; k < D / 16; ++k) {
                                const uint64_t a = operand(smem_addr(queries) + g * Sh::kQuery + k / 4 * kGroupRows * 128) + 2 * (k % 4);
                                const uint64_t b = operand(keys + k / 4 * kKeys * 128) + 2 * (k % 4);
                                issue_product(memory + g * 128 + (j & 1) * 64, a, b, score_kind, k > 0);
                            }
                            commit_products(scored + 8 * (2 * g + (j & 1)));
                        }
                    }
                    __syncwarp();
                }
                if (j > 0) {
                    const int i = j - 1, stage = i % kStages;
                    const uint32_t values = smem_addr(stages) + stage * 2 * Sh::kTile + Sh::kTile;
                    for (int g = 0; g < 2 && ok; ++g) {
                        ok = __all_sync(~0u, barrier_wait(weighed + 8 * (2 * g + (i & 1)), i / 2 & 1));
                        if (!ok) break;
                        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                        if (elected()) {
                            const uint32_t weights = memory + g * 128 + (i & 1) * 64;
#pragma unroll
                            for (int k = 0; k < kKeys / 16; ++k)
                                issue_product(memory + kSums + g * 128, weights + 8 * k, operand(values, kKeys * 128) + k * (16 * 128 / 16), sum_kind,
                                              i > 0 || k > 0);
                            if (kRest) {
#pragma unroll
                                for (int k = 0; k < kKeys / 16; ++k)
                                    issue_product(memory + kSums + g * 128, weights + 32 + 8 * k, operand(values, kKeys * 128) + k * (16 * 128 / 16),
                                                  sum_kind, true);
                            }
                            commit_products(summed + 8 * g);
                            if (g == 1) commit_products(empty + 8 * stage);
                        }
                        __syncwarp();
                    }
                }
            }
            if (!ok) failed = 1;
        } else if (warp <= 8) {
            // weights: a thread a row
            const int g = (warp - 1) / 4, quarter = warp % 4, r = 32 * quarter + lane;
            const int64_t row = row0 + g * kGroupRows + r;
            const bool live = rows.live(p, row);
            const uint32_t lanes = (uint32_t)(32 * quarter) << 16;
            float scale;
            {
                // the query, to fp16 times a power of two
                const T *src = static_cast<const T *>(p.q) + (live ? rows.token(row) * p.q_stride + rows.head(kv, row) * D : 0);
                unsigned top = 0;
#pragma unroll
                for (int o = 0; o < D / 8; ++o)
                    if (live) top = max(top, octet_largest(reinterpret_cast<const uint4 *>(src)[o]));
                const int k = power_for<T>(top);
                scale = p.scale * 1.4426950408889634f * power_of_two(-k);
#pragma unroll
                for (int o = 0; o < D / 8; ++o) {
                    uint4 v{0, 0, 0, 0};
                    if (live) v = octet_in_order<T>(reinterpret_cast<const uint4 *>(src)[o], power_of_two(k));
                    *reinterpret_cast<uint4 *>(queries + g * Sh::kQuery + o / 8 * kGroupRows * 128 + r * 128 + ((o % 8) ^ (r & 7)) * 16) = v;
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) barrier_arrive(asked);
            }
            const int pos = row < rows.count ? (int)max(rows.pos(row), (int64_t)-1) : -1;
            const int from = row < rows.count && p.window > 0 ? (int)max(rows.pos(row) - p.window + 1, (int64_t)0) : 0;
            float top = -INFINITY, sum = 0;
            unsigned spoilt = 0;                                 // bit j: this row sees a value of group j that is not finite
            bool ok = true;
            for (int j = 0; j < n; ++j) {
                const int stage = j % kStages, key0 = (first + j) * kKeys;
                const uint32_t at = memory + lanes + g * 128 + (j & 1) * 64;
                ok = __all_sync(~0u, barrier_wait(scored + 8 * (2 * g + (j & 1)), j / 2 & 1));
                if (!ok) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                uint32_t half[2][32];
                load_columns(half[0], at);
                load_columns(half[1], at + 32);
                const uint32_t present = *reinterpret_cast<const volatile uint32_t *>(there[stage]);
                unsigned long long spoils[GR];
#pragma unroll
                for (int i = 0; i < GR; ++i) spoils[i] = *reinterpret_cast<const volatile unsigned long long *>(bad[stage][i]);
                asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
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
                float most = -INFINITY;
#pragma unroll
                for (int k = 0; k < kKeys; ++k) {
                    s[k] = s[k] == -INFINITY ? -INFINITY : s[k] * scale;              // (hidden whatever the scale)
                    most = fmaxf(most, s[k]);
                }
                // (an all-hidden row keeps -inf)
                const bool renew = most > top + 8.0f || (top == -INFINITY && most > -INFINITY);
                if (__any_sync(~0u, renew)) {
                    const float is = fmaxf(top, most), back = top == is ? 1.0f : power2(top - is);
                    top = is;
                    sum *= back;
                    if (j > 0) {
                        ok = __all_sync(~0u, barrier_wait(summed + 8 * g, (j - 1) & 1));
                        if (!ok) break;
                        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                        const uint32_t o = memory + lanes + kSums + g * 128;
#pragma unroll
                        for (int c = 0; c < D; c += 16) {
                            uint32_t v[16];
                            load_columns(v, o + c);
                            asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
                            for (int k = 0; k < 16; ++k) v[k] = __float_as_uint(__uint_as_float(v[k]) * back);
                            store_columns(o + c, v);
                        }
                        asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
                    }
                }
                const float base = top == -INFINITY ? 0.0f : top - 7.0f;
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    uint32_t w[8], rest[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const float a = power2(s[16 * c + 2 * k] - base), b = power2(s[16 * c + 2 * k + 1] - base);
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
                asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                __syncwarp();
                if (lane == 0) barrier_arrive(weighed + 8 * (2 * g + (j & 1)));
            }
            if (ok && n > 0) ok = __all_sync(~0u, barrier_wait(summed + 8 * g, (n - 1) & 1));
            if (!ok) failed = 1;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const bool lost = !ok || *reinterpret_cast<volatile int *>(&failed);
            const float nan = __int_as_float(0x7fc00000);
            const int head = rows.head(kv, row);
            const float inverse = sum > 0 ? 1.0f / sum : 0.0f;
#pragma unroll
            for (int c = 0; c < D; c += 32) {
                uint32_t v[32] = {};
                if (n > 0) {
                    load_columns(v, memory + lanes + kSums + g * 128 + c);
                    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
                }
                // elements 0, 4, 1, 5, 2, 6, 3, 7
                float x[32];
#pragma unroll
                for (int k = 0; k < 32; ++k) x[k / 8 * 8 + k % 8 / 2 + k % 2 * 4] = __uint_as_float(v[k]);
                const bool none = lost || (spoilt >> (c / E2_CACHE_GROUP) & 1);
                if (live && p.splits == 1) {
                    T *out = static_cast<T *>(p.out) + rows.token(row) * p.out_stride + head * D + c;
#pragma unroll
                    for (int o = 0; o < 4; ++o) {
                        float y[8];
#pragma unroll
                        for (int k = 0; k < 8; ++k) y[k] = none ? nan : sum > 0 ? x[8 * o + k] * inverse : sum;
                        *reinterpret_cast<uint4 *>(out + 8 * o) = pack8<T>(y);
                    }
                } else if (live) {
                    float *to = p.parts + ((rows.token(row) * p.q_heads + head) * p.splits + split) * (D + 2);
#pragma unroll
                    for (int k = 0; k < 32; ++k) to[c + k] = none ? nan : x[k];
                    if (c == 0) to[D] = top, to[D + 1] = lost ? nan : sum;
                }
                __syncwarp();
            }
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        } else {
            // keys and values: a warp 16 of a tile's 64
            const int w = warp - 9, page_mask = (1 << p.page_shift) - 1;
            const int32_t *table = p.table + request * p.table_stride;
            uint8_t *mine = raw + w * kRawStages * Sh::kRaw;
            auto page_of = [&](int j) {
                const int key = (first + j) * kKeys + 16 * w;
                return j < n && key < hi ? table[key >> p.page_shift] : -1;
            };
            int next = page_of(0);
            auto copy = [&](int j, int place) {
                const int page = next;
                next = page_of(j + 1);
                const bool in = page >= 0 && page < p.pages;
                if (j < n) {
                    const uint32_t to = smem_addr(mine) + place * Sh::kRaw;
                    const int64_t vec = ((((int64_t)(in ? page : 0) * p.kv_heads + kv) << p.page_shift) + (((first + j) * kKeys + 16 * w) & page_mask));
#pragma unroll
                    for (int a = 0; a < 2; ++a)
#pragma unroll
                        for (int i = 0; i < D / 64; ++i) {
                            const int e = i * 32 + lane;
                            copy_async16(to + a * Sh::kRawCodes + e * 16, p.codes[a] + vec * (D / 2) + e * 16, in);
                        }
                    if (lane < 8 * GR) {
                        const int a = lane / (4 * GR), e = lane % (4 * GR);
                        copy_async16(to + 2 * Sh::kRawCodes + a * Sh::kRawScales + e * 16,
                                     reinterpret_cast<const uint8_t *>(p.scales[a] + vec * GR) + e * 16, in);
                    }
                }
                copy_commit();
                return in;
            };
            bool in[3];
            in[0] = copy(0, 0);
            in[1] = copy(1, 1);
            in[2] = false;
            bool ok = true;
            int place = 0;
            for (int j = 0; j < n; ++j) {
                copy_wait<1>();
                __syncwarp();
                const bool present = in[0];
                in[0] = in[1];
                in[1] = copy(j + 2, place == 0 ? 2 : place - 1);
                const uint8_t *from = mine + place * Sh::kRaw;
                place = place == 2 ? 0 : place + 1;
                const int stage = j % kStages;
                ok = __all_sync(~0u, barrier_wait(empty + 8 * stage, (j / kStages & 1) ^ 1));
                if (!ok) break;
                // values' groups that are not finite
                auto finite = [](uint32_t dm) { return (dm & 0x7c00u) != 0x7c00u && (dm & 0x7c000000u) != 0x7c000000u; };
                const uint32_t *scales = reinterpret_cast<const uint32_t *>(from + 2 * Sh::kRawCodes);
#pragma unroll
                for (int i = 0; i < GR; ++i) {
                    const bool spoils = lane < 16 && !finite(scales[16 * GR + lane * GR + i]);
                    const unsigned mask = __ballot_sync(~0u, spoils);
                    if (lane == 0) bad[stage][i][w] = (uint16_t)mask;
                }
                if (lane == 0) there[stage][w] = present;
                constexpr int kWords = D / 8, kAtOnce = 32 / kWords;                  // of a key; keys at once
                const int word = lane % kWords, group = word / 8;
#pragma unroll
                for (int a = 0; a < 2; ++a) {
                    uint8_t *to = stages + (stage * 2 + a) * Sh::kTile + word / 8 * kKeys * 128;
#pragma unroll
                    for (int i = 0; i < 16 / kAtOnce; ++i) {
                        const int key = i * kAtOnce + lane / kWords, r = 16 * w + key;
                        const uint32_t codes = reinterpret_cast<const uint32_t *>(from + a * Sh::kRawCodes)[key * kWords + word];
                        const uint32_t dm = scales[a * 16 * GR + key * GR + group];
                        __half2 both = *reinterpret_cast<const __half2 *>(&dm);
                        __half2 d = __low2half2(both), m = __high2half2(both);
                        if (!finite(dm)) {
                            // keys are NaN then, values 0
                            d = __float2half2_rn(0.0f);
                            m = a ? d : __float2half2_rn(__int_as_float(0x7fc00000));
                        }
                        *reinterpret_cast<uint4 *>(to + r * 128 + ((word % 8) ^ (r & 7)) * 16) = unpack_word(codes, d, m);
                    }
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) barrier_arrive(full + 8 * stage);
            }
            if (!ok) failed = 1;
            copy_wait<0>();
        }
        __syncthreads();
        if (threadIdx.x == 0)
            for (int i = 0; i < kBarriers; ++i) asm volatile("mbarrier.inval.shared::cta.b64 [%0];" ::"r"(full + 8 * i) : "memory");
        __syncthreads();
    }
    asm volatile("griddepcontrol.launch_dependents;");
    __syncwarp();
    if (warp == 0)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(*reinterpret_cast<volatile uint32_t *>(&tensor_memory)),
                     "r"(kColumns)
                     : "memory");
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
    kernel<<<dim3((unsigned)blocks, (unsigned)pairs, (unsigned)p.splits), kThreads, smem, s>>>(p);
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
