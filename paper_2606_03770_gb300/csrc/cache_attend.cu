// cache_attend.cu -- e2_cache_attend: attention over the paged 4-bit cache.
#include <atomic>
#include <type_traits>

#include "cache_attend.cuh"

namespace e2ops {

int check_cache(const e2_cache *c, int dev);

namespace {

// ---- a few rows ------------------------------------------------------------------
//
// Bound by reading the cache.  S^T = K q^T and O^T = V^T P^T on the warp-level
// tensor cores, keys and then dimensions being the 16-row operand and eight rows the
// other, so that one query head per KV head wastes no cache read.  A warp streams
// tiles of 32 keys through a ring of its own (no block barrier) and keeps its own running
// maximum; warps, and splits of a long context over blocks, are joined at the end in
// a fixed order.
//
// A code in the low four bits of a 16-bit word is the fp16 number code x 2^-24, in the
// next four code x 2^-20 (subnormal, exact): codes go to the tensor cores after one shift
// and four ANDs a word.  For the keys the queries carry the other 1/16 and a power of
// two each; a key's scale and minimum are applied to its sums in 32 bits.  The values'
// words are loaded transposed, which pairs two keys of one dimension; their scales
// multiply the weights before these are rounded to fp16, against a running power of two so
// that neither range ends; fp16 outputs take the rounding's rest in a second product.
// Minima are summed in 32 bits.
//
// Measured, us (bf16, 128 elements, 8 KV heads): 8 requests x 65,536 keys of 64 query heads
// 125 (71% of the memory's rate; fp16 139), of 128 heads 177 (50%); 8 x 2,304 keys 16 (joined
// by a second kernel 19), one request 11, of 65,536 keys 32.  A long context is bound by its
// instructions, some 600 a warp and tile (1,000 for sixteen rows), which three warps of a
// scheduler issue at half its rate; four, with two stages or 128 registers, are no faster
// (130, 181).

constexpr int kFewWarps = 4, kTile = 32, kFewStages = 3, kFewBlocks = 3;
constexpr int kMostSplits = 128, kMostCluster = 8;

template <int D> struct FewStage {
    static constexpr int kKeyBytes = D / 2 + 16, kCodes = kTile * kKeyBytes, kScales = kTile * (D / E2_CACHE_GROUP) * 4;
    static constexpr int kBytes = 2 * kCodes + 2 * kScales + 16;
};

__device__ __forceinline__ uint32_t transpose8x8(uint32_t v)
{
    uint32_t d;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(v));
    return d;
}
// What a part's sums are brought to the joint maximum by (without a maximum it saw nothing, or NaN).
__device__ __forceinline__ float part_factor(float top, float weights, float best)
{
    return top == -INFINITY ? (weights == 0 ? 0.0f : weights) : power2(top - best);
}

template <class T, int D, int NT> __global__ void __launch_bounds__(32 * kFewWarps, kFewBlocks) few_kernel(const AttendParams p)
{
    using St = FewStage<D>;
    constexpr int U = D / 32, GR = D / E2_CACHE_GROUP, C = 8 * NT;
    constexpr bool kRest = std::is_same<T, __half>::value;
    extern __shared__ __align__(128) uint8_t smem[];
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, g = lane / 4, t = lane % 4;
    const int request = blockIdx.y / p.kv_heads, kv = blockIdx.y % p.kv_heads, split = blockIdx.x;
    const Rows rows(p, request);
    const int page_mask = (1 << p.page_shift) - 1;
    const int32_t *table = p.table + request * p.table_stride;
    uint8_t *ring = smem + warp * kFewStages * St::kBytes;
    const uint32_t ring_at = smem_addr(ring);

    for (int64_t row0 = (int64_t)blockIdx.z * C; row0 < rows.count; row0 += (int64_t)gridDim.z * C) {
        // the keys that some row sees, in tiles; this split's
        const Slab slab(rows, row0);
        const int last = (int)min((int64_t)C, slab.left) - 1;
        // (32 bits: lengths stop 64 short of 2^31)
        const int lo = p.window > 0 ? (int)max(slab.pos(0) - p.window + 1, (int64_t)0) : 0;
        const int hi = (int)max(min(min(slab.pos(last) + 1, (int64_t)p.table_cols << p.page_shift), (int64_t)0x7fffffc0), (int64_t)0);
        const int tile_lo = lo / kTile, tiles = hi > lo ? (hi + kTile - 1) / kTile - tile_lo : 0;
        const int units = (tiles + kFewWarps - 1) / kFewWarps, per = (units + p.splits - 1) / p.splits * kFewWarps;
        const int first = (int)min((int64_t)tile_lo + (int64_t)split * per, (int64_t)tile_lo + tiles);
        const int end = min(first + per, tile_lo + tiles);

        int ahead = first + warp;                    // the next tile to fetch
        int pages[2];
        auto look_up = [&](int tile) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int j = tile * kTile + 16 * h;
                pages[h] = tile < end && j < hi ? table[j >> p.page_shift] : -1;
            }
        };
        auto issue = [&](int slot) {
            if (ahead < end) {
                const uint32_t dst = ring_at + slot * St::kBytes;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const bool there = pages[h] >= 0 && pages[h] < p.pages;
                    const int64_t vec = ((((int64_t)(there ? pages[h] : 0) * p.kv_heads + kv) << p.page_shift) +
                                         ((ahead * kTile + 16 * h) & page_mask));
                    constexpr int kParts = D / 32;       // 16-byte parts of a key
#pragma unroll
                    for (int w = 0; w < 2; ++w) {
#pragma unroll
                        for (int i = 0; i < kParts / 2; ++i) {
                            const int e = i * 32 + lane, key = e / kParts, part = e % kParts;
                            copy_async16(dst + w * St::kCodes + (16 * h + key) * St::kKeyBytes + part * 16,
                                         p.codes[w] + (vec + key) * (D / 2) + part * 16, there);
                        }
                    }
                    // 16 keys' scales: 4 GR pieces, keys' and values'
                    if (lane < 8 * GR) {
                        const int w = lane / (4 * GR), e = lane % (4 * GR);
                        copy_async16(dst + 2 * St::kCodes + w * St::kScales + h * 64 * GR + e * 16,
                                     reinterpret_cast<const uint8_t *>(p.scales[w] + vec * GR) + e * 16, there);
                    }
                    if (lane == 0)
                        asm volatile("st.shared.u32 [%0], %1;" ::"r"(dst + 2 * St::kCodes + 2 * St::kScales + 4 * h),
                                     "r"((uint32_t)there)
                                     : "memory");
                }
            }
            copy_commit();
            ahead += kFewWarps;
            look_up(ahead);
        };
        look_up(ahead);
#pragma unroll
        for (int i = 0; i < kFewStages - 1; ++i) issue(i);

        // queries: this lane's column g of each eight, octets t of each 32 elements
        uint4 *q_shared = reinterpret_cast<uint4 *>(smem + kFewWarps * kFewStages * St::kBytes);   // [NT][U][32]
        __syncthreads();
        float q_sum[NT][GR][2], q_scale[NT][2];          // of columns 2t, 2t + 1
        int seen_hi[NT][2], seen_lo[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int row = 8 * n + g;
            const bool live = slab.live(row);
            const T *src = static_cast<const T *>(p.q) + (live ? slab.token(row) * p.q_stride + slab.head(kv, row) * D : 0);
            unsigned top = 0;
            uint4 qf[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                qf[u] = live ? *reinterpret_cast<const uint4 *>(src + 32 * u + 8 * t) : uint4{0, 0, 0, 0};
                top = max(top, octet_largest(qf[u]));
            }
            top = max(top, __shfl_xor_sync(~0u, top, 1));
            top = max(top, __shfl_xor_sync(~0u, top, 2));
            const int k = power_for<T>(top);
            float sum[GR];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                float s;
                qf[u] = octet_convert<T>(qf[u], p.scale < 0 ? -power_of_two(k) : power_of_two(k), s);
                if (warp == 0) q_shared[(n * U + u) * 32 + lane] = qf[u];
                sum[u / 2] = u % 2 ? sum[u / 2] + s : s;
            }
#pragma unroll
            for (int j = 0; j < GR; ++j) {
                sum[j] += __shfl_xor_sync(~0u, sum[j], 1);
                sum[j] += __shfl_xor_sync(~0u, sum[j], 2);
            }
            // scores to base 2; a code 1 counts 2^-24
            // (of a query that is not finite every score is infinite or NaN, and its softmax NaN)
            const float f = not_finite<T>(top) ? NAN : fabsf(p.scale) * 1.4426950408889634f * power_of_two(-k);
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                q_scale[n][e] = __shfl_sync(~0u, f, (2 * t + e) * 4);
#pragma unroll
                for (int j = 0; j < GR; ++j) q_sum[n][j][e] = __shfl_sync(~0u, sum[j], (2 * t + e) * 4);
                const int at = 8 * n + 2 * t + e;
                const bool seen = slab.live(at);
                seen_hi[n][e] = seen ? (int)max(slab.pos(at), (int64_t)-1) : -1;
                seen_lo[n][e] = seen && p.window > 0 ? (int)max(slab.pos(at) - p.window + 1, (int64_t)0) : 0;
            }
        }
        __syncthreads();
        // tiles in this range need no mask for any column
        const int full_lo = p.window > 0 ? (int)max(slab.pos(last) - p.window + 1, (int64_t)0) : 0;
        const int full_hi = (int)max(slab.pos(0), (int64_t)-1);
        const bool all_live = C <= slab.left;

        float o[U][2][NT][4] = {};                       // sums for dimensions 32 u + 4 g + {0, 1}, {2, 3}
        float low[NT][GR][2] = {}, sum[NT][2] = {};      // minima's sums, weights' sums: this lane's keys
        float top[NT][2], limit[NT][2];                  // maxima, a little stale at times: scores up to limit do not renew them
        float v_power = 0x1p40f;                         // 1 / a power of two: no scale so far is twice as large
#pragma unroll
        for (int n = 0; n < NT; ++n) top[n][0] = top[n][1] = -INFINITY;
        bool started = false;
        int slot = 0;
        for (int tile = first + warp; tile < end; tile += kFewWarps) {
            copy_wait<kFewStages - 2>();
            __syncwarp();
            issue(slot == 0 ? kFewStages - 1 : slot - 1);
            const uint8_t *st = ring + slot * St::kBytes;
            const uint32_t st_at = ring_at + slot * St::kBytes;
            slot = slot == kFewStages - 1 ? 0 : slot + 1;
            const uint2 there = *reinterpret_cast<const uint2 *>(st + 2 * St::kCodes + 2 * St::kScales);

            // scores, but for q_scale: keys 16 m + g + 8 r, columns 8 n + 2 t + e
            float s[2][2][NT][2];
            const uint32_t lo4 = 0x000f000fu, hi4 = 0x00f000f0u;
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                float acc[GR][NT][4];
                const uint32_t mat = st_at + (16 * m + lane % 16) * St::kKeyBytes + lane / 16 * 16;
#pragma unroll
                for (int u = 0; u < U; u += 2) {
                    uint32_t w[4];
                    load_matrices(w, mat + u * 16);
#pragma unroll
                    for (int v = 0; v < 2; ++v) {
                        const uint32_t a = w[2 * v], d = w[2 * v + 1], a8 = a >> 8, d8 = d >> 8;
#pragma unroll
                        for (int n = 0; n < NT; ++n) {
                            const uint4 x = q_shared[(n * U + u + v) * 32 + lane];
                            const float zero[4] = {0, 0, 0, 0};
                            if (v == 0) multiply(acc[u / 2][n], a & lo4, d & lo4, a & hi4, d & hi4, x.x, x.y, zero);
                            else multiply(acc[u / 2][n], a & lo4, d & lo4, a & hi4, d & hi4, x.x, x.y, acc[u / 2][n]);
                            multiply(acc[u / 2][n], a8 & lo4, d8 & lo4, a8 & hi4, d8 & hi4, x.z, x.w, acc[u / 2][n]);
                        }
                    }
                }
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    float2 dm[GR];
                    const __half2 *sc = reinterpret_cast<const __half2 *>(st + 2 * St::kCodes) + (16 * m + g + 8 * r) * GR;
#pragma unroll
                    for (int j = 0; j < GR; ++j) {
                        dm[j] = __half22float2(sc[j]);
                        dm[j].x *= 0x1p24f;
                    }
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            float x = 0;
#pragma unroll
                            for (int j = 0; j < GR; ++j)
                                x = __fmaf_rn(dm[j].x, acc[j][n][2 * r + e], __fmaf_rn(dm[j].y, q_sum[n][j][e], x));
                            s[m][r][n][e] = x;
                        }
                }
            }
            // masks, where the tile is not seen whole by every column
            const int key0 = tile * kTile;
            const bool whole = all_live && key0 >= full_lo && key0 + kTile - 1 <= full_hi && there.x && there.y;
            unsigned hidden[NT][2] = {};                  // bit 2 m + r
            if (!whole) {
#pragma unroll
                for (int m = 0; m < 2; ++m)
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const int key = key0 + 16 * m + g + 8 * r;
                        const bool in = (m ? there.y : there.x) != 0 && key < hi;
#pragma unroll
                        for (int n = 0; n < NT; ++n)
#pragma unroll
                            for (int e = 0; e < 2; ++e)
                                if (!in || key > seen_hi[n][e] || key < seen_lo[n][e]) {
                                    s[m][r][n][e] = -INFINITY;
                                    hidden[n][e] |= 1u << (2 * m + r);
                                }
                    }
            }
            unsigned every = ~0u;
#pragma unroll
            for (int n = 0; n < NT; ++n) every &= hidden[n][0] & hidden[n][1];
            // values' scales of this lane's keys
            float2 vs[2][2][GR];
            float most = 0;
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
                for (int r = 0; r < 2; ++r)
#pragma unroll
                    for (int j = 0; j < GR; ++j) {
                        vs[m][r][j] = __half22float2(reinterpret_cast<const __half2 *>(
                            st + 2 * St::kCodes + St::kScales)[(16 * m + g + 8 * r) * GR + j]);
                        // (not of keys hidden from all of this lane's columns; an infinite one counts as fp16's largest)
                        if (whole || !(every >> (2 * m + r) & 1)) most = fmaxf(most, fminf(fabsf(vs[m][r][j].x), 65504.0f));
                    }
            // a new maximum, or scale, only where the old one is exceeded by a factor
            // of four (or two): then all sums so far are brought to the new one
            bool renew = !started || most * v_power >= 2.0f;
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    renew |= fmaxf(fmaxf(s[0][0][n][e], s[0][1][n][e]), fmaxf(s[1][0][n][e], s[1][1][n][e])) > limit[n][e];
            if (__any_sync(~0u, renew)) {
                started = true;
#pragma unroll
                for (int k = 16; k; k >>= 1) most = fmaxf(most, __shfl_xor_sync(~0u, most, k));
                const float power = most > 0 ? power_of_two(127 - (int)(__float_as_uint(most) >> 23)) : v_power;
                const float now = fminf(v_power, power), back = now / v_power;
                v_power = now;
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float x = fmaxf(fmaxf(s[0][0][n][e], s[0][1][n][e]), fmaxf(s[1][0][n][e], s[1][1][n][e]));
#pragma unroll
                        for (int k = 4; k < 32; k *= 2) x = fmaxf(x, __shfl_xor_sync(~0u, x, k));
                        // (hidden is -inf whatever the scale, 0 too)
                        x = x == -INFINITY ? x : x * q_scale[n][e];
                        const float was = top[n][e], is = fmaxf(was, x);
                        const float f = was == is || was == -INFINITY ? (was == is ? 1.0f : 0.0f) : power2(was - is);
                        top[n][e] = is;
                        // (a column that has seen nothing takes its first score whatever the scale, 0 too)
                        limit[n][e] = is == -INFINITY ? -INFINITY : q_scale[n][e] > 0 ? (is + 2.0f) / q_scale[n][e] : INFINITY;
                        sum[n][e] *= f;
#pragma unroll
                        for (int j = 0; j < GR; ++j) low[n][j][e] *= f;
                        const float fo = f * back;
#pragma unroll
                        for (int u = 0; u < U; ++u)
#pragma unroll
                            for (int v = 0; v < 2; ++v) {
                                o[u][v][n][e] *= fo;
                                o[u][v][n][2 + e] *= fo;
                            }
                    }
            }
            // weights, times 2^11; and with the values' scales, in fp16, keys in pairs
            uint32_t pb[GR][2][NT][2], pr[kRest ? GR : 1][2][NT][2];
            float base[NT][2];
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) base[n][e] = top[n][e] == -INFINITY ? 0.0f : top[n][e];
            auto weigh = [&](auto masked) {
#pragma unroll
                for (int m = 0; m < 2; ++m)
#pragma unroll
                    for (int r = 0; r < 2; ++r)
#pragma unroll
                        for (int n = 0; n < NT; ++n) {
                            float w[2];
                            bool out[2] = {false, false};
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                w[e] = masked.value && (hidden[n][e] >> (2 * m + r) & 1)
                                           ? 0.0f
                                           : power2(__fmaf_rn(s[m][r][n][e], q_scale[n][e], -base[n][e]));
                                sum[n][e] += w[e];
                                if (masked.value) out[e] = hidden[n][e] >> (2 * m + r) & 1;
                            }
#pragma unroll
                            for (int j = 0; j < GR; ++j) {
                                const float2 &v = vs[m][r][j];
                                const float f = v.x * v_power * 2048.0f;
                                float x[2];
#pragma unroll
                                for (int e = 0; e < 2; ++e) {
                                    // (a hidden key's scale may be anything)
                                    low[n][j][e] = __fmaf_rn(w[e], out[e] ? 0.0f : v.y, low[n][j][e]);
                                    x[e] = w[e] * (out[e] ? 0.0f : f);
                                }
                                const uint32_t h = pack_half(x[0], x[1]);
                                pb[j][m][n][r] = transpose8x8(h);
                                if constexpr (kRest) {
                                    const float2 back = __half22float2(*reinterpret_cast<const __half2 *>(&h));
                                    pr[j][m][n][r] = transpose8x8(pack_half(x[0] - back.x, x[1] - back.y));
                                }
                            }
                        }
            };
            if (whole) weigh(std::false_type{});
            else weigh(std::true_type{});
            // values: matrices of a load are keys 0-7, 8-15, 16-23, 24-31 of 32 dimensions
            const uint32_t mat = st_at + St::kCodes + lane * St::kKeyBytes;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                uint32_t w[4];
                load_matrices_t(w, mat + u * 16);
#pragma unroll
                for (int m = 0; m < 2; ++m) {
                    const uint32_t a = w[2 * m], d = w[2 * m + 1], a8 = a >> 8, d8 = d >> 8;
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        const uint32_t b0 = pb[u / 2][m][n][0], b1 = pb[u / 2][m][n][1];
                        multiply(o[u][0][n], a & lo4, a & hi4, d & lo4, d & hi4, b0, b1, o[u][0][n]);
                        multiply(o[u][1][n], a8 & lo4, a8 & hi4, d8 & lo4, d8 & hi4, b0, b1, o[u][1][n]);
                        if constexpr (kRest) {
                            const uint32_t c0 = pr[u / 2][m][n][0], c1 = pr[u / 2][m][n][1];
                            multiply(o[u][0][n], a & lo4, a & hi4, d & lo4, d & hi4, c0, c1, o[u][0][n]);
                            multiply(o[u][1][n], a8 & lo4, a8 & hi4, d8 & lo4, d8 & hi4, c0, c1, o[u][1][n]);
                        }
                    }
                }
            }
        }
        copy_wait<0>();
        allow_next();

        // this warp's sums, whole: [C] maxima, [C] weights, [C][D + 1] sums (rows apart in banks)
        __syncthreads();
        float *mine = reinterpret_cast<float *>(smem) + warp * (C * (D + 3));
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int c = 8 * n + 2 * t + e;
#pragma unroll
                for (int k = 4; k < 32; k *= 2) {
                    sum[n][e] += __shfl_xor_sync(~0u, sum[n][e], k);
#pragma unroll
                    for (int j = 0; j < GR; ++j) low[n][j][e] += __shfl_xor_sync(~0u, low[n][j][e], k);
                }
                if (g == 0) mine[c] = top[n][e], mine[C + c] = sum[n][e];
                // codes count 2^-24 (2^-20 the second and fourth), weights 2^11
                const float f = 0x1p13f / v_power;
                float *to = mine + 2 * C + c * (D + 1) + 4 * g;
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const float z = low[n][u / 2][e];
                    to[32 * u] = __fmaf_rn(o[u][0][n][e], f, z);
                    to[32 * u + 1] = __fmaf_rn(o[u][0][n][2 + e], f * 0.0625f, z);
                    to[32 * u + 2] = __fmaf_rn(o[u][1][n][e], f, z);
                    to[32 * u + 3] = __fmaf_rn(o[u][1][n][2 + e], f * 0.0625f, z);
                }
            }
        __syncthreads();
        float *shared_parts = reinterpret_cast<float *>(smem) + kFewWarps * (C * (D + 3));
        for (int i = threadIdx.x; i < C * D; i += 32 * kFewWarps) {
            const int c = i / D, d = i % D;
            if (!slab.live(c)) continue;
            const float *all = reinterpret_cast<const float *>(smem);
            float best = -INFINITY, total = 0, x = 0;
#pragma unroll
            for (int w = 0; w < kFewWarps; ++w) best = fmaxf(best, all[w * (C * (D + 3)) + c]);
#pragma unroll
            for (int w = 0; w < kFewWarps; ++w) {
                const float *from = all + w * (C * (D + 3));
                const float f = from[c] == -INFINITY ? 0.0f : power2(from[c] - best);
                if (from[c] == -INFINITY && !(from[C + c] != from[C + c])) continue;
                total = __fmaf_rn(from[C + c], f, total);
                x = __fmaf_rn(from[2 * C + c * (D + 1) + d], f, x);
            }
            const int64_t token = slab.token(c);
            const int head = slab.head(kv, c);
            if (p.splits == 1) {
                static_cast<T *>(p.out)[token * p.out_stride + head * D + d] =
                    from_float<T>(total > 0 ? x / total : total);
            } else {
                float *to = p.parts ? p.parts + ((token * p.q_heads + head) * p.splits + split) * (D + 2)
                                    : shared_parts + c * (D + 2);
                to[d] = x;
                if (d == 0) to[D] = best, to[D + 1] = total;
            }
        }
        if (p.splits > 1 && !p.parts) {
            // the cluster's parts, in their order
            cluster_barrier();
            const uint32_t part_at = smem_addr(shared_parts);
            for (int i = threadIdx.x + split * 32 * kFewWarps; i < C * D; i += 32 * kFewWarps * p.splits) {
                const int c = i / D, d = i % D;
                if (!slab.live(c)) continue;
                float tops[kMostCluster], weights[kMostCluster], x[kMostCluster], best = -INFINITY;
#pragma unroll
                for (int k = 0; k < kMostCluster; ++k) {
                    const uint32_t at = peer_addr(part_at + c * (D + 2) * 4, min(k, p.splits - 1));
                    tops[k] = peer_load(at + D * 4), weights[k] = peer_load(at + D * 4 + 4), x[k] = peer_load(at + d * 4);
                    best = fmaxf(best, tops[k]);
                }
                float total = 0, sum = 0;
#pragma unroll
                for (int k = 0; k < kMostCluster; ++k) {
                    const float f = part_factor(tops[k], weights[k], best);
                    if (k < p.splits) total = __fmaf_rn(weights[k], f, total), sum = __fmaf_rn(x[k], f, sum);
                }
                static_cast<T *>(p.out)[slab.token(c) * p.out_stride + slab.head(kv, c) * D + d] =
                    from_float<T>(total > 0 ? sum / total : total);
            }
            cluster_barrier();                           // (peers have been read)
        }
        __syncthreads();                                 // (the next rows' tiles overwrite the sums)
    }
}

// A split context's parts, joined in a fixed order: a block per row, its warps over
// the parts.
template <class T, int D> __global__ void __launch_bounds__(128) join_kernel(const AttendParams p)
{
    __shared__ float factor[kMostSplits], partial[3][D];
    wait_before();
    const int request = blockIdx.y / p.kv_heads, kv = blockIdx.y % p.kv_heads, lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const Rows rows(p, request);
    for (int64_t row = blockIdx.x; row < rows.count; row += gridDim.x) {
        const Slab slab(rows, row);
        const int head = slab.head(kv, 0);
        const float *from = p.parts + (slab.token(0) * p.q_heads + head) * p.splits * (D + 2);
        // every warp: the maximum, the parts' factors, the weights' sum
        float best = -INFINITY, total = 0;
        for (int k = lane; k < p.splits; k += 32) best = fmaxf(best, from[k * (D + 2) + D]);
#pragma unroll
        for (int k = 16; k; k >>= 1) best = fmaxf(best, __shfl_xor_sync(~0u, best, k));
        for (int k = lane; k < p.splits; k += 32) {
            const float top = from[k * (D + 2) + D], weights = from[k * (D + 2) + D + 1];
            const float f = part_factor(top, weights, best);
            if (warp == 0) factor[k] = f;
            total = __fmaf_rn(weights, f, total);
        }
#pragma unroll
        for (int k = 16; k; k >>= 1) total += __shfl_xor_sync(~0u, total, k);
        __syncthreads();
        float x[D / 32] = {};
#pragma unroll 4
        for (int k = warp; k < p.splits; k += 4) {
            const float f = factor[k];
#pragma unroll
            for (int i = 0; i < D / 32; ++i) x[i] = __fmaf_rn(from[k * (D + 2) + 32 * i + lane], f, x[i]);
        }
        if (warp > 0) {
#pragma unroll
            for (int i = 0; i < D / 32; ++i) partial[warp - 1][32 * i + lane] = x[i];
        }
        __syncthreads();
        if (warp == 0) {
            T *out = static_cast<T *>(p.out) + slab.token(0) * p.out_stride + head * D;
#pragma unroll
            for (int i = 0; i < D / 32; ++i) {
                const int d = 32 * i + lane;
                const float v = x[i] + partial[0][d] + partial[1][d] + partial[2][d];
                out[d] = from_float<T>(total > 0 ? v / total : total);
            }
        }
        __syncthreads();
    }
}

// From so many rows of a request and KV head on they are a prompt's.  Measured, us (8 KV heads
// of 128 elements; rows by sixteen / by 256): 32 rows of 8 requests x 2,304 keys 33 / 42, 64
// rows 42 / 46, 128 rows 79 / 52; 40 rows of 8 x 65,536 keys 609 / 696; of one request, 64 rows
// x 16,384 keys 44 / 38, 264 x 5,000 keys 51 / 43.
constexpr int kPrompt = 65;

// Up to so many times 128 keys a block, up to eight parts joined in a cluster are better than more
// with a second kernel, if seven eighths of the places hold them (clusters that do not fit wait
// for a whole wave).
constexpr int kClusterUnits = 8;

struct Plan {
    int nt, slabs, splits;      // nt 0: a prompt
    bool cluster;               // joined there
};

// Rows by eight or sixteen, or by 256; keys split until every multiprocessor has its
// blocks, no finer than 128 keys (512).
Plan plan(const e2_cache *c, const e2_attend_args *a, int sms)
{
    Plan f;
    const int64_t rows = (int64_t)(a->max_new > 0 ? a->max_new : 1) * (a->q_heads / c->kv_heads);
    f.nt = rows >= kPrompt ? 0 : rows <= 8 ? 1 : 2;
    const int at_once = f.nt ? 8 * f.nt : kPromptRows;
    const int64_t slabs = (rows + at_once - 1) / at_once;
    f.slabs = (int)(slabs < 65535 ? slabs : 65535);
    int64_t keys = a->max_len;
    if (a->window > 0 && keys > (int64_t)a->window + a->max_new) keys = (int64_t)a->window + a->max_new;
    const int least = f.nt ? kTile * kFewWarps : 512;
    const int64_t units = (keys + least - 1) / least;
    const int64_t pairs = (int64_t)a->batch * c->kv_heads * slabs, places = (int64_t)sms * (f.nt ? kFewBlocks : 1);
    int64_t splits = places / pairs;
    if (splits > units) splits = units;
    f.cluster = f.nt && units <= kMostCluster * kClusterUnits;
    if (f.cluster && splits > kMostCluster) splits = kMostCluster;
    while (f.cluster && splits > 2 && pairs * splits * 8 > places * 7) --splits;
    f.splits = (int)(splits < 1 ? 1 : splits > kMostSplits ? kMostSplits : splits);
    return f;
}

size_t workspace_for(const e2_cache *c, const e2_attend_args *a, const Plan &f)
{
    return f.splits > 1 && !f.cluster ? (size_t)a->tokens * a->q_heads * f.splits * (c->head_dim + 2) * sizeof(float) : 0;
}

template <class T, int D, int NT> int launch_few(const AttendParams &p, const Plan &f, dim3 grid, int dev, cudaStream_t s)
{
    static std::atomic<uint64_t> ready{0};               // devices that have the attribute set
    constexpr size_t ring = (size_t)kFewWarps * kFewStages * FewStage<D>::kBytes, queries = NT * (D / 32) * 512;
    constexpr size_t sums = 8 * NT * (kFewWarps * (D + 3) + D + 2) * sizeof(float);
    constexpr size_t smem = ring + queries > sums ? ring + queries : sums;
    auto kernel = few_kernel<T, D, NT>;
    if (smem > 48 * 1024 && !(ready.load(std::memory_order_relaxed) >> dev & 1)) {
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return cuda_status(e);
        ready.fetch_or(1ull << dev, std::memory_order_relaxed);
    }
    return launch<AttendParams>(kernel, grid, 32 * kFewWarps, smem, f.cluster ? f.splits : 1, false, s, p);
}

template <class T, int D> int launch_attend(const AttendParams &p, const Plan &f, int dev, cudaStream_t s)
{
    const unsigned pairs = (unsigned)p.batch * p.kv_heads;
    const dim3 grid((unsigned)f.splits, pairs, (unsigned)f.slabs);
    const int st = f.nt == 0   ? launch_prompt(p, D, std::is_same<T, __half>::value, f.slabs, (int)pairs, dev, s)
                   : f.nt == 1 ? launch_few<T, D, 1>(p, f, grid, dev, s)
                               : launch_few<T, D, 2>(p, f, grid, dev, s);
    if (st != E2_OK || f.splits == 1 || f.cluster) return st;
    const dim3 rows((unsigned)f.slabs * (f.nt ? 8 * f.nt : kPromptRows), pairs);
    return launch<AttendParams>(join_kernel<T, D>, rows, 128, 0, 1, true, s, p);
}

int check_args(const e2_cache *c, const e2_attend_args *a)
{
    if (!a) return fail(E2_EINVAL, "no arguments");
    if (a->tokens < 0 || a->batch < 0) return fail(E2_EINVAL, "tokens and batch must not be negative");
    if (a->dtype != E2_F16 && a->dtype != E2_BF16) return fail(E2_EINVAL, "q and out are fp16 or bf16");
    if (a->q_heads < 1 || a->q_heads > 4096 || a->q_heads % c->kv_heads)
        return fail(E2_EINVAL, "q_heads must be a multiple of kv_heads in 1..4096");
    if (a->max_new < 0 || a->max_len < 0 || a->window < 0 || a->table_cols < 1 || a->table_stride < a->table_cols)
        return fail(E2_EINVAL, "max_new, max_len and window must not be negative, table_cols in 1..table_stride");
    if (!(a->scale > -INFINITY && a->scale < INFINITY)) return fail(E2_EINVAL, "scale must be finite");
    return E2_OK;
}

}  // namespace
}  // namespace e2ops

using namespace e2ops;

extern "C" size_t e2_cache_attend_workspace(const e2_cache *c, const e2_attend_args *a)
{
    Device dev;
    if (!c || c->kv_heads < 1 || check_args(c, a) || a->tokens == 0 || a->batch == 0 || current_device(&dev)) return 0;
    return workspace_for(c, a, plan(c, a, dev.sms));
}

extern "C" int e2_cache_attend(const e2_cache *c, const e2_attend_args *a, void *workspace, size_t workspace_bytes,
                               void *stream)
{
    Device dev;
    if (int st = current_device(&dev)) return st;
    if (int st = check_cache(c, dev.id)) return st;
    if (int st = check_args(c, a)) return st;
    if (a->tokens == 0 || a->batch == 0) return E2_OK;
    const int64_t row = (int64_t)a->q_heads * c->head_dim;
    if (!a->q || !a->out || !aligned(a->q, 16) || !aligned(a->out, 16) || a->q_stride % 8 || a->out_stride % 8 ||
        a->q_stride < row || a->out_stride < row)
        return fail(E2_EINVAL, "q, out: 16-byte aligned, token strides multiples of 8 and at least a row");
    if (!a->table || !a->lens || !a->starts) return fail(E2_EINVAL, "table, lens and starts must be given");
    const void *ptrs[] = {a->q, a->out, a->table, a->lens, a->starts};
    for (const void *p : ptrs)
        if (!on_device(p, dev.id)) return fail(E2_EINVAL, "arrays must be memory of the current device");
    if ((int64_t)a->batch * c->kv_heads > 65535) return fail(E2_EINVAL, "batch * kv_heads must not exceed 65535");
    const Plan f = plan(c, a, dev.sms);
    const size_t need = workspace_for(c, a, f);
    if (need && (!workspace || workspace_bytes < need)) return fail(E2_ENOMEM, "workspace too small");
    if (need && (!aligned(workspace, 256) || !on_device(workspace, dev.id)))
        return fail(E2_EINVAL, "workspace must be 256-byte aligned memory of the current device");
    AttendParams p{c->pages, __builtin_ctz((unsigned)c->page_size), c->kv_heads, a->tokens, a->q_heads, a->batch, a->window,
                   a->table_cols, f.splits, a->table_stride, a->q_stride, a->out_stride, {c->k_codes, c->v_codes},
                   {reinterpret_cast<const __half2 *>(c->k_scales), reinterpret_cast<const __half2 *>(c->v_scales)},
                   a->table, a->lens, a->starts, a->scale, a->q, a->out, need ? static_cast<float *>(workspace) : nullptr};
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const bool half = a->dtype == E2_F16;
    if (c->head_dim == 64)
        return half ? launch_attend<__half, 64>(p, f, dev.id, s) : launch_attend<__nv_bfloat16, 64>(p, f, dev.id, s);
    return half ? launch_attend<__half, 128>(p, f, dev.id, s) : launch_attend<__nv_bfloat16, 128>(p, f, dev.id, s);
}
