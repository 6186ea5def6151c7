// quant_matmul.cuh -- the kernel of e2_quant_matmul for a few tokens, and what its
// translation units share.
#pragma once

#include <atomic>
#include <type_traits>

#include "ops_x.cuh"

namespace e2ops {

struct MatmulParams {
    int rows, cols, group, tokens, gated, half;                // half: x, residual and y are fp16, else bf16
    const uint8_t *codes;
    const __half *scales, *mins;
    const void *x, *residual;
    void *y;
    int64_t x_stride, residual_stride, y_stride;
};

// ---- few tokens --------------------------------------------------------------
//
// Bound by reading the weights, then by the instructions that unpack them.  y^T = W
// x^T on the warp-level tensor cores: the weights are the 16-row operand, eight
// tokens the other, so a code is unpacked once and no row is padding.  A warp owns
// 16 rows and streams them through a ring of its own in shared memory, two
// stages of 512 columns, without a block barrier: 256 bytes of a row at a time come at 6.2
// TB/s, 128 bytes of 32 rows at 5.8, and at 4.4 where rows are 14 KB apart.
//
// A code in the low four bits of a 16-bit word is the fp16 number code x 2^-24, in
// the next four code x 2^-20 (both subnormal, exact, and the tensor cores take
// them as they are): unpacking a word is one shift and four ANDs, and the sums hold no
// rounded weight.  x goes to fp16 with a power of two per token (its largest
// value to 2^14..2^15: lossless over 24 binades below it), the columns that meet high
// nibbles with another 1/16, once in a kernel before, or for small calls by each block.  The 8
// that codes are off by is taken out by starting each group's sum at -8 sum x; each group's sum
// is scaled in 32 bits.  Few rows are split over columns, among a block's warps (wk) and the
// blocks of a cluster (split), and joined in a fixed order.
//
// Measured, us (64 columns a group): 57344 x 8192 gated 47 with one token (78% of the memory's
// rate), 55 with eight; 8192 x 28672 32 and 39; 4096 x 4096 6.6 and 7.2; sixteen tokens 92, 63
// and 10.  With eight tokens three warps a scheduler issue in 45% of all slots; four are no faster.

constexpr int kRows = 16;                    // of a warp
constexpr int kChunk = 512;                  // columns of a stage
constexpr int kRowBytes = kChunk / 2 + 16;   // (a stage's rows 16 bytes apart in banks)
constexpr int kWarps = 4;

constexpr int kOwnOctets = 8;                // octets of x that a thread prepares of its own block's

constexpr int kSmemPerSm = 227 * 1024;

// The launch of `tokens` tokens: how the columns are split.
struct FewPlan {
    int nt, wk, split, x_cols, x_pad;
    size_t smem, workspace;
};

// Stages of a warp's ring.  Two leave room for longer segments of x, at whose ends a block's
// warps meet: 57344 x 8192, 8 tokens, us: three and 512 columns 65, two and 1,024 54.
constexpr int kFewStages = 2;

template <int G, bool MINS> struct Stage {
    static constexpr int kPer = kChunk / G;                                 // scales of a row
    static constexpr int kScaleBytes = kRows * kPer * 2;
    static constexpr int kBytes = kRows * kRowBytes + kScaleBytes * (MINS ? 2 : 1);
};

struct FewParams {
    MatmulParams m;
    int outs, wk, split, x_cols, scales_by;     // scales copied by 16 or 8 bytes, by 4, or one by one (2)
    // x as prepared: fp16 octets [8 NT tokens][x_pad], the groups' sums
    // [x_pad / group][8 NT], and 1 / the token's power of two (null: blocks make it themselves)
    uint8_t *prepared;
    int x_pad;
};

// x's bytes in shared memory per token and segment (rows half a 128-byte line apart in banks).
__host__ __device__ constexpr int x_row_bytes(int cols) { return cols * 2 + 64; }

template <class T>
__device__ __forceinline__ void finish_as(const MatmulParams &p, int token, int row, float a, float b)
{
    // (a few units in the last of 24 bits, before the rounding to 16)
    float y = p.gated ? __fdividef(a, 1.0f + __expf(-a)) * b : a;
    if (p.residual) y += to_float(static_cast<const T *>(p.residual)[token * p.residual_stride + row]);
    static_cast<T *>(p.y)[token * p.y_stride + row] = from_float<T>(y);
}
__device__ __forceinline__ void finish(const MatmulParams &p, int token, int row, float a, float b)
{
    if (p.half) finish_as<__half>(p, token, row, a, b);
    else finish_as<__nv_bfloat16>(p, token, row, a, b);
}

// What a token's infinities and NaN among columns col0..col1 - 1 make of a row's sum (the finite
// ones do not matter then).  The kernel's own sums are NaN there: they hold code x and 8 x apart.
static __device__ __noinline__ float sum_not_finite(const uint8_t *codes, const __half *scales, const __half *mins, const void *x,
                                                    int half, int group, int col0, int col1)
{
    float sum = 0;
    for (int c = col0; c < col1; c += 8) {
        const uint4 v = *reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(x) + c);
        const uint32_t words[4] = {v.x, v.y, v.z, v.w};
        for (int j = 0; j < 8; ++j) {
            const uint32_t bits = words[j / 2] >> (16 * (j % 2)) & 0xffffu;
            const float f = half ? __half2float(__ushort_as_half((uint16_t)bits)) : __uint_as_float(bits << 16);
            if (fabsf(f) < INFINITY) continue;
            const float code = (float)(codes[(c + j) / 2] >> (4 * (j % 2)) & 15), d = __half2float(scales[c / group]);
            sum += f * (mins ? __fmaf_rn(d, code, __half2float(mins[c / group])) : d * (code - 8.0f));
        }
    }
    return sum;
}

// Bytes of 8 nt prepared tokens.
__host__ __device__ constexpr size_t prepared_bytes(int nt, int x_pad, int group)
{
    return (size_t)8 * nt * x_pad * 2 + (size_t)x_pad / group * 8 * nt * 4 + 256;
}

// Sums as the product needs them (code 1 is 2^-24): for mins, or -8 of them.
template <bool MINS> __device__ __forceinline__ float group_sum(float sum) { return MINS ? sum * 0x1p-24f : sum * -0x1p-21f; }

// x prepared once for all blocks: a block per token.
template <class T, int G, bool MINS, int NT> __global__ void __launch_bounds__(512) prepare_kernel(const FewParams q)
{
    constexpr int nt = NT;
    uint8_t *to = q.prepared;
    __shared__ unsigned largest;
    allow_next();
    const MatmulParams &p = q.m;
    const int tok = blockIdx.x, octets = q.x_pad / 8;
    if (threadIdx.x == 0) largest = 0;
    __syncthreads();
    const T *x = static_cast<const T *>(p.x) + tok * p.x_stride;
    unsigned m = 0;
    for (int o = threadIdx.x; o < p.cols / 8; o += blockDim.x) m = max(m, octet_largest(reinterpret_cast<const uint4 *>(x)[o]));
    m = __reduce_max_sync(~0u, m);
    if (threadIdx.x % 32 == 0) atomicMax(&largest, m);
    __syncthreads();
    const int k = power_for<T>(largest);
    const float f = power_of_two(k);
    uint4 *out = reinterpret_cast<uint4 *>(to) + (size_t)tok * octets;
    float *sums = reinterpret_cast<float *>(to + (size_t)8 * nt * q.x_pad * 2);
    // (x_pad is a multiple of 512 columns: whole warps)
    for (int o = threadIdx.x; o < octets; o += blockDim.x) {
        uint4 v{0, 0, 0, 0};
        if (o < p.cols / 8) v = reinterpret_cast<const uint4 *>(x)[o];
        float sum;
        out[o] = octet_convert<T>(v, f, sum);
#pragma unroll
        for (int d = 1; d < G / 8; d *= 2) sum += __shfl_xor_sync(~0u, sum, d);
        if (o % (G / 8) == 0) sums[o / (G / 8) * (8 * nt) + tok] = group_sum<MINS>(sum);
    }
    if (threadIdx.x == 0) sums[(size_t)q.x_pad / G * 8 * nt + tok] = power_of_two(-k);
}

template <int G, bool MINS, int NT>
__global__ void __launch_bounds__(32 * kWarps, 3) few_kernel(const FewParams q)
{
    using St = Stage<G, MINS>;
    constexpr int kPer = St::kPer, kStages = kFewStages;
    const int WK = q.wk, RB = kRows * (kWarps / WK);
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ float unscale[8 * NT];                              // 1 / the token's power of two
    __shared__ unsigned largest[8 * NT];
    const MatmulParams &p = q.m;
    const int nt = p.tokens;
    uint8_t *ring = smem;
    // x (one segment, or two in turn), and the groups' sums [x_cols / G][8 NT] of each
    const int sum_bytes = q.x_cols / G * 8 * NT * 4, seg_bytes = sum_bytes + nt * x_row_bytes(q.x_cols);
    uint8_t *xseg = smem + kWarps * kStages * St::kBytes;
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, wr = warp / WK, wk = warp % WK;
    const int g = lane / 4, t = lane % 4;
    const int rank = blockIdx.x % q.split, block = blockIdx.x / q.split;
    const int chunks = (p.cols + kChunk - 1) / kChunk;
    const int c0 = (int)((int64_t)chunks * rank / q.split), c1 = (int)((int64_t)chunks * (rank + 1) / q.split);
    const int groups = p.cols / G;

    // rows of this warp (gated: 8 rows that gate and the 8 that they gate); past the
    // last row the last one is read again, and its results are dropped
    const int first = block * (p.gated ? RB / 2 : RB) + wr * (p.gated ? 8 : 16);
    const int second = p.gated ? q.outs + first : first + 8;
    auto row_of = [&](int r) {
        const int limit = p.gated && r >= 8 ? 2 * q.outs : q.outs;
        return (int64_t)min(r < 8 ? first + r : second + r - 8, limit - 1);
    };
    const uint32_t my_ring = smem_addr(ring) + warp * kStages * St::kBytes;
    // lane l copies 16 bytes (l % 16) of ring rows l / 16 + 2 i
    const int part = lane % 16;
    const int64_t row_bytes = p.cols / 2;
    const uint8_t *base[2] = {p.codes + row_of(0) * row_bytes, p.codes + row_of(8) * row_bytes};
    uint32_t offset[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
        offset[i] = (uint32_t)((row_of(lane / 16 + 2 * i) - row_of(i < 4 ? 0 : 8)) * row_bytes);
    // its part of the scales' wide copies
    constexpr int kWide = kPer * 2 < 16 ? kPer * 2 : 16, kWideLanes = kRows * kPer * 2 / kWide;
    const int64_t wide = row_of(lane * kRows / kWideLanes % kRows) * groups + lane % (kWideLanes / kRows) * (kWide / 2);

    auto issue = [&](int c, int slot) {
        if (c < c1) {
            const uint32_t dst = my_ring + slot * St::kBytes, code_dst = dst + (lane / 16) * kRowBytes + part * 16;
            // (past the last column any codes will do: x is 0 there)
            const int at = c * (kChunk / 2) + (c * kChunk + part * 32 < p.cols ? part * 16 : 0);
            const uint8_t *s[2] = {base[0] + at, base[1] + at};
#pragma unroll
            for (int i = 0; i < 8; ++i) copy_async16(code_dst + 2 * i * kRowBytes, s[i / 4] + offset[i], true);
            const uint32_t scale_dst = dst + kRows * kRowBytes;
            if (q.scales_by > 4) {
                if (lane < kWideLanes)
#pragma unroll
                    for (int w = 0; w < (MINS ? 2 : 1); ++w)
                        asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(scale_dst + w * St::kScaleBytes + lane * kWide),
                                     "l"((w ? p.mins : p.scales) + wide + c * kPer), "n"(kWide)
                                     : "memory");
            } else {
                // pairs of scales, zeros past the last group
#pragma unroll
                for (int i = 0; i < kPer / 4; ++i) {
                    const int pair = i * 32 + lane, r = pair / (kPer / 2), j = pair % (kPer / 2) * 2, at = c * kPer + j;
                    const int64_t from = row_of(r) * groups + at;
#pragma unroll
                    for (int w = 0; w < (MINS ? 2 : 1); ++w) {
                        const __half *f = w ? p.mins : p.scales;
                        const uint32_t to = scale_dst + w * St::kScaleBytes + pair * 4;
                        if (q.scales_by == 4) {
                            copy_async4(to, at < groups ? f + from : f, at < groups);
                        } else {
                            const uint32_t lo = at < groups ? __half_as_ushort(f[from]) : 0u;
                            const uint32_t hi = at + 1 < groups ? __half_as_ushort(f[from + 1]) : 0u;
                            asm volatile("st.shared.u32 [%0], %1;" ::"r"(to), "r"(lo | hi << 16) : "memory");
                        }
                    }
                }
            }
        }
        copy_commit();
    };

    // this block's columns of x as prepare_kernel leaves them, with powers of two of their own
    auto own_x = [&](auto type) {
        using T = decltype(type);
        float *sx = reinterpret_cast<float *>(xseg);
        uint8_t *xs = reinterpret_cast<uint8_t *>(sx) + sum_bytes;
        const int live = min(q.x_cols, q.x_pad - c0 * kChunk), per_row = live / 8;       // (whole warps: 64 octets a chunk)
        uint4 v[kOwnOctets];
        // octets [token][per_row] in turn
        int tok = 0, o = threadIdx.x;
        auto wrap = [&] {
            for (; o >= per_row; o -= per_row) ++tok;
        };
        wrap();
#pragma unroll
        for (int j = 0; j < kOwnOctets; ++j, o += 32 * kWarps, wrap()) {
            const int col = c0 * kChunk + o * 8;
            v[j] = uint4{0, 0, 0, 0};
            if (tok < nt && col < p.cols) v[j] = *reinterpret_cast<const uint4 *>(static_cast<const T *>(p.x) + tok * p.x_stride + col);
        }
        tok = 0, o = threadIdx.x, wrap();
#pragma unroll
        for (int j = 0; j < kOwnOctets; ++j, o += 32 * kWarps, wrap()) {
            if (tok >= nt) break;
            const unsigned m = __reduce_max_sync(~0u, octet_largest(v[j]));
            if (lane == 0) atomicMax(&largest[tok], m);
        }
        __syncthreads();
        tok = 0, o = threadIdx.x, wrap();
#pragma unroll
        for (int j = 0; j < kOwnOctets; ++j, o += 32 * kWarps, wrap()) {
            if (tok >= nt) break;
            float sum;
            *reinterpret_cast<uint4 *>(xs + tok * x_row_bytes(q.x_cols) + o * 16) =
                octet_convert<T>(v[j], power_of_two(power_for<T>(largest[tok])), sum);
#pragma unroll
            for (int d = 1; d < G / 8; d *= 2) sum += __shfl_xor_sync(~0u, sum, d);
            if (o % (G / 8) == 0) sx[o / (G / 8) * (8 * NT) + tok] = group_sum<MINS>(sum);
        }
        if (threadIdx.x < nt) unscale[threadIdx.x] = power_of_two(-power_for<T>(largest[threadIdx.x]));
    };

    // a prepared segment on its way to shared memory
    auto issue_x = [&](int seg, int buffer) {
        const uint32_t dst = smem_addr(xseg) + buffer * seg_bytes;
        const int live = min(q.x_cols, q.x_pad - seg * kChunk), per_row = live / 8;
        const uint8_t *sums = q.prepared + (size_t)8 * NT * q.x_pad * 2 + (size_t)seg * kPer * 8 * NT * 4;
        for (int i = threadIdx.x; i < live / G * 2 * NT; i += 32 * kWarps) copy_async16(dst + i * 16, sums + i * 16, true);
        for (int tok = warp; tok < nt; tok += kWarps)
            for (int o = lane; o < per_row; o += 32)
                copy_async16(dst + sum_bytes + tok * x_row_bytes(q.x_cols) + o * 16,
                             q.prepared + ((size_t)tok * q.x_pad + seg * kChunk + o * 8) * 2, true);
    };

    float y[NT][4] = {};
    int next = c0 + wk, slot = 0;                                  // the next chunk to fetch
#pragma unroll
    for (int i = 0; i < kStages - 1; ++i, next += WK) issue(next, i);
    if (!q.prepared) {
        if (threadIdx.x < 8 * NT) largest[threadIdx.x] = 0;
        __syncthreads();
        if (p.half) own_x(__half{});
        else own_x(__nv_bfloat16{});
    } else {
        wait_before();
        issue_x(c0, 0);
    }
    copy_commit();
    if (q.prepared && threadIdx.x < nt)
        unscale[threadIdx.x] = reinterpret_cast<const float *>(
            q.prepared + (size_t)8 * NT * q.x_pad * 2)[(size_t)q.x_pad / G * 8 * NT + threadIdx.x];

    int flip = 0;
    for (int seg = c0; seg < c1; seg += q.x_cols / kChunk, flip ^= 1) {
        float *sx = reinterpret_cast<float *>(xseg + flip * seg_bytes);
        uint8_t *xs = reinterpret_cast<uint8_t *>(sx) + sum_bytes;
        // (newer than the segment's copy: nothing of the first's, else a stage or more)
        if (seg != c0) copy_wait<1>();
        else if (q.prepared) copy_wait<0>();
        __syncthreads();
        if (seg + q.x_cols / kChunk < c1) issue_x(seg + q.x_cols / kChunk, flip ^ 1);
        copy_commit();
        const int seg_end = min(seg + q.x_cols / kChunk, c1);
        for (int c = seg + wk; c < seg_end; c += WK) {
            // (the segment's first stage: the next segment's copy is newer too)
            if (c == seg + wk && !q.prepared) copy_wait<kStages>();
            else if (c == seg + wk) copy_wait<kStages - 1>();
            else copy_wait<kStages - 2>();
            __syncwarp();
            issue(next, slot == 0 ? kStages - 1 : slot - 1);
            next += WK;
            const uint8_t *st = ring + (warp * kStages + slot) * St::kBytes;
            slot = slot == kStages - 1 ? 0 : slot + 1;
            // matrices of a load: rows 0-7 and 8-15 of 32 columns, and of the next 32
            const uint32_t mat = smem_addr(st) + lane % 16 * kRowBytes + lane / 16 * 16;
            constexpr int kVec = kPer * 2 < 16 ? 1 : kPer * 2 / 16;
            union Scales {
                uint4 v[kVec];
                uint2 d;
                __half h[kPer < 8 ? 8 : kPer];
            } sc[2], mn[MINS ? 2 : 1];
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const uint8_t *f = st + kRows * kRowBytes + (g + 8 * r) * kPer * 2;
                if constexpr (kPer == 4) {
                    sc[r].d = *reinterpret_cast<const uint2 *>(f);
                    if (MINS) mn[r].d = *reinterpret_cast<const uint2 *>(f + St::kScaleBytes);
                } else {
#pragma unroll
                    for (int j = 0; j < kVec; ++j) {
                        sc[r].v[j] = reinterpret_cast<const uint4 *>(f)[j];
                        if (MINS) mn[r].v[j] = reinterpret_cast<const uint4 *>(f + St::kScaleBytes)[j];
                    }
                }
            }
            const uint8_t *xb[NT];
            const float *sb = sx + (c - seg) * kPer * (8 * NT) + 2 * t;
#pragma unroll
            for (int n = 0; n < NT; ++n)
                xb[n] = xs + min(8 * n + g, nt - 1) * x_row_bytes(q.x_cols) + (c - seg) * kChunk * 2 + t * 16;
            // (the next operands are on their way while these are multiplied)
            uint32_t w[2][4];
            uint4 b[2][NT];
            auto fetch_w = [&](int at) { load_matrices(w[at / 2 % 2], mat + at * 16); };
            auto fetch_x = [&](int at) {
#pragma unroll
                for (int n = 0; n < NT; ++n) b[at % 2][n] = *reinterpret_cast<const uint4 *>(xb[n] + at * 64);
            };
            fetch_w(0);
            fetch_x(0);
#pragma unroll
            for (int j = 0; j < kPer; ++j) {
                float acc[NT][4];
                float2 sums[NT];
#pragma unroll
                for (int n = 0; n < NT; ++n) sums[n] = *reinterpret_cast<const float2 *>(sb + j * (8 * NT) + 8 * n);
#pragma unroll
                for (int u = 0; u < G / 32; ++u) {
                    const int at = j * (G / 32) + u;
                    if (at % 2 == 0 && at + 2 < kChunk / 32) fetch_w(at + 2);
                    if (at + 1 < kChunk / 32) fetch_x(at + 1);
                    const uint32_t lo = 0x000f000fu, hi = 0x00f000f0u;
                    const uint32_t a = w[at / 2 % 2][at % 2 * 2], d = w[at / 2 % 2][at % 2 * 2 + 1], a8 = a >> 8, d8 = d >> 8;
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        const float start[4] = {MINS ? 0.0f : sums[n].x, MINS ? 0.0f : sums[n].y,
                                                MINS ? 0.0f : sums[n].x, MINS ? 0.0f : sums[n].y};
                        const uint4 &x = b[at % 2][n];
                        if (u == 0) multiply(acc[n], a & lo, d & lo, a & hi, d & hi, x.x, x.y, start);
                        else multiply(acc[n], a & lo, d & lo, a & hi, d & hi, x.x, x.y, acc[n]);
                        multiply(acc[n], a8 & lo, d8 & lo, a8 & hi, d8 & hi, x.z, x.w, acc[n]);
                    }
                }
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const float s = __half2float(sc[r].h[j]), z = MINS ? __half2float(mn[MINS ? r : 0].h[j]) : 0.0f;
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            float v = __fmaf_rn(s, acc[n][2 * r + e], y[n][2 * r + e]);
                            if (MINS) v = __fmaf_rn(z, e ? sums[n].y : sums[n].x, v);
                            y[n][2 * r + e] = v;
                        }
                }
            }
        }
    }
    float largest_unscale = 0;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float f = unscale[min(8 * n + 2 * t + e % 2, nt - 1)];
            y[n][e] = y[n][e] * 0x1p24f * f;
            largest_unscale = fmaxf(largest_unscale, f);
        }
    // (no power of two of finite values is as large; one of the warps that share the rows looks)
    if (largest_unscale > 0x1p113f) {
#pragma unroll 1
        for (int i = 0; i < 4 * NT; ++i) {
            const int tok = min(8 * (i / 4) + 2 * t + i % 2, nt - 1);
            if (!(unscale[tok] > 0x1p113f)) continue;
            const int64_t row = row_of(g + 8 * (i / 2 % 2));
            const float sum = wk ? 0.0f
                                 : sum_not_finite(p.codes + row * (p.cols / 2), p.scales + row * groups, MINS ? p.mins + row * groups : nullptr,
                                                  static_cast<const uint16_t *>(p.x) + tok * p.x_stride, p.half, G, c0 * kChunk,
                                                  min(c1 * kChunk, p.cols));
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (4 * n + e == i) y[n][e] = sum;
        }
    }

    if (WK == 1 && q.split == 1) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                // rows g and g + 8: two outputs, or what gates and what is gated
                const int tok = 8 * n + 2 * t + e % 2, r = first + g + (p.gated ? 0 : 8 * (e / 2));
                if (tok >= nt || r >= q.outs || (p.gated && e >= 2)) continue;
                finish(p, tok, r, y[n][e], y[n][e | 2]);
            }
        return;
    }
    // join: the block's warps, then the cluster's blocks, in that order
    copy_wait<0>();
    __syncthreads();
    float *red = reinterpret_cast<float *>(ring);                  // [WK][RB][8 NT]
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            red[(wk * RB + wr * kRows + g + 8 * (e / 2)) * (8 * NT) + 8 * n + 2 * t + e % 2] = y[n][e];
    __syncthreads();
    if (WK > 1) {
        for (int i = threadIdx.x; i < RB * 8 * NT; i += 32 * kWarps) {
            float v = red[i];
            for (int k = 1; k < WK; ++k) v += red[k * RB * 8 * NT + i];
            red[i] = v;
        }
        __syncthreads();
    }
    if (q.split > 1) cluster_barrier();
    const uint32_t mine = smem_addr(red);
    auto joined = [&](int i) {
        if (q.split == 1) return red[i];
        float v = 0;
        for (int k = 0; k < q.split; ++k) v += peer_load(peer_addr(mine + 4 * i, k));
        return v;
    };
    const int rows = p.gated ? RB / 2 : RB, out0 = block * rows;
    for (int i = threadIdx.x + rank * 32 * kWarps; i < rows * 8 * NT; i += 32 * kWarps * q.split) {
        // rows vary fastest: neighbouring outputs
        const int r = i % rows, tok = i / rows;
        if (tok >= nt || out0 + r >= q.outs) continue;
        if (p.gated) {
            const int at = (r / 8 * 16 + r % 8) * (8 * NT) + tok;
            finish(p, tok, out0 + r, joined(at), joined(at + 8 * 8 * NT));
        } else {
            finish(p, tok, out0 + r, joined(r * (8 * NT) + tok), 0.0f);
        }
    }
    if (q.split > 1) cluster_barrier();                            // (peers may still read)
}

template <int G, bool MINS, int NT> int launch_few(const FewParams &q, const FewPlan &f, int dev, cudaStream_t s)
{
    static std::atomic<uint64_t> ready{0};                         // devices that have the attribute set
    auto kernel = few_kernel<G, MINS, NT>;
    if (!(ready.load(std::memory_order_relaxed) >> dev & 1)) {
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemPerSm - 2048);
        if (e != cudaSuccess) return cuda_status(e);
        ready.fetch_or(1ull << dev, std::memory_order_relaxed);
    }
    if (q.prepared) {
        auto prepare = q.m.half ? prepare_kernel<__half, G, MINS, NT> : prepare_kernel<__nv_bfloat16, G, MINS, NT>;
        if (int st = launch<FewParams>(prepare, dim3((unsigned)q.m.tokens), 512, 0, 1, false, s, q)) return st;
    }
    const int rb = (q.m.gated ? 8 : 16) * (kWarps / q.wk);
    const unsigned blocks = (unsigned)((q.outs + rb - 1) / rb * f.split);
    return launch<FewParams>(kernel, dim3(blocks), 32 * kWarps, f.smem, f.split, q.prepared != nullptr, s, q);
}

template <int G> int launch_few_group(const FewParams &q, const FewPlan &f, int dev, cudaStream_t s)
{
    if (q.m.mins)
        return f.nt == 1 ? launch_few<G, true, 1>(q, f, dev, s) : launch_few<G, true, 2>(q, f, dev, s);
    return f.nt == 1 ? launch_few<G, false, 1>(q, f, dev, s) : launch_few<G, false, 2>(q, f, dev, s);
}

// The launch of a prompt (quant_matmul_many.cu).
struct ManyPlan {
    int tile, tiles, row_tiles, split, stages, depth;
    int whole, rest_split;                 // blocks unsplit, before the rest: whole turns (0: all alike)
    size_t image, workspace;
};
ManyPlan plan_many(int outs, bool gated, int cols, int tokens, int sms);
int launch_many(const MatmulParams &m, const ManyPlan &f, void *workspace, int outs, int dev, cudaStream_t s);

// One translation unit per group size.
int launch_few_32(const FewParams &q, const FewPlan &f, int dev, cudaStream_t s);
int launch_few_64(const FewParams &q, const FewPlan &f, int dev, cudaStream_t s);
int launch_few_128(const FewParams &q, const FewPlan &f, int dev, cudaStream_t s);

}  // namespace e2ops
