// quant_matmul.cuh -- the kernel of e2_quant_matmul for a few tokens, and what its
// translation units share.
#pragma once

#include <atomic>
#include <type_traits>

#include "ops_mma.cuh"

namespace e2ops {

struct MatmulParams {
    int rows, cols, group, tokens, gated;
    const uint8_t *codes;
    const __half *scales, *mins;
    const void *x, *residual;
    void *y;
    int64_t x_stride, residual_stride, y_stride;
};

// ---- few tokens --------------------------------------------------------------
//
// Bound by reading the weights.  y^T = W x^T on the warp-level tensor cores: the
// weights are the 16-row operand, eight tokens the other, so a code is unpacked
// once and no row is padding.  A warp owns 32 rows and streams them
// through a ring of its own in shared memory (asynchronous copies of whole 128-byte
// lines, no block barrier), three stages of 256 columns deep.  Codes less 8 are
// exact in 16 bits, so the tensor cores' sums hold no rounded weight; each group's sum
// is scaled in 32 bits.  x lies in shared memory in the order of the codes'
// nibbles, a segment of columns at a time.  Few rows are split over columns, among a block's
// warps (WK) and the blocks of a cluster, and joined in a fixed order.

constexpr int kChunk = 256;                  // columns of a stage
constexpr int kStages = 3;
constexpr int kRowBytes = kChunk / 2 + 16;   // (a stage's rows 16 bytes apart in banks)
constexpr int kWarps = 4;

constexpr int kSmemPerSm = 227 * 1024;

// The launch of `tokens` tokens: how the columns are split.
struct FewPlan {
    int nt, wk, split, x_cols;
    size_t smem;
};

template <int G, bool MINS> struct Stage {
    static constexpr int kPer = kChunk / G;                                 // scales of a row
    static constexpr int kScaleBytes = 32 * kPer * 2;
    static constexpr int kBytes = 32 * kRowBytes + kScaleBytes * (MINS ? 2 : 1);
};

struct FewParams {
    MatmulParams m;
    int outs, wk, split, x_shift, x_cols, scales_aligned;
};

// The bytes of x in shared memory, per token and segment (rows half a 128-byte line apart in banks).
__host__ __device__ constexpr int x_row_bytes(int cols) { return cols * 2 + 64; }

__device__ __forceinline__ uint32_t peer_addr(uint32_t addr, int rank)
{
    uint32_t d;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(d) : "r"(addr), "r"(rank));
    return d;
}
__device__ __forceinline__ float peer_load(uint32_t addr)
{
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ void cluster_barrier()
{
    asm volatile("barrier.cluster.arrive.release;\nbarrier.cluster.wait.acquire;" ::: "memory");
}

template <class T>
__device__ __forceinline__ void finish(const MatmulParams &p, int token, int row, float a, float b)
{
    float y = p.gated ? a / (1.0f + expf(-a)) * b : a;
    if (p.residual) y += to_float(static_cast<const T *>(p.residual)[token * p.residual_stride + row]);
    static_cast<T *>(p.y)[token * p.y_stride + row] = from_float<T>(y);
}

template <class T, int G, bool MINS, int NT>
__global__ void __launch_bounds__(32 * kWarps, NT == 4 ? 2 : 3) few_kernel(const FewParams q)
{
    constexpr bool BF = sizeof(T) == 2 && !std::is_same<T, __half>::value;
    using St = Stage<G, MINS>;
    constexpr int kPer = St::kPer;
    const int WK = q.wk, RB = 32 * (kWarps / WK);
    extern __shared__ __align__(128) uint8_t smem[];
    const MatmulParams &p = q.m;
    const int t0 = blockIdx.y * 8 * NT, nt = min(8 * NT, p.tokens - t0);
    uint8_t *ring = smem;
    uint8_t *xs = smem + kWarps * kStages * St::kBytes;
    float *sx = reinterpret_cast<float *>(xs + nt * x_row_bytes(q.x_cols));
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, wr = warp / WK, wk = warp % WK;
    const int g = lane / 4, t = lane % 4;
    const int rank = blockIdx.x % q.split, block = blockIdx.x / q.split;
    const int chunks = (p.cols + kChunk - 1) / kChunk;
    const int c0 = (int)((int64_t)chunks * rank / q.split), c1 = (int)((int64_t)chunks * (rank + 1) / q.split);
    const int groups = p.cols / G;

    // rows of this warp: gated, 16 rows that gate and the 16 that they gate
    const int first = block * (p.gated ? RB / 2 : RB) + wr * (p.gated ? 16 : 32);
    const int64_t jump = p.gated ? (int64_t)q.outs - 16 : 0;      // from ring row 16 on
    auto source_row = [&](int r) { return (int64_t)first + r + (r >= 16 ? jump : 0); };
    auto row_valid = [&](int r) { return first + (p.gated ? r % 16 : r) < q.outs; };

    const uint32_t my_ring = smem_addr(ring) + warp * kStages * St::kBytes;
    // lane l copies 16 bytes (l % 8) of rows l / 8 + 4 i
    const int part = lane % 8;
    unsigned valid = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) valid |= (unsigned)row_valid(lane / 8 + 4 * i) << i;
    const int64_t row_bytes = p.cols / 2;
    const uint8_t *src = p.codes + source_row(lane / 8) * row_bytes + part * 16;
    const bool my_row = row_valid(lane);
    const __half *my_scales = p.scales + source_row(lane) * groups, *my_mins = MINS ? p.mins + source_row(lane) * groups : nullptr;

    auto issue = [&](int c, int slot) {
        if (c < c1) {
            const uint32_t dst = my_ring + slot * St::kBytes;
            const bool in = c * kChunk + part * 32 < p.cols;
            const uint8_t *s = src + (int64_t)c * (kChunk / 2);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const bool take = in && (valid >> i & 1);
                const int64_t at = 4 * i * row_bytes + (i >= 4 ? jump * row_bytes : 0);
                copy_async16(dst + (lane / 8 + 4 * i) * kRowBytes + part * 16, take ? s + at : p.codes, take);
            }
            // a lane per row: the chunk's scales
            const uint32_t sd = dst + 32 * kRowBytes + lane * kPer * 2;
            if (q.scales_aligned) {
#pragma unroll
                for (int w = 0; w < (MINS ? 2 : 1); ++w) {
                    const __half *f = (w ? my_mins : my_scales) + c * kPer;
                    const bool take = my_row;
                    asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(sd + w * St::kScaleBytes),
                                 "l"(take ? f : p.scales), "n"(kPer * 2), "r"(take ? kPer * 2 : 0)
                                 : "memory");
                }
            } else {
#pragma unroll
                for (int w = 0; w < (MINS ? 2 : 1); ++w)
#pragma unroll
                    for (int j = 0; j < kPer; ++j) {
                        const int at = c * kPer + j;
                        uint16_t v = 0;
                        if (my_row && at < groups) v = __half_as_ushort((w ? my_mins : my_scales)[at]);
                        asm volatile("st.shared.u16 [%0], %1;" ::"r"(sd + w * St::kScaleBytes + 2 * j), "h"(v) : "memory");
                    }
            }
        }
        copy_commit();
    };

    float y[2][NT][4] = {};
    int next = c0 + wk;                                            // the next chunk to fetch
#pragma unroll
    for (int i = 0; i < kStages - 1; ++i, next += WK) issue(next, i);
    int slot = 0;

    const int octets = q.x_cols / 8;
    for (int seg = c0; seg < c1; seg += q.x_cols / kChunk) {
        __syncthreads();
        // x: octets in the codes' order, zeros past the last column, groups' sums beside
        const int total = nt * octets;
        for (int base = 0; base < total; base += 8 * 32 * kWarps) {
            uint4 v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int at = base + i * 32 * kWarps + threadIdx.x;
                const int tok = at >> q.x_shift, o = at & (octets - 1), col = seg * kChunk + o * 8;
                v[i] = uint4{0, 0, 0, 0};
                if (at < total && col < p.cols)
                    v[i] = *reinterpret_cast<const uint4 *>(static_cast<const T *>(p.x) + (t0 + tok) * p.x_stride + col);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int at = base + i * 32 * kWarps + threadIdx.x;
                const int tok = at >> q.x_shift, o = at & (octets - 1);
                if (MINS) {
                    float e[8], sum = 0;
                    unpack8<T>(v[i], e);
#pragma unroll
                    for (int j = 0; j < 8; ++j) sum += e[j];
#pragma unroll
                    for (int d = 1; d < G / 8; d *= 2) sum += __shfl_xor_sync(~0u, sum, d);
                    if (at < total && o % (G / 8) == 0) sx[tok * (q.x_cols / G) + o / (G / 8)] = sum;
                }
                if (at < total) {
                    uint4 w;
                    w.x = __byte_perm(v[i].x, v[i].z, 0x5410);
                    w.y = __byte_perm(v[i].x, v[i].z, 0x7632);
                    w.z = __byte_perm(v[i].y, v[i].w, 0x5410);
                    w.w = __byte_perm(v[i].y, v[i].w, 0x7632);
                    *reinterpret_cast<uint4 *>(xs + tok * x_row_bytes(q.x_cols) + o * 16) = w;
                }
            }
        }
        __syncthreads();
        const int seg_end = min(seg + q.x_cols / kChunk, c1);
        for (int c = seg + wk; c < seg_end; c += WK) {
            copy_wait<kStages - 2>();
            __syncwarp();
            issue(next, slot == 0 ? kStages - 1 : slot - 1);
            next += WK;
            const uint32_t st = my_ring + slot * St::kBytes;
            slot = slot == kStages - 1 ? 0 : slot + 1;
            // matrix i of a load: ring rows 8 i ..
            const uint32_t mat = st + lane * kRowBytes;
            __half2 sc[4][(kPer + 1) / 2], mn[4][MINS ? (kPer + 1) / 2 : 1];
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int j = 0; j < kPer / 2; ++j) {
                    const uint8_t *f = ring + (st - smem_addr(ring)) + 32 * kRowBytes + (g + 8 * r) * kPer * 2 + 4 * j;
                    sc[r][j] = *reinterpret_cast<const __half2 *>(f);
                    if (MINS) mn[r][j] = *reinterpret_cast<const __half2 *>(f + St::kScaleBytes);
                }
            const uint8_t *xb[NT];
#pragma unroll
            for (int n = 0; n < NT; ++n)
                xb[n] = xs + min(8 * n + g, nt - 1) * x_row_bytes(q.x_cols) + (c - seg) * kChunk * 2 + t * 16;
#pragma unroll
            for (int j = 0; j < kPer; ++j) {
                float acc[2][NT][4] = {};
#pragma unroll
                for (int u = 0; u < G / 32; ++u) {
                    const int at = j * (G / 32) + u;
                    uint32_t w[4];
                    load_matrices(w, mat + at * 16);
                    uint4 b[NT];
#pragma unroll
                    for (int n = 0; n < NT; ++n) b[n] = *reinterpret_cast<const uint4 *>(xb[n] + at * 64);
#pragma unroll
                    for (int m = 0; m < 2; ++m) {
                        uint32_t a[4], d[4];
                        centred_codes<BF>(w[2 * m], a);
                        centred_codes<BF>(w[2 * m + 1], d);
#pragma unroll
                        for (int n = 0; n < NT; ++n) {
                            multiply<BF>(acc[m][n], a[0], d[0], a[1], d[1], b[n].x, b[n].y);
                            multiply<BF>(acc[m][n], a[2], d[2], a[3], d[3], b[n].z, b[n].w);
                        }
                    }
                }
#pragma unroll
                for (int m = 0; m < 2; ++m)
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const __half2 s2 = sc[2 * m + r][j / 2];
                        const float s = __half2float(j % 2 ? __high2half(s2) : __low2half(s2));
                        float z = 0;
                        if (MINS) {
                            const __half2 m2 = mn[2 * m + r][j / 2];
                            z = __fmaf_rn(8.0f, s, __half2float(j % 2 ? __high2half(m2) : __low2half(m2)));
                        }
#pragma unroll
                        for (int n = 0; n < NT; ++n)
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                float v = __fmaf_rn(s, acc[m][n][2 * r + e], y[m][n][2 * r + e]);
                                if (MINS)
                                    v = __fmaf_rn(z, sx[min(8 * n + 2 * t + e, nt - 1) * (q.x_cols / G) + (c - seg) * kPer + j], v);
                                y[m][n][2 * r + e] = v;
                            }
                    }
            }
        }
    }

    if (WK == 1 && q.split == 1) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int tok = 8 * n + 2 * t + e % 2, r = first + g + 8 * (e / 2);
                if (tok >= nt) continue;
                if (p.gated) {
                    if (r < q.outs) finish<T>(p, t0 + tok, r, y[0][n][e], y[1][n][e]);
                } else {
                    if (r < q.outs) finish<T>(p, t0 + tok, r, y[0][n][e], 0.0f);
                    if (r + 16 < q.outs) finish<T>(p, t0 + tok, r + 16, y[1][n][e], 0.0f);
                }
            }
        return;
    }
    // join: the block's warps, then the cluster's blocks, in that order
    copy_wait<0>();
    __syncthreads();
    float *red = reinterpret_cast<float *>(ring);                  // [WK][RB][8 NT]
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                red[(wk * RB + wr * 32 + 16 * m + g + 8 * (e / 2)) * (8 * NT) + 8 * n + 2 * t + e % 2] = y[m][n][e];
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
    auto total = [&](int i) {
        if (q.split == 1) return red[i];
        float v = 0;
        for (int k = 0; k < q.split; ++k) v += peer_load(peer_addr(mine + 4 * i, k));
        return v;
    };
    const int rows = p.gated ? RB / 2 : RB, base = block * rows;
    for (int i = threadIdx.x + rank * 32 * kWarps; i < rows * 8 * NT; i += 32 * kWarps * q.split) {
        // rows vary fastest: neighbouring outputs
        const int r = i % rows, tok = i / rows;
        if (tok >= nt || base + r >= q.outs) continue;
        if (p.gated) {
            const int at = (r / 16 * 32 + r % 16) * (8 * NT) + tok;
            finish<T>(p, t0 + tok, base + r, total(at), total(at + 16 * 8 * NT));
        } else {
            finish<T>(p, t0 + tok, base + r, total(r * (8 * NT) + tok), 0.0f);
        }
    }
    if (q.split > 1) cluster_barrier();                            // (peers may still read)
}

template <class T, int G, bool MINS, int NT>
int launch_few(const FewParams &q, const FewPlan &f, int dev, cudaStream_t s)
{
    static std::atomic<uint64_t> ready{0};                         // devices that have the attribute set
    auto kernel = few_kernel<T, G, MINS, NT>;
    if (!(ready.load(std::memory_order_relaxed) >> dev & 1)) {
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemPerSm);
        if (e != cudaSuccess) return cuda_status(e);
        ready.fetch_or(1ull << dev, std::memory_order_relaxed);
    }
    const int rb = (q.m.gated ? 16 : 32) * (kWarps / q.wk);
    cudaLaunchAttribute at{};
    at.id = cudaLaunchAttributeClusterDimension;
    at.val.clusterDim.x = (unsigned)f.split;
    at.val.clusterDim.y = at.val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)((q.outs + rb - 1) / rb * f.split), (unsigned)((q.m.tokens + 8 * NT - 1) / (8 * NT)));
    cfg.blockDim = dim3(32 * kWarps);
    cfg.dynamicSmemBytes = f.smem;
    cfg.stream = s;
    cfg.attrs = &at;
    cfg.numAttrs = f.split > 1 ? 1 : 0;
    return cuda_status(cudaLaunchKernelEx(&cfg, kernel, q));
}

template <class T, int G, bool MINS> int launch_group(const FewParams &q, const FewPlan &f, int dev, cudaStream_t s)
{
    return f.nt == 1   ? launch_few<T, G, MINS, 1>(q, f, dev, s)
           : f.nt == 2 ? launch_few<T, G, MINS, 2>(q, f, dev, s)
                       : launch_few<T, G, MINS, 4>(q, f, dev, s);
}

template <class T> int launch_type(const FewParams &q, const FewPlan &f, int dev, cudaStream_t s)
{
    const bool mins = q.m.mins != nullptr;
    if (q.m.group == 32) return mins ? launch_group<T, 32, true>(q, f, dev, s) : launch_group<T, 32, false>(q, f, dev, s);
    if (q.m.group == 64) return mins ? launch_group<T, 64, true>(q, f, dev, s) : launch_group<T, 64, false>(q, f, dev, s);
    return mins ? launch_group<T, 128, true>(q, f, dev, s) : launch_group<T, 128, false>(q, f, dev, s);
}



// One translation unit per type of x.
int launch_few_f16(const FewParams &q, const FewPlan &f, int dev, cudaStream_t s);
int launch_few_bf16(const FewParams &q, const FewPlan &f, int dev, cudaStream_t s);

}  // namespace e2ops
