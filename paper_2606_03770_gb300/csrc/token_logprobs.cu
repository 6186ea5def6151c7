// token_logprobs.cu -- e2_token_logprobs: log probabilities of given tokens,
// entropy and top alternatives of rows of logits.
#include "ops_mma.cuh"

namespace e2ops {
namespace {

// One pass over a row, by a block or, where there are few rows, by the blocks of a
// cluster; bound by reading it.  A thread keeps the maximum m of what it has read, sum
// e and sum e (x - m), e = exp(x - m), all in 32 bits, and brings them to a new maximum
// when one comes.  The differences are taken before the exponent's scaling, so that
// logits of any size keep their digits.
//
// Alternatives: a warp keeps the best so far sorted over its lanes, (value, then lower
// index), and looks at eight elements a lane only when some maximum of eight beats its
// last one, or what any warp of the block has as its last.  The first elements are let in
// through the `top`-th largest of the lanes' maxima, which `top` of them reach.

constexpr int kMostThreads = 512, kMostWarps = kMostThreads / 32;
constexpr float kLog2e = 1.4426950408889634f, kNegligible = -1e30f;

struct LogprobParams {
    int rows, vocab, top, split;
    const void *logits;
    int64_t stride;
    const int32_t *tokens;
    float *logprob, *entropy, *values;
    int32_t *ids;
};

struct Sums {
    float m, s, u;                       // maximum (-inf: nothing), sum e, sum e (x - m)
};

__device__ __forceinline__ float power2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float max_or_nan(float a, float b)
{
    float y;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
    return y;
}

// a's sums brought to the maximum m >= a.m.
__device__ __forceinline__ Sums rebase(const Sums &a, float m)
{
    if (a.m == -INFINITY) return Sums{m, 0.0f, 0.0f};
    const float d = a.m - m, f = power2(d * kLog2e);
    // (u + d s before the factor: both shrink together)
    return Sums{m, a.s * f, f == 0.0f ? 0.0f : f * __fmaf_rn(d, a.s, a.u)};
}
__device__ __forceinline__ Sums merge(const Sums &a, const Sums &b)
{
    const float m = fmaxf(a.m, b.m);
    const Sums x = rebase(a, m), y = rebase(b, m);
    return Sums{m, x.s + y.s, x.u + y.u};
}

// Floats in the order of unsigned integers.
__device__ __forceinline__ unsigned ordered(float x)
{
    const unsigned b = __float_as_uint(x);
    return b >> 31 ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float unordered(unsigned o) { return __uint_as_float(o >> 31 ? o & 0x7fffffffu : ~o); }
// The float below a finite one (below either zero: the largest negative one).
__device__ __forceinline__ float below(float x) { return x == 0.0f ? __uint_as_float(0x80000001u) : unordered(ordered(x) - 1); }

// A warp's best, one per lane, largest first.
struct Best {
    float v;
    int id;
    __device__ void clear() { v = -INFINITY, id = 0x7fffffff; }
    // a candidate, the same in all lanes
    __device__ void insert(float x, int at, int lane)
    {
        const bool before = v > x || (v == x && id < at);
        const float pv = __shfl_up_sync(~0u, v, 1);
        const int pid = __shfl_up_sync(~0u, id, 1);
        const int place = __popc(__ballot_sync(~0u, before));
        if (lane == place) v = x, id = at;
        else if (lane > place) v = pv, id = pid;
    }
};

template <class T, bool TOP> __global__ void __launch_bounds__(kMostThreads, 3) logprob_kernel(const LogprobParams p)
{
    constexpr int kVec = 16 / sizeof(T), kLoads = 8 / kVec;       // eight elements a lane: one load, or two
    __shared__ Sums warp_sums[kMostWarps];
    __shared__ int any_bad[kMostWarps];
    __shared__ unsigned floor_bits;                               // what some warp has as its last
    __shared__ float list_v[kMostWarps][E2_MAX_TOP];
    __shared__ int list_id[kMostWarps][E2_MAX_TOP];
    __shared__ Sums block_sums;
    __shared__ int block_bad;
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, warps = blockDim.x / 32;
    const int rank = blockIdx.x % p.split, row = blockIdx.x / p.split;
    const T *x = static_cast<const T *>(p.logits) + row * p.stride;
    if (threadIdx.x == 0) floor_bits = ordered(-INFINITY);
    __syncthreads();

    // elements before the first 16-byte boundary, whole vectors, the rest
    const int head = min(p.vocab, (int)((16 - reinterpret_cast<uintptr_t>(x) % 16) % 16 / sizeof(T)));
    const int vectors = (p.vocab - head) / kVec, tail = head + vectors * kVec;
    const int v0 = (int)((int64_t)vectors * rank / p.split), v1 = (int)((int64_t)vectors * (rank + 1) / p.split);

    Sums a{-INFINITY, 0.0f, 0.0f};
    bool bad = false;
    Best best;
    best.clear();
    float last = -INFINITY;                                       // below it nothing is let in
    bool first = true;

    // eight elements of each lane, -inf where there are none; element j is index(j)
    auto take = [&](const float (&e)[8], auto index) {
        float m = e[0];
#pragma unroll
        for (int j = 1; j < 8; ++j) m = max_or_nan(m, e[j]);
        bad |= !(m < INFINITY);
        if (m > a.m) a = rebase(a, m);
        const float base = a.m == -INFINITY ? 0.0f : a.m;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float d = fmaxf(e[j] - base, kNegligible), w = power2(d * kLog2e);
            a.s += w;
            a.u = __fmaf_rn(w, d, a.u);
        }
        if (!TOP) return;
        if (first) {
            // the `top`-th largest of the lanes' maxima: sorted over the lanes
            float v = m;
#pragma unroll
            for (int k = 2; k <= 32; k *= 2)
#pragma unroll
                for (int j = k / 2; j; j /= 2) {
                    const float o = __shfl_xor_sync(~0u, v, j);
                    const bool up = ((lane & k) == 0) == ((lane & j) == 0);   // (larger ones to lower lanes)
                    v = up ? fmaxf(v, o) : fminf(v, o);
                }
            const float bound = __shfl_sync(~0u, v, p.top - 1);
            // (fewer lanes than that have any: again next time)
            if (bound > -INFINITY) {
                first = false;
                last = fmaxf(last, below(bound));                 // equal ones are let in
            }
        }
        if (!__any_sync(~0u, m > last)) return;
        const float others = unordered(*reinterpret_cast<volatile unsigned *>(&floor_bits));
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            unsigned b = __ballot_sync(~0u, e[j] > last && e[j] >= others);
            while (b) {
                const int from = __ffs(b) - 1;
                b &= b - 1;
                const float v = __shfl_sync(~0u, e[j], from);
                const int at = __shfl_sync(~0u, index(j), from);
                best.insert(v, at, lane);
            }
        }
        const float worst = __shfl_sync(~0u, best.v, p.top - 1);
        // (only elements of later rounds come after this: equal ones have higher indices)
        last = fmaxf(last, worst);
        if (worst > -INFINITY) {
            if (lane == 0) atomicMax(&floor_bits, ordered(worst));
            if (others > -INFINITY) last = fmaxf(last, below(others));
        }
    };

    if (rank == 0 && warp == 0 && head > 0) {
        float e[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) e[j] = -INFINITY;
        if (lane < head) e[0] = to_float(x[lane]);
        take(e, [&](int) { return lane; });
    }
    const uint4 *vec = reinterpret_cast<const uint4 *>(x + head);
    const int step = warps * 32 * kLoads;
    auto load = [&](uint4 (&w)[kLoads], int at) {
#pragma unroll
        for (int l = 0; l < kLoads; ++l)
            if (at + 32 * l + lane < v1) w[l] = __ldcs(vec + at + 32 * l + lane);
    };
    int at = v0 + warp * 32 * kLoads;
    uint4 ahead[kLoads];
    load(ahead, at);
    for (; at < v1; at += step) {
        uint4 now[kLoads];
#pragma unroll
        for (int l = 0; l < kLoads; ++l) now[l] = ahead[l];
        load(ahead, at + step);
        float e[8];
#pragma unroll
        for (int j = 0; j < 8; ++j)
            e[j] = at + 32 * (j / kVec) + lane < v1 ? to_float(reinterpret_cast<const T *>(now)[j]) : -INFINITY;
        take(e, [&](int j) { return head + (at + 32 * (j / kVec) + lane) * kVec + j % kVec; });
    }
    if (rank == p.split - 1 && warp == warps - 1 && tail < p.vocab) {
        float e[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) e[j] = -INFINITY;
        if (tail + lane < p.vocab) e[0] = to_float(x[tail + lane]);
        take(e, [&](int) { return tail + lane; });
    }

    // the warp's sums, the block's, the cluster's, in fixed orders
#pragma unroll
    for (int k = 16; k; k >>= 1)
        a = merge(a, Sums{__shfl_xor_sync(~0u, a.m, k), __shfl_xor_sync(~0u, a.s, k), __shfl_xor_sync(~0u, a.u, k)});
    bad = __any_sync(~0u, bad);
    if (lane == 0) warp_sums[warp] = a, any_bad[warp] = bad;
    if (TOP && lane < p.top) list_v[warp][lane] = best.v, list_id[warp][lane] = best.id;
    __syncthreads();
    if (warp == 0) {
        Sums total = warp_sums[0];
        int spoilt = any_bad[0];
        for (int w = 1; w < warps; ++w) total = merge(total, warp_sums[w]), spoilt |= any_bad[w];
        if (lane == 0) block_sums = total, block_bad = spoilt;
        if (TOP) {
            const float least = unordered(floor_bits);
            for (int w = 1; w < warps; ++w) {
                const float v = lane < p.top ? list_v[w][lane] : -INFINITY;
                const int id = lane < p.top ? list_id[w][lane] : 0x7fffffff;
                unsigned b = __ballot_sync(~0u, v >= least && v > -INFINITY);
                while (b) {
                    const int from = __ffs(b) - 1;
                    b &= b - 1;
                    best.insert(__shfl_sync(~0u, v, from), __shfl_sync(~0u, id, from), lane);
                }
            }
            if (p.split > 1 && lane < p.top) list_v[0][lane] = best.v, list_id[0][lane] = best.id;
        }
    }
    if (p.split > 1) {
        cluster_barrier();
        if (rank == 0 && warp == 0) {
            Sums total = block_sums;
            int spoilt = block_bad;
            const uint32_t sums_at = smem_addr(&block_sums), bad_at = smem_addr(&block_bad);
            for (int r = 1; r < p.split; ++r) {
                const uint32_t s = peer_addr(sums_at, r);
                total = merge(total, Sums{peer_load(s), peer_load(s + 4), peer_load(s + 8)});
                spoilt |= __float_as_int(peer_load(peer_addr(bad_at, r)));
                if (TOP) {
                    float v = -INFINITY;
                    int id = 0x7fffffff;
                    if (lane < p.top) {
                        v = peer_load(peer_addr(smem_addr(&list_v[0][lane]), r));
                        id = __float_as_int(peer_load(peer_addr(smem_addr(&list_id[0][lane]), r)));
                    }
                    const float worst = __shfl_sync(~0u, best.v, p.top - 1);
                    unsigned b = __ballot_sync(~0u, v >= worst && v > -INFINITY);
                    while (b) {
                        const int from = __ffs(b) - 1;
                        b &= b - 1;
                        best.insert(__shfl_sync(~0u, v, from), __shfl_sync(~0u, id, from), lane);
                    }
                }
            }
            if (lane == 0) block_sums = total, block_bad = spoilt;
        }
        cluster_barrier();                                        // (peers have been read)
    }
    if (rank != 0 || warp != 0) return;
    __syncwarp();
    const Sums total = block_sums;
    const bool spoilt = block_bad, empty = total.m == -INFINITY;
    const float nan = __int_as_float(0x7fc00000), ln = empty ? 0.0f : logf(total.s), lse = empty ? 0.0f : total.m + ln;
    if (lane == 0) {
        if (p.entropy) p.entropy[row] = spoilt ? nan : empty ? 0.0f : ln - total.u / total.s;
        if (p.logprob) {
            const int y = p.tokens[row];
            p.logprob[row] = spoilt || y < 0 || y >= p.vocab ? nan : to_float(x[y]) - lse;
        }
    }
    if (TOP && lane < p.top) {
        const bool none = !(best.v > -INFINITY);
        p.values[(int64_t)row * p.top + lane] = spoilt ? nan : none ? -INFINITY : best.v - lse;
        p.ids[(int64_t)row * p.top + lane] = spoilt || none ? -1 : best.id;
    }
}

// Rows fewer than two per multiprocessor are split over clusters of up to eight.
template <class T> int launch_rows(LogprobParams p, int sms, cudaStream_t s)
{
    p.split = 1;
    while (p.split < 8 && (int64_t)p.rows * p.split * 2 <= (int64_t)sms * 2 && p.vocab / p.split >= 8192) p.split *= 2;
    const int share = p.vocab / p.split;
    const int threads = share <= 2048 ? 128 : share <= 8192 ? 256 : kMostThreads;
    cudaLaunchAttribute at{};
    at.id = cudaLaunchAttributeClusterDimension;
    at.val.clusterDim.x = (unsigned)p.split;
    at.val.clusterDim.y = at.val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)p.rows * p.split);
    cfg.blockDim = dim3((unsigned)threads);
    cfg.stream = s;
    cfg.attrs = &at;
    cfg.numAttrs = p.split > 1 ? 1 : 0;
    return cuda_status(p.top ? cudaLaunchKernelEx(&cfg, logprob_kernel<T, true>, p) : cudaLaunchKernelEx(&cfg, logprob_kernel<T, false>, p));
}

}  // namespace
}  // namespace e2ops

using namespace e2ops;

extern "C" int e2_token_logprobs(const e2_logprobs_args *a, void *stream)
{
    if (!a) return fail(E2_EINVAL, "no arguments");
    Device dev;
    if (int st = current_device(&dev)) return st;
    if (a->rows < 0 || a->vocab < 1) return fail(E2_EINVAL, "rows must not be negative, vocab positive");
    if (a->dtype != E2_F16 && a->dtype != E2_BF16 && a->dtype != E2_F32) return fail(E2_EINVAL, "unknown dtype");
    if (a->top < 0 || a->top > E2_MAX_TOP) return fail(E2_EINVAL, "top must be in 0..E2_MAX_TOP");
    if (a->rows == 0) return E2_OK;
    if (!a->tokens != !a->logprob) return fail(E2_EINVAL, "tokens and logprob go together");
    if (a->top && (!a->values || !a->ids)) return fail(E2_EINVAL, "values and ids must be given");
    if (!a->logits || !aligned(a->logits, a->dtype == E2_F32 ? 4 : 2) || (a->rows > 1 && a->stride < a->vocab))
        return fail(E2_EINVAL, "logits must be given, with a row stride of at least vocab");
    const void *ptrs[] = {a->logits, a->tokens, a->logprob, a->entropy, a->top ? a->values : nullptr, a->top ? a->ids : nullptr};
    for (const void *p : ptrs)
        if (p && (!aligned(p, p == a->logits ? 2 : 4) || !on_device(p, dev.id)))
            return fail(E2_EINVAL, "arrays must be memory of the current device");
    LogprobParams p{a->rows, a->vocab, a->top, 1, a->logits, a->stride, a->tokens, a->logprob, a->entropy, a->values, a->ids};
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return a->dtype == E2_F16    ? launch_rows<__half>(p, dev.sms, s)
           : a->dtype == E2_BF16 ? launch_rows<__nv_bfloat16>(p, dev.sms, s)
                                 : launch_rows<float>(p, dev.sms, s);
}
