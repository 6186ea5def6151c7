// token_logprobs.cu -- e2_token_logprobs: log probabilities of given tokens,
// entropy and top alternatives of rows of logits.
#include "ops_mma.cuh"

namespace e2ops {
namespace {

// One pass over a row, by a block or, where there are few rows, by the blocks of a
// cluster; bound by reading it (fp32) or by instructions (16 bits: some fourteen issue slots an
// element, seven of them arithmetic).
// A thread keeps the maximum m of what it has read, sum w and sum w t, with w = 2^t, t = x
// log2 e - c and c = m log2 e rounded once, all in 32 bits, and brings them to a new
// maximum when one comes.  The product in t is not rounded before c is taken off, and c is the
// same for all, so logits of any size keep their digits; what c was rounded by comes back at
// the end.

// Alternatives: a warp keeps the best so far sorted over its lanes, (value, then lower
// index), and looks at eight elements a lane only when some maximum of eight beats a
// bound: the `top`-th largest of 64 lanes' maxima so far, the largest few of each warp of the
// block, which `top` elements reach.  Warps publish theirs at rounds 0, 2, 8 and 32, and
// the first warp draws the bound, from old ones too, which bound as well.
// Measured, us, 128,256 logits (none / 5 / 20 alternatives): 8 rows of bf16 6.1 / 11 / 12, 1,152
// rows of fp32 91 / 109 / 116 (94, 78 and 73% of the memory's rate), of bf16 74 / 100 / 113
// (the issue of instructions, three quarters of all slots).  512 threads, three blocks on a
// multiprocessor; 256 and five 110 / 114 / 118, 512 and two 99 / 121 / 131 (fp32).

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
    float m, s, u;                       // maximum (-inf: nothing), sum w, sum w t
};

// Maxima from here on (in magnitude) do not go through c: its rounding, a power of two
// in every w, would grow with it.  Below, it is 2^-16 at most, and that is what sums of one kind
// are off by when they are brought to a maximum of the other.  (From 64 on 2^-18, but rows with such
// maxima take a quarter longer: 1,152 rows of bf16 94 us for 74.)
constexpr float kHuge = 256.0f;

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

__device__ __forceinline__ float max_or_nan(float a, float b, float c)
{
    float y;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
    return y;
}

__device__ __forceinline__ float centre(float m) { return m * kLog2e; }

// One more element; 2^t stays out of sum w t where it is 0 (-inf times 0).
__device__ __forceinline__ void add(Sums &a, float t)
{
    t = fmaxf(t, kNegligible);
    const float w = power2(t);
    a.s += w;
    a.u = __fmaf_rn(w, t, a.u);
}

// a's sums brought to the maximum m >= a.m.
__device__ __forceinline__ Sums rebase(const Sums &a, float m)
{
    if (a.m == -INFINITY) return Sums{m, 0.0f, 0.0f};
    const bool plain = fmaxf(fabsf(m), fabsf(a.m)) < kHuge;
    const float d = plain ? centre(a.m) - centre(m) : (a.m - m) * kLog2e, f = power2(d);
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
    // in the order of unsigned integers (either zero the same), 0: none
    __device__ uint64_t key() const { return v > -INFINITY ? (uint64_t)ordered(v + 0.0f) << 32 | ~(unsigned)id : 0; }
    __device__ void from(uint64_t k)
    {
        clear();
        if (k) v = unordered((unsigned)(k >> 32)), id = (int)~(unsigned)k;
    }
};

// The 32 largest of two lists, all falling over the lanes: the larger of each lane and its
// mirror fall and rise once, which five exchanges sort.
__device__ __forceinline__ uint64_t merge_lists(uint64_t a, uint64_t b, int lane)
{
    a = max(a, __shfl_sync(~0u, b, 31 - lane));
#pragma unroll
    for (int j = 16; j; j /= 2) {
        const uint64_t o = __shfl_xor_sync(~0u, a, j);
        a = (lane & j) ? min(a, o) : max(a, o);
    }
    return a;
}

template <class T, bool TOP> __global__ void __launch_bounds__(kMostThreads, 3) logprob_kernel(const LogprobParams p)
{
    constexpr int kVec = 16 / sizeof(T), kLoads = 8 / kVec;       // eight elements a lane: one load, or two
    __shared__ Sums warp_sums[kMostWarps];
    __shared__ int any_bad[kMostWarps];
    __shared__ float floor_value;
    __shared__ float published[64];                               // lanes' maxima, the largest of each warp
    __shared__ uint64_t list[TOP ? kMostWarps : 1][32];
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, warps = blockDim.x / 32;
    const int rank = blockIdx.x % p.split, row = blockIdx.x / p.split;
    const T *x = static_cast<const T *>(p.logits) + row * p.stride;
    if (TOP && threadIdx.x < 64) published[threadIdx.x] = -INFINITY;
    if (TOP && threadIdx.x == 0) floor_value = -INFINITY;
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

    // eight elements of each lane, -inf where there are none; element j is index(j)
    auto take = [&](const float (&e)[8], auto index) {
        const float m = max_or_nan(max_or_nan(e[0], e[1], e[2]), max_or_nan(e[3], e[4], e[5]), max_or_nan(e[6], e[7]));
        bad |= !(m < INFINITY);
        if (m > a.m) a = rebase(a, m);
        const float base = a.m == -INFINITY ? 0.0f : a.m;
        if (fabsf(base) < kHuge) {
            const float c = centre(base);
#pragma unroll
            for (int j = 0; j < 8; ++j) add(a, __fmaf_rn(e[j], kLog2e, -c));
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) add(a, (e[j] - base) * kLog2e);
        }
        if (!TOP) return;
        last = fmaxf(last, *reinterpret_cast<volatile float *>(&floor_value));
        if (!__any_sync(~0u, m > last)) return;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            unsigned b = __ballot_sync(~0u, e[j] > last);
            while (b) {
                const int from = __ffs(b) - 1;
                b &= b - 1;
                const float v = __shfl_sync(~0u, e[j], from);
                const int at = __shfl_sync(~0u, index(j), from);
                best.insert(v, at, lane);
            }
        }
        // (elements of later rounds have higher indices: equal ones stay out)
        last = fmaxf(last, __shfl_sync(~0u, best.v, p.top - 1));
    };
    const int share = 64 / warps;                                 // published values of a warp
    auto publish = [&](float m) {
        unsigned o = ordered(m);
        for (int i = 0; i < share; ++i) {
            const unsigned most = __reduce_max_sync(~0u, o);
            if (lane == 0) reinterpret_cast<volatile float *>(published)[warp * share + i] = unordered(most);
            // (one lane's, where several have it)
            if (lane == __ffs(__ballot_sync(~0u, o == most)) - 1) o = 0;
        }
    };
    // The `top`-th largest published value, by the first warp: below it nothing is let in.
    auto draw_bound = [&] {
        const volatile float *from = published;
        float a = from[lane], b = from[lane + 32];
        auto exchange = [&](float &v, int j, bool larger) {
            const float o = __shfl_xor_sync(~0u, v, j);
            v = larger ? fmaxf(v, o) : fminf(v, o);
        };
#pragma unroll
        for (int k = 2; k <= 32; k *= 2)
#pragma unroll
            for (int j = k / 2; j; j /= 2) {
                exchange(a, j, ((lane & k) == 0) == ((lane & j) == 0));     // falling over the lanes
                exchange(b, j, ((lane & k) == 0) != ((lane & j) == 0));     // rising
            }
        // the larger half of both, sorted
        a = fmaxf(a, b);
#pragma unroll
        for (int j = 16; j; j /= 2) exchange(a, j, (lane & j) == 0);
        const float bound = __shfl_sync(~0u, a, p.top - 1);
        if (lane == 0 && bound > -INFINITY && bound < INFINITY) *reinterpret_cast<volatile float *>(&floor_value) = below(bound);
    };

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
    auto element = [&](const uint4 (&w)[kLoads], int j) {
        return at + 32 * (j / kVec) + lane < v1 ? to_float(reinterpret_cast<const T *>(w)[j]) : -INFINITY;
    };
    auto index = [&](int j) { return head + (at + 32 * (j / kVec) + lane) * kVec + j % kVec; };
    if (TOP) {
        float m = element(ahead, 0);
#pragma unroll
        for (int j = 1; j < 8; ++j) m = fmaxf(m, element(ahead, j));
        publish(m);
        __syncthreads();
        if (warp == 0) draw_bound();
        __syncthreads();
    }
    if (rank == 0 && warp == 0 && head > 0) {
        float e[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) e[j] = -INFINITY;
        if (lane < head) e[0] = to_float(x[lane]);
        take(e, [&](int) { return lane; });
    }
    int round = 0;
    for (; at + 32 * kLoads <= v1; at += step, ++round) {         // whole rounds, then at most one that is not
        float e[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) e[j] = to_float(reinterpret_cast<const T *>(ahead)[j]);
        load(ahead, at + step);
        take(e, index);
        if (TOP && (round == 2 || round == 8 || round == 32)) {
            publish(a.m);
            if (warp == 0) draw_bound();
        }
    }
    if (at < v1) {
        float e[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) e[j] = element(ahead, j);
        take(e, index);
    }
    if (rank == p.split - 1 && warp == warps - 1 && tail < p.vocab) {
        float e[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) e[j] = -INFINITY;
        if (lane < p.vocab - tail) e[0] = to_float(x[tail + lane]);
        take(e, [&](int) { return tail + lane; });
    }

    // the warp's sums, the block's, the cluster's, in fixed orders
#pragma unroll
    for (int k = 16; k; k >>= 1)
        a = merge(a, Sums{__shfl_xor_sync(~0u, a.m, k), __shfl_xor_sync(~0u, a.s, k), __shfl_xor_sync(~0u, a.u, k)});
    bad = __any_sync(~0u, bad);
    if (lane == 0) warp_sums[warp] = a, any_bad[warp] = bad;
    if (TOP) list[warp][lane] = best.key();
    __syncthreads();
    // sums of `n` lanes, over the lanes
    auto join = [&](Sums mine, int n) {
        if (lane >= n) mine = Sums{-INFINITY, 0.0f, 0.0f};
#pragma unroll
        for (int k = 1; k < 32; k *= 2)
            mine = merge(mine, Sums{__shfl_xor_sync(~0u, mine.m, k), __shfl_xor_sync(~0u, mine.s, k), __shfl_xor_sync(~0u, mine.u, k)});
        return mine;
    };
    // the first n lists (a power of two, as many warps at least), pair by pair into the first
    auto join_lists = [&](int n) {
        for (n /= 2; n; n /= 2) {
            if (warp < n) list[warp][lane] = merge_lists(list[warp][lane], list[warp + n][lane], lane);
            __syncthreads();
        }
    };
    Sums total{-INFINITY, 0.0f, 0.0f};
    bool spoilt = false;
    if (warp == 0) {
        total = join(warp_sums[lane % warps], warps);
        spoilt = __any_sync(~0u, any_bad[lane % warps]);
    }
    if (TOP) join_lists(warps);
    if (p.split > 1) {
        if (threadIdx.x == 0) warp_sums[0] = total, any_bad[0] = spoilt;
        cluster_barrier();
        if (rank == 0) {
            // (clusters are of blocks with a warp for each)
            if (TOP && warp < p.split) {
                const uint32_t at = peer_addr(smem_addr(&list[0][lane]), warp);
                const uint64_t low = __float_as_uint(peer_load(at)), high = __float_as_uint(peer_load(at + 4));
                if (warp > 0) list[warp][lane] = high << 32 | low;
            }
            if (warp == 0) {
                const int r = lane % p.split;
                const uint32_t at = peer_addr(smem_addr(&warp_sums[0]), r);
                total = join(Sums{peer_load(at), peer_load(at + 4), peer_load(at + 8)}, p.split);
                spoilt = __any_sync(~0u, __float_as_int(peer_load(peer_addr(smem_addr(&any_bad[0]), r))));
            }
            __syncthreads();
            if (TOP) join_lists(p.split);
        }
        cluster_barrier();                                        // (peers have been read)
    }
    if (rank != 0 || warp != 0) return;
    const bool empty = total.m == -INFINITY;
    const float nan = __int_as_float(0x7fc00000), kLn2 = 0.6931471805599453f, ln = empty ? 0.0f : logf(total.s);
    // c was off by this
    const float rest = empty || !(fabsf(total.m) < kHuge) ? 0.0f : __fmaf_rn(total.m, kLog2e, -centre(total.m));
    const float lse = empty ? 0.0f : total.m + __fmaf_rn(-rest, kLn2, ln);
    if (lane == 0) {
        if (p.entropy) p.entropy[row] = spoilt ? nan : empty ? 0.0f : __fmaf_rn(-total.u / total.s, kLn2, ln);
        if (p.logprob) {
            const int y = p.tokens[row];
            p.logprob[row] = spoilt || y < 0 || y >= p.vocab ? nan : to_float(x[y]) - lse;
        }
    }
    if (TOP && lane < p.top) {
        best.from(list[0][lane]);
        const bool none = !(best.v > -INFINITY);
        p.values[(int64_t)row * p.top + lane] = spoilt ? nan : none ? -INFINITY : best.v - lse;
        p.ids[(int64_t)row * p.top + lane] = spoilt || none ? -1 : best.id;
    }
}

// While rows have no more blocks than there are multiprocessors they are split in two, over
// clusters of up to eight: two blocks a multiprocessor at most.
template <class T> int launch_rows(LogprobParams p, int sms, cudaStream_t s)
{
    p.split = 1;
    while (p.split < 8 && (int64_t)p.rows * p.split <= sms && p.vocab / p.split >= 8192) p.split *= 2;
    const int share = p.vocab / p.split;
    const int threads = share <= 2048 ? 128 : share <= 8192 ? 256 : kMostThreads;
    return launch<LogprobParams>(p.top ? logprob_kernel<T, true> : logprob_kernel<T, false>,
                                 dim3((unsigned)p.rows * p.split), threads, 0, p.split, false, s, p);
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
