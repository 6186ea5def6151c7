// token_logprobs.cu -- e2_token_logprobs: log probabilities of given tokens,
// entropy and top alternatives of rows of logits.
#include "ops_common.cuh"

namespace e2ops {
namespace {

constexpr int kThreads = 512;

struct LogprobParams {
    int rows, vocab, top;
    const void *logits;
    int64_t stride;
    const int32_t *tokens;
    float *logprob, *entropy, *values;
    int32_t *ids;
};

template <class F> __device__ float block_reduce(float v, float *buf, F f)
{
    for (int o = 16; o; o >>= 1) v = f(v, __shfl_xor_sync(~0u, v, o));
    __syncthreads();
    if (threadIdx.x % 32 == 0) buf[threadIdx.x / 32] = v;
    __syncthreads();
    v = buf[0];
    for (int i = 1; i < kThreads / 32; ++i) v = f(v, buf[i]);
    return v;
}

// A block per row: a pass for the maximum, one for the sums, one per alternative.
template <class T> __global__ void __launch_bounds__(kThreads) logprob_kernel(const LogprobParams p)
{
    __shared__ float buf[kThreads / 32];
    __shared__ int best_id;
    const int r = blockIdx.x;
    const T *x = static_cast<const T *>(p.logits) + r * p.stride;
    auto larger = [](float a, float b) { return fmaxf(a, b); };
    auto plus = [](float a, float b) { return a + b; };
    float top = -INFINITY, bad = 0;
    for (int i = threadIdx.x; i < p.vocab; i += kThreads) {
        const float v = to_float(x[i]);
        if (!(v < INFINITY)) bad = 1;
        top = fmaxf(top, v);
    }
    top = block_reduce(top, buf, larger);
    bad = block_reduce(bad, buf, larger);
    const float nan = __int_as_float(0x7fc00000);
    float sum = 0, dot = 0;
    if (top > -INFINITY)
        for (int i = threadIdx.x; i < p.vocab; i += kThreads) {
            const float v = to_float(x[i]) - top, e = expf(v);
            sum += e;
            if (e > 0) dot += e * v;
        }
    sum = block_reduce(sum, buf, plus);
    dot = block_reduce(dot, buf, plus);
    const bool empty = !(top > -INFINITY);
    const float lse = empty ? 0 : top + logf(sum);
    if (threadIdx.x == 0) {
        if (p.entropy) p.entropy[r] = bad ? nan : empty ? 0.0f : logf(sum) - dot / sum;
        if (p.logprob) {
            const int y = p.tokens[r];
            p.logprob[r] = bad || y < 0 || y >= p.vocab ? nan : to_float(x[y]) - lse;
        }
    }
    float last = INFINITY;
    int last_id = -1;
    for (int k = 0; k < p.top; ++k) {
        float v = -INFINITY;
        int id = 0x7fffffff;
        for (int i = threadIdx.x; i < p.vocab; i += kThreads) {
            const float u = to_float(x[i]);
            if (u > v && (u < last || (u == last && i > last_id))) v = u, id = i;
        }
        const float m = block_reduce(v, buf, larger);
        __syncthreads();
        if (threadIdx.x == 0) best_id = 0x7fffffff;
        __syncthreads();
        if (v == m && m > -INFINITY) atomicMin(&best_id, id);
        __syncthreads();
        last = m, last_id = best_id;
        if (threadIdx.x == 0) {
            const bool none = bad || !(m > -INFINITY);
            p.values[(int64_t)r * p.top + k] = bad ? nan : none ? -INFINITY : m - lse;
            p.ids[(int64_t)r * p.top + k] = none ? -1 : last_id;
        }
    }
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
    LogprobParams p{a->rows, a->vocab, a->top, a->logits, a->stride, a->tokens, a->logprob, a->entropy, a->values, a->ids};
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (a->dtype == E2_F16) logprob_kernel<__half><<<a->rows, kThreads, 0, s>>>(p);
    else if (a->dtype == E2_BF16) logprob_kernel<__nv_bfloat16><<<a->rows, kThreads, 0, s>>>(p);
    else logprob_kernel<float><<<a->rows, kThreads, 0, s>>>(p);
    return cuda_status(cudaGetLastError());
}
