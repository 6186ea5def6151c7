// cache_attend.cu -- e2_cache_attend: attention over the paged 4-bit cache.
#include "ops_common.cuh"

namespace e2ops {

int check_cache(const e2_cache *c, int dev);

namespace {

struct AttendParams {
    int pages, page_shift, kv_heads, tokens, q_heads, batch, window, table_cols;
    int64_t table_stride, q_stride, out_stride;
    const uint8_t *codes[2];
    const __half2 *scales[2];
    const int32_t *table, *lens, *starts;
    float scale;
    const void *q;
    void *out;
};

// A warp per (token, query head), its lanes over the head's elements.
template <class T, int D> __global__ void __launch_bounds__(128) head_kernel(const AttendParams p)
{
    constexpr int E = D / 32;
    const int64_t unit = (int64_t)blockIdx.x * 4 + threadIdx.x / 32;
    const int lane = threadIdx.x % 32;
    if (unit >= (int64_t)p.tokens * p.q_heads) return;
    const int t = (int)(unit / p.q_heads), h = (int)(unit % p.q_heads), kv = h / (p.q_heads / p.kv_heads);
    int r = 0;
    while (r < p.batch && !(p.starts[r] <= t && t < p.starts[r + 1])) ++r;
    if (r == p.batch) return;
    const int64_t pos = (int64_t)p.lens[r] - p.starts[r + 1] + t;
    float q[E], o[E] = {}, top = -INFINITY, sum = 0;
    const T *qp = static_cast<const T *>(p.q) + t * p.q_stride + h * D + lane * E;
#pragma unroll
    for (int i = 0; i < E; ++i) q[i] = to_float(qp[i]) * p.scale;
    int64_t first = p.window > 0 && pos - p.window + 1 > 0 ? pos - p.window + 1 : 0;
    for (int64_t j = first; j <= pos; ++j) {
        const int64_t at = j >> p.page_shift;
        if (at >= p.table_cols) break;
        const int page = p.table[r * p.table_stride + at];
        if (page < 0 || page >= p.pages) continue;
        const int64_t vec = ((((int64_t)page * p.kv_heads + kv) << p.page_shift) + (j & ((1 << p.page_shift) - 1)));
        float x[2][E];
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            const uint8_t *c = p.codes[n] + vec * (D / 2) + lane * E / 2;
            const float2 dm = __half22float2(p.scales[n][vec * (D / E2_CACHE_GROUP) + lane * E / E2_CACHE_GROUP]);
#pragma unroll
            for (int i = 0; i < E; ++i) x[n][i] = __fmaf_rn((float)(c[i / 2] >> (4 * (i % 2)) & 15), dm.x, dm.y);
        }
        float a = 0;
#pragma unroll
        for (int i = 0; i < E; ++i) a = __fmaf_rn(q[i], x[0][i], a);
        for (int k = 16; k; k >>= 1) a += __shfl_xor_sync(~0u, a, k);
        const float now = fmaxf(top, a), f = expf(top - now), e = expf(a - now);
        sum = __fmaf_rn(sum, f, e);
#pragma unroll
        for (int i = 0; i < E; ++i) o[i] = __fmaf_rn(o[i], f, e * x[1][i]);
        top = now;
    }
    T *op = static_cast<T *>(p.out) + t * p.out_stride + h * D + lane * E;
#pragma unroll
    for (int i = 0; i < E; ++i) op[i] = from_float<T>(sum > 0 ? o[i] / sum : sum);
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

extern "C" size_t e2_cache_attend_workspace(const e2_cache *, const e2_attend_args *) { return 0; }

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
    const size_t need = e2_cache_attend_workspace(c, a);
    if (need && (!workspace || workspace_bytes < need)) return fail(E2_ENOMEM, "workspace too small");
    AttendParams p{c->pages, __builtin_ctz((unsigned)c->page_size), c->kv_heads, a->tokens, a->q_heads, a->batch, a->window, a->table_cols,
                   a->table_stride, a->q_stride, a->out_stride, {c->k_codes, c->v_codes},
                   {reinterpret_cast<const __half2 *>(c->k_scales), reinterpret_cast<const __half2 *>(c->v_scales)},
                   a->table, a->lens, a->starts, a->scale, a->q, a->out};
    const int64_t blocks = ((int64_t)a->tokens * a->q_heads + 3) / 4;
    if (blocks > 0x7fffffff) return fail(E2_EINVAL, "too many tokens for one call");
    const bool half = a->dtype == E2_F16;
    void (*f)(AttendParams) = c->head_dim == 64 ? (half ? head_kernel<__half, 64> : head_kernel<__nv_bfloat16, 64>)
                                                : (half ? head_kernel<__half, 128> : head_kernel<__nv_bfloat16, 128>);
    f<<<(unsigned)blocks, 128, 0, static_cast<cudaStream_t>(stream)>>>(p);
    return cuda_status(cudaGetLastError());
}
