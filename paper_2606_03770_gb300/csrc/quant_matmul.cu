// quant_matmul.cu -- e2_quant_matmul: products with 4-bit weights.
#include "ops_common.cuh"

namespace e2ops {
namespace {

struct MatmulParams {
    int rows, cols, group, tokens, gated;
    const uint8_t *codes;
    const __half *scales, *mins;
    const void *x, *residual;
    void *y;
    int64_t x_stride, residual_stride, y_stride;
};

constexpr int kTokens = 8;

// A warp per output row, its lanes over words of eight columns.
template <class T> __global__ void __launch_bounds__(128) row_kernel(const MatmulParams p)
{
    const int outs = p.gated ? p.rows / 2 : p.rows;
    const int row = blockIdx.x * 4 + threadIdx.x / 32, lane = threadIdx.x % 32;
    if (row >= outs) return;
    const int t0 = blockIdx.y * kTokens, nt = min(kTokens, p.tokens - t0);
    float sum[2][kTokens] = {};
    for (int part = 0; part <= p.gated; ++part) {
        const int64_t r = row + (int64_t)part * outs;
        const uint32_t *w = reinterpret_cast<const uint32_t *>(p.codes + r * (p.cols / 2));
        const int groups = p.cols / p.group;
        for (int j = lane; j < p.cols / 8; j += 32) {
            const uint32_t c = w[j];
            const float s = __half2float(p.scales[r * groups + 8 * j / p.group]);
            const float m = p.mins ? __half2float(p.mins[r * groups + 8 * j / p.group]) : -8.0f * s;
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = __fmaf_rn((float)(c >> (4 * i) & 15), s, m);
#pragma unroll
            for (int t = 0; t < kTokens; ++t)
                if (t < nt) {
                    float x[8];
                    unpack8<T>(*reinterpret_cast<const uint4 *>(static_cast<const T *>(p.x) + (t0 + t) * p.x_stride + 8 * j), x);
#pragma unroll
                    for (int i = 0; i < 8; ++i) sum[part][t] = __fmaf_rn(v[i], x[i], sum[part][t]);
                }
        }
    }
#pragma unroll
    for (int t = 0; t < kTokens; ++t)
        for (int o = 16; o; o >>= 1) {
            sum[0][t] += __shfl_xor_sync(~0u, sum[0][t], o);
            sum[1][t] += __shfl_xor_sync(~0u, sum[1][t], o);
        }
#pragma unroll
    for (int t = 0; t < kTokens; ++t)
        if (lane == t && t < nt) {
            float y = sum[0][t];
            if (p.gated) y = y / (1.0f + expf(-y)) * sum[1][t];
            if (p.residual) y += to_float(static_cast<const T *>(p.residual)[(t0 + t) * p.residual_stride + row]);
            static_cast<T *>(p.y)[(t0 + t) * p.y_stride + row] = from_float<T>(y);
        }
}

}  // namespace
}  // namespace e2ops

using namespace e2ops;

extern "C" size_t e2_quant_matmul_workspace(int32_t, int32_t, int32_t) { return 0; }

extern "C" int e2_quant_matmul(const e2_quant_weight *w, const e2_matmul_args *a, void *workspace,
                               size_t workspace_bytes, void *stream)
{
    if (!w || !a) return fail(E2_EINVAL, "no arguments");
    Device dev;
    if (int st = current_device(&dev)) return st;
    if (w->group != 32 && w->group != 64 && w->group != 128) return fail(E2_EINVAL, "group must be 32, 64 or 128");
    if (w->rows < 1 || w->cols < w->group || w->cols > E2_MAX_COLS || w->cols % w->group)
        return fail(E2_EINVAL, "rows must be positive, cols a multiple of group up to E2_MAX_COLS");
    if (a->dtype != E2_F16 && a->dtype != E2_BF16) return fail(E2_EINVAL, "x and y are fp16 or bf16");
    if (a->tokens < 0) return fail(E2_EINVAL, "tokens must not be negative");
    if (a->gated && w->rows % 2) return fail(E2_EINVAL, "gated products need an even number of rows");
    if (!w->codes || !w->scales || !aligned(w->codes, 16) || !aligned(w->scales, 2) || !aligned(w->mins, 2))
        return fail(E2_EINVAL, "codes (16-byte aligned) and scales must be given");
    if (a->tokens == 0) return E2_OK;
    const int outs = a->gated ? w->rows / 2 : w->rows;
    if (!a->x || !aligned(a->x, 16) || a->x_stride % 8 || a->x_stride < w->cols)
        return fail(E2_EINVAL, "x: 16-byte aligned, a row stride that is a multiple of 8 and at least cols");
    if (!a->y || !aligned(a->y, 2) || a->y_stride < outs || (a->residual && (!aligned(a->residual, 2) || a->residual_stride < outs)))
        return fail(E2_EINVAL, "y, residual: row strides of at least the outputs");
    const void *ptrs[] = {w->codes, w->scales, w->mins, a->x, a->residual, a->y};
    for (const void *p : ptrs)
        if (p && !on_device(p, dev.id)) return fail(E2_EINVAL, "arrays must be memory of the current device");
    const size_t need = e2_quant_matmul_workspace(w->rows, w->cols, a->tokens);
    if (need && (!workspace || workspace_bytes < need)) return fail(E2_ENOMEM, "workspace too small");
    MatmulParams p{w->rows, w->cols, w->group, a->tokens, a->gated != 0, w->codes,
                   reinterpret_cast<const __half *>(w->scales), reinterpret_cast<const __half *>(w->mins),
                   a->x, a->residual, a->y, a->x_stride, a->residual_stride, a->y_stride};
    const dim3 grid((outs + 3) / 4, (a->tokens + kTokens - 1) / kTokens);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (a->dtype == E2_F16) row_kernel<__half><<<grid, 128, 0, s>>>(p);
    else row_kernel<__nv_bfloat16><<<grid, 128, 0, s>>>(p);
    return cuda_status(cudaGetLastError());
}
