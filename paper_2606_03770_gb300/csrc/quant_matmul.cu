// quant_matmul.cu -- e2_quant_matmul: products with 4-bit weights.
#include "quant_matmul.cuh"

namespace e2ops {
namespace {

FewPlan plan_few(int rows, int cols, int tokens, int group, bool mins, int sms)
{
    FewPlan best{};
    double best_t = 1e30;
    const int nt = tokens <= 8 ? 1 : tokens <= 16 ? 2 : 4, live = tokens < 8 * nt ? tokens : 8 * nt;
    const int chunks = (cols + kChunk - 1) / kChunk;
    const int per = kChunk / group, stage = 32 * kRowBytes + 32 * per * 2 * (mins ? 2 : 1);
    int x_cols = kChunk;
    while (x_cols < 8192 && live * x_cols * 4 <= (nt == 1 ? 16 : 32) * 1024) x_cols *= 2;
    const size_t smem = (size_t)kWarps * kStages * stage + (size_t)live * x_row_bytes(x_cols) +
                        (mins ? (size_t)live * (x_cols / group) * 4 : 0);
    const int fit = (int)(kSmemPerSm / (smem + 1024)), resident = fit < 4 ? fit : 4;
    const int slabs = (tokens + 8 * nt - 1) / (8 * nt);
    for (int wk = 1; wk <= kWarps; wk *= 2)
        for (int split = 1; split <= 8; split *= 2) {
            if (wk * kChunk > x_cols || (split > 1 && split * wk > chunks)) continue;
            const int rb = 32 * (kWarps / wk);
            const double blocks = (double)((rows + rb - 1) / rb) * split * slabs;
            const double turns = (double)(int64_t)((blocks + sms - 1) / sms);
            const double bytes = (double)((chunks + split - 1) / split) * kChunk * (rb * 0.54 + live * 1.0);
            const double together = turns < resident ? turns : resident;
            const double rate = 28.0 * together < 45.0 ? 28.0 * together : 45.0;      // bytes per ns and SM
            const double t = turns * bytes / rate + (split > 1 ? 700 : 0) + (wk > 1 ? 100 : 0);
            if (t < best_t) best_t = t, best = FewPlan{nt, wk, split, x_cols, smem};
        }
    return best;
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
    const FewPlan f = plan_few(w->rows, w->cols, a->tokens, w->group, w->mins != nullptr, dev.sms);
    const int per = kChunk / w->group;
    FewParams q{p, outs, f.wk, f.split, __builtin_ctz((unsigned)(f.x_cols / 8)), f.x_cols,
                w->cols % kChunk == 0 && aligned(w->scales, per * 2) && aligned(w->mins, per * 2)};
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return a->dtype == E2_F16 ? launch_few_f16(q, f, dev.id, s) : launch_few_bf16(q, f, dev.id, s);
}
