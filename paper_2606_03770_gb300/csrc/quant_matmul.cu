// quant_matmul.cu -- e2_quant_matmul: products with 4-bit weights.
#include "quant_matmul.cuh"

namespace e2ops {
namespace {

// Blocks to have at least: 1.6 per multiprocessor keep the memory busy; and those that run at once
// on one.
constexpr int kFewBlocks = 250, kAtOnce = 3;

// So few elements of x a block prepares for itself: one launch and no workspace, where weights
// are read in less time than that costs the caller.  Measured, us a call (a graph's; by
// blocks / by a kernel before): 4096 x 4096, 1 token 13.6 / 17.2 (6.4 / 5.9), 1001 x 1376, 5
// tokens 14.3 / 19.7 (7.4 / 6.0); 57344 x 8192, 1 token (50 / 48).
constexpr size_t kOwn = kOwnOctets * 32 * kWarps * 8;
constexpr int64_t kOwnWeights = 1 << 27;

// Rows alone where they make enough blocks; else columns are split: in two by a cluster (three
// where all run at once), further among the four warps of a block first (no cluster to join), then
// by clusters of up to eight.  Measured, us (one token, 64 columns a group; joined by warps x
// clusters): 4096 x 4096 4x1 6.7, 1x4 7.0, 2x2 7.1; 10240 x 8192 1x2 15.4, 2x1 15.7, 1x1 18.9,
// 4x1 19.9; 8192 x 28672 1x3 31.9, 1x2 34.6, 2x1 35.6; 57344 x 8192 gated 1x1 46.6, 2x1 50.8, 1x2
// 55; 1024 x 16384 4x4 7.7, 1x8 9.0.
FewPlan plan_few(int rows, int cols, int tokens, int group, bool mins, int sms)
{
    const int nt = tokens <= 8 ? 1 : 2;
    const int chunks = (cols + kChunk - 1) / kChunk, x_pad = chunks * kChunk;
    const int per = kChunk / group, stage = kRows * (kRowBytes + per * 2 * (mins ? 2 : 1));
    auto plan = [&](int wk, int split) {
        // all of x at once where that leaves room for three blocks, else as many stages of each
        // warp as it does, two such segments in turn
        auto bytes = [&](int cols) { return (size_t)tokens * x_row_bytes(cols) + (size_t)8 * nt * (cols / group) * 4; };
        const int mine = (chunks + split - 1) / split * kChunk;
        const size_t ring = (size_t)kWarps * kFewStages * stage, room = kSmemPerSm / 3 - 1536 - ring;
        const bool whole = bytes(mine) <= room;
        int times = 1;
        while (bytes((times + 1) * wk * kChunk) * 2 <= room) ++times;
        const int xc = whole ? mine : times * wk * kChunk;
        const size_t smem = ring + (whole ? 1 : 2) * bytes(xc);
        const bool own = (size_t)tokens * mine <= kOwn && (int64_t)rows * cols <= kOwnWeights;
        return FewPlan{nt, wk, split, xc, x_pad, smem, own ? 0 : prepared_bytes(nt, x_pad, 32)};
    };
    auto blocks = [&](int wk, int split) {
        const int rb = kRows * kWarps / wk;
        return (int64_t)((rows + rb - 1) / rb) * split;
    };
    if (blocks(1, 1) >= kFewBlocks || chunks == 1) return plan(1, 1);
    if (blocks(1, 2) >= kFewBlocks) return plan(1, blocks(1, 3) <= kAtOnce * sms && chunks > 2 ? 3 : 2);
    int wk = kWarps, split = 1;
    while (wk > 1 && plan(wk, split).smem > (size_t)kSmemPerSm / 2 - 2048) wk /= 2;
    while (split < 8 && blocks(wk, split) < kFewBlocks && wk * split * 2 <= chunks) split *= 2;
    return plan(wk, split);
}

// From so many tokens on x is a tile of its own for the block-wide products.  Measured at 17
// tokens, us (by eights / as a tile): 8192 x 28672 81 / 67, 57344 x 8192 gated 133 / 124,
// 4096 x 4096 12.5 / 11.
constexpr int kMany = 17;

// Whether two matrices of `rows` rows of 16-bit elements share memory.  Rows of one stride (side by
// side in wider ones) are compared as columns; of two strides, all that lies between a matrix's
// first and last element.
bool share_memory(const void *a, int a_cols, int64_t a_stride, const void *b, int b_cols, int64_t b_stride, int rows)
{
    const uintptr_t a0 = reinterpret_cast<uintptr_t>(a), b0 = reinterpret_cast<uintptr_t>(b);
    const uintptr_t a1 = a0 + 2 * ((rows - 1) * a_stride + a_cols), b1 = b0 + 2 * ((rows - 1) * b_stride + b_cols);
    if (a1 <= b0 || b1 <= a0) return false;
    if (rows == 1 || a_stride != b_stride) return true;
    const uintptr_t row = 2 * a_stride;
    // b's first column, from a's
    const uintptr_t at = b0 >= a0 ? (b0 - a0) % row : (row - (a0 - b0) % row) % row;
    return at < 2 * (uintptr_t)a_cols || at + 2 * (uintptr_t)b_cols > row;
}

// Rows and tokens of whole blocks are counted in 32 bits.
constexpr int kMostRows = 0x7fffffff - 1023;

}  // namespace
}  // namespace e2ops

using namespace e2ops;

extern "C" size_t e2_quant_matmul_workspace(int32_t rows, int32_t cols, int32_t tokens)
{
    Device dev;
    if (rows < 1 || rows > kMostRows || cols < 1 || cols > E2_MAX_COLS || tokens < 1 || tokens > kMostRows || current_device(&dev))
        return 0;
    // the larger of what groups of any size, with and without gates, need
    size_t few = 0;
    for (int group = 32; tokens < kMany && group <= 128; group *= 2)
        for (int mins = 0; mins < 2; ++mins) {
            const size_t one = plan_few(rows, cols, tokens, group, mins, dev.sms).workspace;
            few = one > few ? one : few;
        }
    if (tokens < kMany) return few;
    const size_t plain = plan_many(rows, false, cols, tokens, dev.sms).workspace;
    const size_t gated = rows % 2 ? 0 : plan_many(rows / 2, true, cols, tokens, dev.sms).workspace;
    return plain > gated ? plain : gated;
}

extern "C" int e2_quant_matmul(const e2_quant_weight *w, const e2_matmul_args *a, void *workspace,
                               size_t workspace_bytes, void *stream)
{
    if (!w || !a) return fail(E2_EINVAL, "no arguments");
    Device dev;
    if (int st = current_device(&dev)) return st;
    if (w->group != 32 && w->group != 64 && w->group != 128) return fail(E2_EINVAL, "group must be 32, 64 or 128");
    if (w->rows < 1 || w->rows > kMostRows || w->cols < w->group || w->cols > E2_MAX_COLS || w->cols % w->group)
        return fail(E2_EINVAL, "rows must be in 1..2^31 - 1024, cols a multiple of group up to E2_MAX_COLS");
    if (a->dtype != E2_F16 && a->dtype != E2_BF16) return fail(E2_EINVAL, "x and y are fp16 or bf16");
    if (a->tokens < 0 || a->tokens > kMostRows) return fail(E2_EINVAL, "tokens must be in 0..2^31 - 1024");
    if (a->gated && w->rows % 2) return fail(E2_EINVAL, "gated products need an even number of rows");
    if (!w->codes || !w->scales || !aligned(w->codes, 16) || !aligned(w->scales, 2) || !aligned(w->mins, 2))
        return fail(E2_EINVAL, "codes (16-byte aligned) and scales must be given");
    if (a->tokens == 0) return E2_OK;
    const int outs = a->gated ? w->rows / 2 : w->rows;
    if (!a->x || !aligned(a->x, 16) || a->x_stride % 8 || a->x_stride < w->cols)
        return fail(E2_EINVAL, "x: 16-byte aligned, a row stride that is a multiple of 8 and at least cols");
    if (!a->y || !aligned(a->y, 2) || a->y_stride < outs || (a->residual && (!aligned(a->residual, 2) || a->residual_stride < outs)))
        return fail(E2_EINVAL, "y, residual: row strides of at least the outputs");
    if (share_memory(a->x, w->cols, a->x_stride, a->y, outs, a->y_stride, a->tokens)) return fail(E2_EINVAL, "y may not overlap x");
    const void *ptrs[] = {w->codes, w->scales, w->mins, a->x, a->residual, a->y};
    for (const void *p : ptrs)
        if (p && !on_device(p, dev.id)) return fail(E2_EINVAL, "arrays must be memory of the current device");
    const size_t need = e2_quant_matmul_workspace(w->rows, w->cols, a->tokens);
    if (need && (!workspace || workspace_bytes < need)) return fail(E2_ENOMEM, "workspace too small");
    if (need && (!aligned(workspace, 256) || !on_device(workspace, dev.id)))
        return fail(E2_EINVAL, "workspace must be 256-byte aligned memory of the current device");
    MatmulParams p{w->rows, w->cols, w->group, a->tokens, a->gated != 0, a->dtype == E2_F16, w->codes,
                   reinterpret_cast<const __half *>(w->scales), reinterpret_cast<const __half *>(w->mins),
                   a->x, a->residual, a->y, a->x_stride, a->residual_stride, a->y_stride};
    if (a->tokens >= kMany) {
        const ManyPlan f = plan_many(outs, p.gated, w->cols, a->tokens, dev.sms);
        if ((int64_t)f.row_tiles * f.tiles * 8 > 0x7fffffff) return fail(E2_EINVAL, "too many tokens for one call");
        return launch_many(p, f, workspace, outs, dev.id, static_cast<cudaStream_t>(stream));
    }
    const FewPlan f = plan_few(w->rows, w->cols, a->tokens, w->group, w->mins != nullptr, dev.sms);
    // how the scales' rows are aligned
    const int wide = w->group == 128 ? 8 : 16, groups = w->cols / w->group;
    auto all_aligned = [&](int to) { return groups * 2 % to == 0 && aligned(w->scales, to) && aligned(w->mins, to); };
    const int by = w->cols % kChunk == 0 && all_aligned(wide) ? wide : all_aligned(4) ? 4 : 2;
    FewParams q{p, outs, f.wk, f.split, f.x_cols, by, f.workspace ? static_cast<uint8_t *>(workspace) : nullptr, f.x_pad};
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return w->group == 32   ? launch_few_32(q, f, dev.id, s)
           : w->group == 64 ? launch_few_64(q, f, dev.id, s)
                            : launch_few_128(q, f, dev.id, s);
}
