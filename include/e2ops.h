/*
 * e2ops.h -- the operators of one served decoder block on the GB300 (sm_103a):
 * 4-bit weights (the models the paper deploys), a paged key/value cache in 4
 * bits (the search's workloads count one of fp16), decode batches of a few
 * requests and prompts of a few thousand tokens.  They are what a user runs to
 * measure a block on this GPU (Sec. 3.1 of the paper: load a reduced number of
 * blocks, time them) and to serve with it.  Same library (libe2ga.so) and
 * conventions as e2ga.h:
 *
 *  - Every function returns an e2_status; e2_ops_error() has the text of the
 *    calling thread's last failed call of this header.  Nothing aborts or throws.
 *  - Work is enqueued on `stream` (cudaStream_t; NULL = legacy default) and is
 *    asynchronous.  No call synchronises or allocates device memory, so every
 *    call may be captured in a CUDA graph (each kernel once outside a capture
 *    first).  Workspaces are the caller's; a workspace belongs to one call at a time.
 *  - All arrays are device memory of the current device, rows contiguous in
 *    their last axis; strides are in elements.  Host pointers are refused.
 *  - E2_EINVAL for sizes, strides, alignments and pointers outside what is
 *    written below; nothing is launched then.  Values in device arrays (page
 *    numbers, slots, positions, token ids, lengths) are checked by the kernels:
 *    what is out of range is never followed, with the result written below.
 *  - A call with zero tokens, rows or requests does nothing and returns E2_OK.
 *  - The kernels for prompts (products from 17 tokens, attention from 65 rows of a
 *    request and KV head) wait for copies and products of their own block.  Such a
 *    wait ends after some seconds at the latest; the block's outputs are NaN then,
 *    with E2_OK, which is returned long before.
 */
#ifndef E2OPS_H
#define E2OPS_H

#include "e2ga.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { E2_F16 = 0, E2_BF16 = 1, E2_F32 = 2 } e2_dtype;

const char *e2_ops_error(void);

/* ---- products with 4-bit weights ------------------------------------------
 *
 * W[n][k] = scales[n][k / group] * (code - 8)                 (mins NULL)
 *         = scales[n][k / group] * code + mins[n][k / group]  (mins given)
 *
 * codes [rows][cols / 2]: column 2j in the low four bits of byte j, 2j + 1 in
 * the high ones; 16-byte aligned.  scales, mins: fp16 [rows][cols / group].
 * group is 32, 64 or 128; cols a multiple of group, up to E2_MAX_COLS; rows, and
 * the tokens of a call, up to 2^31 - 1024. */
typedef struct {
    int32_t rows, cols, group;
    const uint8_t *codes;
    const uint16_t *scales;
    const uint16_t *mins;
} e2_quant_weight;

#define E2_MAX_COLS (1 << 20)

/* y[t][n] = sum_k x[t][k] W[n][k] (+ residual[t][n]), t < tokens.
 * gated != 0: rows = 2 F, the first F rows gate the others, y [tokens][F]:
 * y[t][f] = a / (1 + exp(-a)) * b (+ residual), a from row f, b from row F + f.
 * x, residual (or NULL) and y are fp16 or bf16 (dtype); x 16-byte aligned, its
 * row stride a multiple of 8.  Sums are in 32 bits, y is rounded once; x goes to
 * the tensor cores as fp16 times a power of two per token (values below 2^-24 of the
 * token's largest lose bits).  From 17 tokens on W does too, rounded once to fp16
 * (2^-11 of a weight; what passes 65,504 stays there), so 16 and 17 tokens differ
 * in more than the order of their sums.  An x that is infinite or NaN gives the formula's infinities and NaN, in its own row of y only.  y may not
 * overlap x or the weights; it may be residual itself.
 * workspace: e2_quant_matmul_workspace() bytes (0: may be NULL), 256-byte
 * aligned, contents of no consequence. */
typedef struct {
    int32_t tokens, dtype, gated;
    const void *x;
    int64_t x_stride;
    const void *residual;
    int64_t residual_stride;
    void *y;
    int64_t y_stride;
} e2_matmul_args;

size_t e2_quant_matmul_workspace(int32_t rows, int32_t cols, int32_t tokens);
int e2_quant_matmul(const e2_quant_weight *w, const e2_matmul_args *a, void *workspace, size_t workspace_bytes,
                    void *stream);

/* ---- a paged 4-bit cache of keys and values ----------------------------------
 *
 * Slot s is token s % page_size of page s / page_size.  Per token and head,
 * each E2_CACHE_GROUP elements x share an fp16 minimum m = f16(min x) and an
 * fp16 scale d = f16((max x - min x) / 15); an element's code is
 * (x - m) / d rounded to even and clamped to 0..15 (0 where d is 0), and
 * stands for m + d * code.  min x and max x are first clamped to fp16's finite
 * range; of a group that holds a NaN m is NaN, d and the codes are 0.
 *
 *   codes  [pages][kv_heads][page_size][head_dim / 2] bytes, element 2j low
 *   scales [pages][kv_heads][page_size][head_dim / E2_CACHE_GROUP][2] fp16: d, m
 *
 * head_dim 64 or 128; page_size 16, 32, 64, 128 or 256; arrays 16-byte aligned. */
#define E2_CACHE_GROUP 64

typedef struct {
    int32_t pages, page_size, kv_heads, head_dim;
    uint8_t *k_codes;
    uint16_t *k_scales;
    uint8_t *v_codes;
    uint16_t *v_scales;
} e2_cache;

/* Appends `tokens` keys and values [tokens][kv_heads][head_dim] (fp16 or bf16)
 * at slots[t], keys turned by their positions first, and turns the queries
 * [tokens][q_heads][head_dim] likewise into q_out (q NULL: no queries).  The
 * turn, in 32 bits with each product and sum rounded, of the pair (a, b) with
 * row positions[t] of cos, sin [table_rows][rot / 2]: (a cos - b sin, b cos +
 * a sin).  Pairs are (i, i + rot/2) for i < rot/2, or (2i, 2i + 1) when
 * interleaved; elements from rot on stay.  rot: a multiple of 16, 0..head_dim.
 * q_out may be q.  Token strides are multiples of 8, bases 16-byte aligned.
 * A slot outside the cache (-1: padding) is not written.  A position outside
 * the table: nothing of the token is cached, its q_out is NaN.  Two tokens of
 * one call with the same slot leave either one's bytes, piece by piece. */
typedef struct {
    int32_t tokens, dtype, q_heads, rot, interleaved, table_rows;
    const int64_t *slots;
    const int32_t *positions;
    const float *cos, *sin;
    const void *k;
    int64_t k_stride;
    const void *v;
    int64_t v_stride;
    const void *q;
    int64_t q_stride;
    void *q_out;
    int64_t q_out_stride;
} e2_append_args;

int e2_cache_append(const e2_cache *c, const e2_append_args *a, void *stream);

/* Reads tokens back, as the values their codes stand for: k, v
 * [tokens][kv_heads][head_dim] (fp16, bf16 or fp32, either may be NULL),
 * strides multiples of 8, bases 16-byte aligned.  A slot outside the cache
 * reads as zeros. */
int e2_cache_read(const e2_cache *c, const int64_t *slots, int32_t tokens, int32_t dtype, void *k,
                  int64_t k_stride, void *v, int64_t v_stride, void *stream);

/* Attention over the cache.  Request r has keys 0..lens[r]-1, key j in slot
 * table[r][j / page_size] * page_size + j % page_size, and the queries
 * starts[r]..starts[r+1]-1 of q [tokens][q_heads][head_dim]; they are its last
 * positions: query i stands at p = lens[r] - new + i.  It sees key j when
 * j <= p and, with a window > 0, j > p - window.  Query head h reads KV head
 * h / (q_heads / kv_heads).
 *   out[i][h] = sum_j softmax_j(scale * q.k_j) v_j, 0 where no key is seen.
 * A query that is infinite or NaN gives NaN where it sees a key.  Sums are in 32
 * bits, out is rounded once; what the tensor cores take is fp16:
 *  - queries, times a power of two each (elements below 2^-24 of the largest of a
 *    query and head lose bits);
 *  - up to 64 rows (max_new times query heads) of a request and KV head: weights
 *    times their values' scales, 2^-11 of each; minima are not rounded, so the
 *    error is 2^-11 of sum p |d code|, which outputs may be far below;
 *  - from 65 rows on: keys, values and weights, 2^-11 of each (keys and values that
 *    pass 65,504, which appended ones do not, stay there);
 *  - fp16 outputs: what rounding took from the weights is in a product of its own.
 * q, out: fp16 or bf16, [tokens][q_heads][head_dim], token strides multiples of
 * 8, bases 16-byte aligned; out may be q only if a request has one query.
 * max_new and max_len are the largest new and lens: they shape the launch, larger ones on
 * the device only cost time.  Keys of pages outside the cache are not seen, nor
 * those from table_cols * page_size on; a token of q outside every request is not
 * written.  batch * kv_heads is at most 65535.
 * workspace: e2_cache_attend_workspace() bytes (0: may be NULL), 256-byte
 * aligned, contents of no consequence. */
typedef struct {
    int32_t tokens, dtype, q_heads, batch;
    const int32_t *table;   /* [batch][table_cols] */
    int32_t table_cols;
    int64_t table_stride;
    const int32_t *lens, *starts;
    int32_t max_new, max_len;
    float scale;
    int32_t window;
    const void *q;
    int64_t q_stride;
    void *out;
    int64_t out_stride;
} e2_attend_args;

size_t e2_cache_attend_workspace(const e2_cache *c, const e2_attend_args *a);
int e2_cache_attend(const e2_cache *c, const e2_attend_args *a, void *workspace, size_t workspace_bytes,
                    void *stream);

/* ---- the output layer ---------------------------------------------------------
 *
 * Of each row x of logits [rows][vocab] (fp16, bf16 or fp32, any row stride):
 *   lse = max x + ln sum exp(x - max x), in 32 bits
 *   logprob = x[tokens[row]] - lse        (tokens, logprob may both be NULL)
 *   entropy = lse - sum p x, p = exp(x - lse)                (may be NULL)
 *   values, ids [rows][top]: the `top` largest x - lse and their indices,
 *   largest first, equal ones by their index; 0 <= top <= E2_MAX_TOP.
 * -inf marks a forbidden token: it is never listed.  Rows with fewer than `top`
 * allowed tokens end in values -inf, ids -1.  A row without any: logprob -inf,
 * entropy 0.  A row that holds a NaN or +inf has no distribution: NaN, ids -1.
 * A token id outside the vocabulary: logprob NaN. */
#define E2_MAX_TOP 32

typedef struct {
    int32_t rows, vocab, dtype, top;
    const void *logits;
    int64_t stride;
    const int32_t *tokens;
    float *logprob, *entropy, *values;
    int32_t *ids;
} e2_logprobs_args;

int e2_token_logprobs(const e2_logprobs_args *a, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* E2OPS_H */
