// cache_attend.cuh -- what the kernels of e2_cache_attend share.
#pragma once

#include <atomic>
#include <type_traits>

#include "ops_x.cuh"

namespace e2ops {

struct AttendParams {
    int pages, page_shift, kv_heads, tokens, q_heads, batch, window, table_cols, splits;
    int64_t table_stride, q_stride, out_stride;
    const uint8_t *codes[2];
    const __half2 *scales[2];
    const int32_t *table, *lens, *starts;
    float scale;
    const void *q;
    void *out;
    float *parts;            // [tokens][q_heads][splits][D + 2]: a split's sums, maximum and sum of weights
    const int32_t *parents;  // [tokens], of trees
};

// One request and KV head: its queries, times the query heads that share the KV head,
// are rows, row = query * share + head.  Queries that are not tokens of q (`starts` out of
// range) are none of them; the others keep their positions, which may be far below 0.
struct Rows {
    int start, share;
    int64_t count, first_pos, skipped;       // rows; position of the first query; queries before it
    __device__ Rows(const AttendParams &p, int request)
    {
        const int64_t from = p.starts[request], to = p.starts[request + 1];
        const int64_t first = max(from, (int64_t)0), end = min(to, (int64_t)p.tokens);
        start = (int)min(first, (int64_t)p.tokens);
        share = p.q_heads / p.kv_heads;
        count = end > first ? (end - first) * share : 0;
        first_pos = p.lens[request] - (to - first);
        skipped = first - from;
    }
};

// Rows row0 + c of them (one division in 64 bits at most, 32 bits for each c).
struct Slab {
    unsigned share, over;                    // row0 = query * share + over
    int start;
    int64_t left, query, first_pos;          // rows from row0 on
    __device__ Slab(const Rows &r, int64_t row0) : share(r.share), start(r.start), left(r.count - row0), first_pos(r.first_pos)
    {
        query = row0 >> 32 ? row0 / share : (unsigned)row0 / share;
        over = (unsigned)(row0 - query * share);
    }
    __device__ int64_t pos(int c) const { return first_pos + query + (over + c) / share; }
    __device__ int64_t token(int c) const { return start + query + (over + c) / share; }
    __device__ int head(int kv, int c) const { return (int)(kv * share + (over + c) % share); }
    __device__ bool live(int c) const { return c < left; }
};

// A request's tree: what its nodes see.  Keys before `base` are of the tokens before the tree, key
// base + a is node a's (a tree far below token 0 has no keys, wherever it is).
struct Tree {
    int base, window;
    const int8_t *parents;                   // [E2_MAX_DRAFT], in shared memory
    __device__ Tree(const AttendParams &p, const Rows &r, const int8_t *parents)
        : base((int)max(r.first_pos - r.skipped, (int64_t)-E2_MAX_DRAFT)), window(p.window), parents(parents)
    {
    }
    // All threads of a block; a barrier has to follow.
    static __device__ void load(const AttendParams &p, int request, int8_t *parents)
    {
        for (int i = threadIdx.x; i < E2_MAX_DRAFT; i += blockDim.x) {
            const int64_t t = (int64_t)p.starts[request] + i;
            const int parent = t >= 0 && t < p.tokens ? p.parents[t] : -1;
            parents[i] = parent >= 0 && parent < i ? (int8_t)parent : (int8_t)-1;
        }
    }
    // Bit a: whether the node sees node a's key; and the first key of those before `base`.
    __device__ uint64_t way(int64_t node, int &lowest) const
    {
        uint64_t seen = 0;
        int depth = 0;
        for (int a = (int)node; a >= 0; a = parents[a], ++depth)
            if (window == 0 || depth < window) seen |= 1ull << a;
        lowest = window > 0 ? max(base + (depth - window), 0) : 0;
        return seen;
    }
};

__device__ __forceinline__ float power2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t pack_half(float lo, float hi)
{
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&h);
}

// The rows of a prompt (cache_attend_prompt.cu): blocks of kPromptRows, `splits` parts of the keys.
constexpr int kPromptRows = 256;
int launch_prompt(const AttendParams &p, int head_dim, bool half, int blocks, int pairs, int dev, cudaStream_t s);
// The rows of trees (cache_attend_tree.cu), likewise by kTreeRows; without room for parts (p.parts) up to kTreeCluster
// of them are joined in a cluster.
constexpr int kTreeRows = 128, kTreeCluster = 4;
int launch_tree(const AttendParams &p, int head_dim, bool half, int blocks, int pairs, int dev, cudaStream_t s);

}  // namespace e2ops
