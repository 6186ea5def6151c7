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
    const uint64_t *ways;                    // [E2_MAX_DRAFT], in shared memory; bit a: node a is on the way up, itself among it
    __device__ Tree(const AttendParams &p, const Rows &r, const uint64_t *ways)
        : base((int)max(r.first_pos - r.skipped, (int64_t)-E2_MAX_DRAFT)), window(p.window), ways(ways)
    {
    }
    // One warp; a barrier has to follow.  Each node takes in what the node at the end of its way so far has, whose way
    // goes on from there: as many rounds as the logarithm of the longest way.
    static __device__ void load(const AttendParams &p, int request, uint64_t *ways)
    {
        const int lane = threadIdx.x % 32;
        int next[2];
        uint64_t way[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int i = lane + 32 * h;
            const int64_t t = (int64_t)p.starts[request] + i;
            const int parent = t >= 0 && t < p.tokens ? p.parents[t] : -1;
            next[h] = parent >= 0 && parent < i ? parent : -1;
            way[h] = 1ull << i;
        }
        while (__any_sync(~0u, next[0] >= 0 || next[1] >= 0)) {
            uint64_t more[2];
            int then[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int from = next[h] & 31;
                const uint64_t w0 = __shfl_sync(~0u, way[0], from), w1 = __shfl_sync(~0u, way[1], from);
                const int n0 = __shfl_sync(~0u, next[0], from), n1 = __shfl_sync(~0u, next[1], from);
                more[h] = next[h] < 0 ? 0 : next[h] < 32 ? w0 : w1;
                then[h] = next[h] < 0 ? -1 : next[h] < 32 ? n0 : n1;
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) way[h] |= more[h], next[h] = then[h];
        }
        ways[lane] = way[0], ways[lane + 32] = way[1];
    }
    // Bit a: whether the node sees node a's key; and the first key of those before `base`.  (A way's nodes stand
    // in the order of their numbers: the farthest are the lowest bits.)
    __device__ uint64_t way(int64_t node, int &lowest) const
    {
        uint64_t seen = ways[node];
        int far = __popcll(seen);
        lowest = 0;
        if (window > 0) {
            lowest = max(base + (far - window), 0);
            for (; far > window; --far) seen &= seen - 1;
        }
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
// The rows of trees (cache_attend_tree.cu), likewise by kTreeRows, or by half as many (few); without room for parts (p.parts) up to kTreeCluster
// of them are joined in a cluster.
constexpr int kTreeRows = 128, kTreeCluster = 4;
int launch_tree(const AttendParams &p, int head_dim, bool half, bool few, int blocks, int pairs, int dev, cudaStream_t s);

}  // namespace e2ops
