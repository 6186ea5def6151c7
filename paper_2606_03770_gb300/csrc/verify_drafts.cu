// verify_drafts.cu -- e2_verify_drafts: which drafted tokens of a tree the target's
// probabilities accept, and the token after them.
#include <stddef.h>

#include "ops_mma.cuh"
#include "ops_two.cuh"

namespace e2ops {
namespace {

// A cluster of blocks walks a request's tree, and all its warps take the same decisions.  Each
// warp has a run of the vocabulary; what a pass over a row gives is the warps' sums, which every
// warp reads after one barrier of the cluster.  With p = w / Z, w = exp((x - max x) / T), and q
// likewise of the draft's row, after k rejections
//   P = (p - A q)+ / B,  A_0 = 0, B_0 = 1, A_{k+1} = A_k + B_k, B_{k+1} = sum (p - A_{k+1} q)+,
// as (P - q)+ is (p - A q - B q)+ / B.  Without the draft's rows a rejected token leaves P.
// The token after the last is found in the warps' sums, then in the sums of a sixteenth of a
// warp's run, then element by element.  The numbers that decide have some 45 bits.

constexpr int kThreads = 512, kWarps = kThreads / 32, kMostCluster = 8, kRuns = kWarps * kMostCluster / 32;
constexpr float kNothing = 0x1p-36f;             // a sum below it, of what it is a part of, is rounding's

struct VerifyParams {
    int tokens, vocab, batch, max_new, split;
    const void *logits, *draft;
    int64_t logits_stride, draft_stride;
    const int32_t *ids, *parents, *starts;
    const float *uniforms, *temperature;
    int32_t *kept, *nodes, *answer;
};

// What a warp tells the others in a pass.
struct Part {
    Two p, q;                                    // sums
    float p_top, q_top;
    int first;                                   // of the largest
    int bad;
};

struct Shared {
    float2 table[PowerTable::kSize];
    Part parts[2][kWarps];                       // (a block may be one pass ahead of another)
    Two sub[kWarps];
    int32_t ids[E2_MAX_DRAFT], parents[E2_MAX_DRAFT];
    float uniforms[E2_MAX_DRAFT];
};

__device__ const PowerTable power_table = PowerTable();

__device__ __forceinline__ int peer_load_int(uint32_t at) { return __float_as_int(peer_load(at)); }
__device__ __forceinline__ Two peer_load_two(uint32_t at) { return Two{peer_load(at), peer_load(at + 4)}; }

// w times 2^e, e <= 0, with its second part in its place; 0 from 2^-120 on.
__device__ __forceinline__ Two scaled(const Two &w, int e)
{
    if (e < -120) return Two{0, 0};
    const float f = __int_as_float((e + 127) << 23);
    return sum_of_larger(w.h * f, w.l * f);
}

template <class T> struct Walk {
    const VerifyParams &p;
    Shared &m;
    int lane, warp, rank, turn;
    int first, end;                              // this warp's run
    const T *x, *y;                              // the node's rows
    Two heat;                                    // 1 / T
    float x_top, y_top;
    Two runs[kRuns];                             // sums of the runs kRuns lane + j

    __device__ Walk(const VerifyParams &p, Shared &m) : p(p), m(m), turn(0)
    {
        lane = threadIdx.x % 32, warp = threadIdx.x / 32, rank = blockIdx.x % p.split;
        first = run_start(rank * kWarps + warp), end = run_start(rank * kWarps + warp + 1);
    }
    __device__ int run_start(int run) const
    {
        const int64_t units = ((int64_t)p.vocab + 31) / 32;
        return (int)min(32 * (units * run / (kWarps * p.split)), (int64_t)p.vocab);
    }

    // Every warp's part, to all: visit(run, address).  The next pass writes the other half.
    template <class F> __device__ void exchange(const Part &mine, F visit)
    {
        if (lane == 0) m.parts[turn][warp] = mine;
        cluster_barrier();
        const uint32_t at = smem_addr(m.parts[turn]);
#pragma unroll
        for (int j = 0; j < kRuns; ++j) {
            const int run = kRuns * lane + j;
            if (run < kWarps * p.split) visit(j, peer_addr(at + run % kWarps * (int)sizeof(Part), run / kWarps));
        }
        turn ^= 1;
    }

    // The largest of x (and of y): whether both rows have a distribution, and x's first largest.
    __device__ bool tops(bool both, int &where)
    {
        Part mine{{0, 0}, {0, 0}, -INFINITY, -INFINITY, 0x7fffffff, 0};
        for (int i = first + lane; i < end; i += 32) {
            const float a = to_float(x[i]), b = both ? to_float(y[i]) : 0.0f;
            if (a > mine.p_top) mine.p_top = a, mine.first = i;
            mine.q_top = fmaxf(mine.q_top, b);
            mine.bad |= !(a < INFINITY) || !(b < INFINITY);
        }
        auto join = [&](float a, float b, int at, int bad) {
            if (a > mine.p_top || (a == mine.p_top && at < mine.first)) mine.first = at;
            mine.p_top = fmaxf(mine.p_top, a);
            mine.q_top = fmaxf(mine.q_top, b);
            mine.bad |= bad;
        };
        auto warp_join = [&] {
#pragma unroll
            for (int k = 16; k; k /= 2)
                join(__shfl_xor_sync(~0u, mine.p_top, k), __shfl_xor_sync(~0u, mine.q_top, k), __shfl_xor_sync(~0u, mine.first, k),
                     __shfl_xor_sync(~0u, mine.bad, k));
        };
        warp_join();
        exchange(mine, [&](int, uint32_t at) {
            join(peer_load(at + offsetof(Part, p_top)), peer_load(at + offsetof(Part, q_top)), peer_load_int(at + offsetof(Part, first)),
                 peer_load_int(at + offsetof(Part, bad)));
        });
        warp_join();
        x_top = mine.p_top, y_top = mine.q_top, where = mine.first;
        return !mine.bad && x_top > -INFINITY && (!both || y_top > -INFINITY);
    }

    // One element of what P is of: w, or (w - share of the draft's)+.
    __device__ __forceinline__ Two weight(int i, bool less, const Two &share) const
    {
        const Two a = exp_of(to_float(x[i]), x_top, heat, m.table);
        if (!less) return a;
        const Two b = share * exp_of(to_float(y[i]), y_top, heat, m.table), d = a - b;
        return d.h > 0 ? d : Two{0, 0};
    }

    // Sums of x's weights, less `share` of y's where it says so, by runs and whole; and of y's alone.
    __device__ Two sums(bool less, const Two &share, bool both, Two &q)
    {
        LongSum a, b;
        for (int i = first + lane; i < end; i += 32) {
            a.add(weight(i, less, share));
            if (both) b.add(exp_of(to_float(y[i]), y_top, heat, m.table));
        }
        const Part mine{warp_sum(a.value()), both ? warp_sum(b.value()) : Two{0, 0}, 0, 0, 0, 0};
        Two total{0, 0};
        q = Two{0, 0};
#pragma unroll
        for (int j = 0; j < kRuns; ++j) runs[j] = Two{0, 0};
        exchange(mine, [&](int j, uint32_t at) {
            runs[j] = peer_load_two(at + offsetof(Part, p));
            total = total + runs[j];
            if (both) q = q + peer_load_two(at + offsetof(Part, q));
        });
        if (both) q = warp_sum(q);
        return warp_sum(total);
    }

    // The first v whose share of the sums in order passes u, in one warp of one block, which it
    // returns true to.  gone(i): tokens that P has lost.
    template <class F> __device__ bool find(float u, bool less, const Two &share, F gone, int &answer)
    {
        // the run
        Two mine{0, 0};
#pragma unroll
        for (int j = 0; j < kRuns; ++j) mine = mine + runs[j];
        const Two up_to = warp_prefix(mine, lane);
        const Two total{__shfl_sync(~0u, up_to.h, 31), __shfl_sync(~0u, up_to.l, 31)};
        const Two target = Two{u, 0} * total;
        Two before = up_to - mine, found_before{0, 0};
        int found = 0x7fffffff, last = -1;
        Two last_before{0, 0};
#pragma unroll
        for (int j = 0; j < kRuns; ++j) {
            const Two after = before + runs[j];
            if (runs[j].h > 0) {
                if (found == 0x7fffffff && target < after) found = kRuns * lane + j, found_before = before;
                last = kRuns * lane + j, last_before = before;
            }
            before = after;
        }
        // (by rounding no run may seem to pass it: the last that has anything)
        choose(found, found_before, last, last_before);
        if (found / kWarps != rank) return false;
        // its sixteenths
        const int from = run_start(found), units = (run_start(found + 1) - from + 31) / 32, stop = run_start(found + 1);
        auto sixteenth = [&](int k) { return min(from + 32 * (int)((int64_t)units * k / kWarps), stop); };
        LongSum a;
        for (int i = sixteenth(warp) + lane; i < sixteenth(warp + 1); i += 32)
            if (!gone(i)) a.add(weight(i, less, share));
        const Two sub = warp_sum(a.value());
        if (lane == 0) m.sub[warp] = sub;
        __syncthreads();
        mine = lane < kWarps ? m.sub[lane] : Two{0, 0};
        const Two upto = found_before + warp_prefix(mine, lane);
        Two was{__shfl_up_sync(~0u, upto.h, 1), __shfl_up_sync(~0u, upto.l, 1)};
        if (lane == 0) was = found_before;
        found = mine.h > 0 && target < upto ? lane : 0x7fffffff;
        Two base = was;
        choose(found, base, mine.h > 0 ? lane : -1, was);
        if (found != warp) return false;
        // element by element
        answer = -1;
        for (int i0 = sixteenth(warp); i0 < sixteenth(warp + 1); i0 += 32) {
            const int i = i0 + lane;
            const Two w = i < sixteenth(warp + 1) && !gone(i) ? weight(i, less, share) : Two{0, 0};
            const Two sum = base + warp_prefix(w, lane);
            const unsigned some = __ballot_sync(~0u, w.h > 0), hit = __ballot_sync(~0u, w.h > 0 && target < sum);
            if (some) answer = i0 + (hit ? __ffs(hit) - 1 : 31 - __clz(some));
            if (hit) break;
            base = Two{__shfl_sync(~0u, sum.h, 31), __shfl_sync(~0u, sum.l, 31)};
        }
        return true;
    }
    // The lowest `found` of the lanes, or else the highest `last`, with what came before it.
    __device__ void choose(int &found, Two &before, int last, const Two &last_before)
    {
        const unsigned some = __ballot_sync(~0u, found != 0x7fffffff), any = __ballot_sync(~0u, last >= 0);
        const int from = some ? __ffs(some) - 1 : any ? 31 - __clz(any) : 0;
        const int at = some ? found : last;
        const Two b = some ? before : last_before;
        found = max(__shfl_sync(~0u, at, from), 0);
        before = Two{__shfl_sync(~0u, b.h, from), __shfl_sync(~0u, b.l, from)};
    }
};

template <class T> __global__ void __launch_bounds__(kThreads) verify_kernel(const VerifyParams p)
{
    __shared__ Shared m;
    const int request = blockIdx.x / p.split;
    Walk<T> walk(p, m);
    const bool writer = walk.rank == 0 && threadIdx.x == 0;
    const int64_t start = p.starts[request], stop = p.starts[request + 1];
    const int n = start >= 0 && stop <= p.tokens ? (int)min(max(stop - start, (int64_t)0), (int64_t)p.max_new) : 0;
    for (int i = threadIdx.x; i < PowerTable::kSize; i += kThreads) m.table[i] = power_table.v[i];
    if (threadIdx.x < n) {
        m.ids[threadIdx.x] = p.ids[start + threadIdx.x];
        m.parents[threadIdx.x] = p.parents[start + threadIdx.x];
        const float u = p.uniforms[start + threadIdx.x];
        m.uniforms[threadIdx.x] = u > 0 ? fminf(u, 1.0f) : 0.0f;
    }
    __syncthreads();
    int32_t *nodes = p.nodes + (int64_t)request * p.max_new, *answer = p.answer + (int64_t)request * p.max_new;
    const float degree = p.temperature ? p.temperature[request] : 1.0f;
    const bool greedy = degree == 0, heated = degree > 0 && degree < INFINITY;
    walk.heat = heated ? Two{1, 0} / Two{fmaxf(degree, 0x1p-126f), 0} : Two{1, 0};
    auto inside = [&](int v) { return v >= 0 && v < p.vocab; };

    int here = 0, kept = n > 0;
    int token = -1;                                       // the token after the last, in the thread that knows it
    bool knows = writer;
    while (n > 0) {
        walk.x = static_cast<const T *>(p.logits) + (start + here) * p.logits_stride;
        walk.y = p.draft ? static_cast<const T *>(p.draft) + (start + here) * p.draft_stride : nullptr;
        int child = here + 1, first;
        auto next_child = [&] {
            while (child < n && m.parents[child] != here) ++child;
            return child < n;
        };
        bool open = next_child();
        const bool both = p.draft && open && heated;
        if (!(greedy || heated) || !walk.tops(both, first)) break;
        int accepted = -1;
        if (greedy) {
            for (; open && accepted < 0; ++child, open = next_child())
                if (m.ids[child] == first) accepted = child;
            if (accepted < 0) token = first;
        } else {
            const Two none{0, 0};
            Two q, share = none, A = none, B{1, 0};
            const Two all = walk.sums(false, none, both, q);
            Two left = all;                               // (without the draft's rows)
            uint64_t lost = 0;                            // rejected children whose tokens P has lost
            bool less = false;
            auto gone = [&](int v) {
                for (uint64_t r = lost; r; r &= r - 1)
                    if (m.ids[__ffsll(r) - 1] == v) return true;
                return false;
            };
            for (; open; ++child, open = next_child()) {
                const int v = m.ids[child];
                const bool in = inside(v);
                const float u = m.uniforms[child];
                // its weight, however small
                Two w = none, wq = none;
                int e = 0, eq = 0;
                const bool some = in && exp_parts(to_float(walk.x[v]), walk.x_top, walk.heat, m.table, kLowestWideExp, w, e);
                if (p.draft) {
                    // u q(v) < P(v), times Z_p Z_q B and a power of two
                    const bool some_q = in && exp_parts(to_float(walk.y[v]), walk.y_top, walk.heat, m.table, kLowestWideExp, wq, eq);
                    const int most = some && some_q ? max(e, eq) : some ? e : eq;
                    w = scaled(w, some ? e - most : -127);
                    wq = scaled(wq, some_q ? eq - most : -127);
                    const Two mine = w * q - A * wq * all;
                    if ((u == 0 && !less && some) || Two{u, 0} * wq * all * B < (mine.h > 0 ? mine : none)) {
                        accepted = child;
                        break;
                    }
                    Two before[kRuns], unused;
#pragma unroll
                    for (int j = 0; j < kRuns; ++j) before[j] = walk.runs[j];
                    const Two more = A + B, part = more * all / q, sum = walk.sums(true, part, false, unused) / all;
                    if (sum.h > kNothing * B.h) {
                        A = more, B = sum, share = part, less = true;
                    } else {
#pragma unroll
                        for (int j = 0; j < kRuns; ++j) walk.runs[j] = before[j];
                    }
                } else if (in && !gone(v)) {
                    w = scaled(w, some ? e : -127);
                    if ((u == 0 && some) || Two{u, 0} * left < w) {
                        accepted = child;
                        break;
                    }
                    const Two rest = left - w;
                    if (some && rest.h > kNothing * left.h) {
                        left = rest;
                        lost |= 1ull << child;
                        // its run loses it too
#pragma unroll
                        for (int j = 0; j < kRuns; ++j) {
                            const int run = kRuns * walk.lane + j;
                            if (run < kWarps * p.split && v >= walk.run_start(run) && v < walk.run_start(run + 1)) {
                                walk.runs[j] = walk.runs[j] - w;
                                if (!(walk.runs[j].h > 0)) walk.runs[j] = none;
                            }
                        }
                    }
                }
            }
            if (accepted < 0) {
                knows = walk.find(m.uniforms[0], less, share, gone, token) && walk.lane == 0;
            }
        }
        if (accepted < 0) break;
        if (writer) nodes[kept] = accepted, answer[kept - 1] = m.ids[accepted];
        here = accepted;
        ++kept;
    }
    if (knows && n > 0) answer[kept - 1] = token;
    if (writer) {
        p.kept[request] = kept;
        if (kept) nodes[0] = 0;
        for (int i = kept; i < p.max_new; ++i) nodes[i] = answer[i] = -1;
    }
    cluster_barrier();                                    // (peers have been read)
}

// Requests over clusters, while they have no more blocks than there are multiprocessors.
template <class T> int launch_walks(VerifyParams p, int sms, cudaStream_t s)
{
    p.split = 1;
    while (p.split < kMostCluster && (int64_t)p.batch * p.split <= sms && p.vocab / p.split >= 4096) p.split *= 2;
    return launch<VerifyParams>(verify_kernel<T>, dim3((unsigned)p.batch * p.split), kThreads, 0, p.split, false, s, p);
}

}  // namespace
}  // namespace e2ops

using namespace e2ops;

extern "C" int e2_verify_drafts(const e2_verify_args *a, void *stream)
{
    if (!a) return fail(E2_EINVAL, "no arguments");
    Device dev;
    if (int st = current_device(&dev)) return st;
    if (a->tokens < 0 || a->batch < 0 || a->batch > (1 << 20) || a->vocab < 1 || a->vocab > (1 << 30))
        return fail(E2_EINVAL, "tokens must not be negative, batch in 0..2^20, vocab in 1..2^30");
    if (a->dtype != E2_F16 && a->dtype != E2_BF16 && a->dtype != E2_F32) return fail(E2_EINVAL, "unknown dtype");
    if (a->max_new < 0 || a->max_new > E2_MAX_DRAFT) return fail(E2_EINVAL, "max_new must be in 0..E2_MAX_DRAFT");
    if (a->batch == 0) return E2_OK;
    const size_t size = a->dtype == E2_F32 ? 4 : 2;
    if (!a->starts || !a->kept || (a->max_new && (!a->nodes || !a->answer)))
        return fail(E2_EINVAL, "starts, kept, nodes and answer must be given");
    if (a->tokens && a->max_new && (!a->logits || !a->ids || !a->parents || !a->uniforms))
        return fail(E2_EINVAL, "logits, ids, parents and uniforms must be given");
    if (!aligned(a->logits, size) || !aligned(a->draft, size) ||
        (a->tokens > 1 && (a->logits_stride < a->vocab || (a->draft && a->draft_stride < a->vocab))))
        return fail(E2_EINVAL, "rows of logits and draft must be aligned to their type, with strides of at least vocab");
    const void *ptrs[] = {a->logits, a->draft, a->ids, a->parents, a->starts, a->uniforms, a->temperature, a->kept, a->nodes, a->answer};
    for (int i = 0; i < 10; ++i)
        if (ptrs[i] && ((i > 1 && !aligned(ptrs[i], 4)) || !on_device(ptrs[i], dev.id)))
            return fail(E2_EINVAL, "arrays must be memory of the current device");
    VerifyParams p{a->tokens && a->max_new ? a->tokens : 0, a->vocab, a->batch, a->max_new, 1, a->logits, a->draft,
                   a->logits_stride, a->draft_stride, a->ids, a->parents, a->starts, a->uniforms, a->temperature,
                   a->kept, a->nodes, a->answer};
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    return a->dtype == E2_F16    ? launch_walks<__half>(p, dev.sms, s)
           : a->dtype == E2_BF16 ? launch_walks<__nv_bfloat16>(p, dev.sms, s)
                                 : launch_walks<float>(p, dev.sms, s);
}
