// verify_drafts.cu -- e2_verify_drafts: which drafted tokens of a tree the target's
// probabilities accept, and the token after them.
#include <atomic>
#include <type_traits>

#include "ops_mma.cuh"
#include "ops_two.cuh"

namespace e2ops {
namespace {

// Bound by latency where there are few requests: some five dependent steps a node (its rows, the block's sums, the
// cluster's barrier, the decision), two microseconds; by the rows' bytes and, at a walk's end, by instructions where
// there are many.  Measured, us: 1 request x 5 nodes of 32,000 tokens 16, 8 x 16 of 128,256 (bf16) 39, 64 x 8 of
// 128,256 (fp32) 137, of which the levels of the longest walk 60 at 5 TB/s, then 30 for the sums in 45 bits (85% of
// issue slots, some 55 an element); 13 x 13 of 50,001 without the draft's rows 20; T = 0, 8 x 16 of 128,256 (bf16) 17.
//
// A cluster of blocks walks a request's tree, and all its warps take the same decisions.  Each
// warp has a run of the vocabulary; what a pass over a row gives is sums, the blocks' of which
// every block gets before one barrier of the cluster.  A node's rows are summed in 32 bits first, and a first child
// that is clear by one part in 2^14 is taken; only what is not, and a walk's end, goes through 45 bits.
// With p = w / Z, w = exp((x - max x) / T), and q likewise of the draft's row, after k rejections
//   P = (p - A q)+ / B,  A_0 = 0, B_0 = 1, A_{k+1} = A_k + B_k, B_{k+1} = sum (p - A_{k+1} q)+,
// as (P - q)+ is (p - A q - B q)+ / B.  Without the draft's rows a rejected token leaves P: all children's are left out of
// the sums and come to what is left one by one, as a difference would leave its rounding where nothing is.  The first of the
// sums of (p - q)+ comes out of the pass that gives Z: by the 32-bit sums it is known well enough which p are above q.
// The token after the last is found in the blocks' sums, the warps', those of an eighth of a
// warp's run, of a lane's share of it, and then element by element.
// Tried: 512 threads of 128 registers (spills went through the caches: 287 for 64 x 8), all parts read from their blocks by
// every warp (5 us a pass), four likely nodes at once whatever the vocabulary (64 x 8 205, 8 x 16 40), two elements in each
// instruction of the 45-bit sums (64 x 8 145: half the independent chains, and spills), groups of six nodes (no faster for ways of two).

constexpr int kThreads = 256, kWarps = kThreads / 32, kMostCluster = 16;
constexpr int kRing = 6144;                      // bytes of a warp's copies on their way
constexpr int kGroup = 4;                        // nodes that are looked at together
static_assert(kGroup * kWarps == 32, "a lane for each node and warp");
constexpr float kNothing = 0x1p-36f;             // a sum below it, of what it is a part of, is rounding's
constexpr float kLeast = 0x1p-40f;               // and what several rejections have left of p below that (p and A q are known to 2^-44)

struct VerifyParams {
    int tokens, vocab, batch, max_new, split;
    const void *logits, *draft;
    int64_t logits_stride, draft_stride;
    const int32_t *ids, *parents, *starts;
    const float *uniforms, *temperature;
    int32_t *kept, *nodes, *answer;
};

// What a warp, or a block, tells the others in a pass.
struct __align__(16) Part {
    Two p, q;                                    // sums
    float p_top, q_top;
    int first;                                   // of the largest
    int bad;
    Two p_more, q_more;                          // sums where p is above the draft's, and p's near the border
    float border;
};

struct Shared {
    float2 table[PowerTable::kSize], shared_table[PowerTable::kSize];
    Part parts[kWarps], blocks[2][kMostCluster];  // (a block may be one pass ahead of another)
    Two sub[kWarps];
    float2 tops[kGroup], sums[kWarps][kGroup], block_sums[2][kMostCluster][kGroup];           // (x, y)
    float2 lane_sums[kWarps][kGroup][32];
    int group[kGroup];                           // the nodes
    int32_t ids[E2_MAX_DRAFT], parents[E2_MAX_DRAFT];
    float uniforms[E2_MAX_DRAFT];
    Two asked[E2_MAX_DRAFT], counted[E2_MAX_DRAFT];            // without the draft's rows: children's weights, alone and in sums
    bool some[E2_MAX_DRAFT];
};

__device__ const PowerTable power_table = PowerTable();

__device__ __forceinline__ void peer_store4(uint32_t at, const float4 &v)
{
    asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(at), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w) : "memory");
}

// w times 2^e, e <= 0, with its second part in its place; 0 from 2^-120 on.
__device__ __forceinline__ Two scaled(const Two &w, int e)
{
    if (e < -120) return Two{0, 0};
    const float f = __int_as_float((e + 127) << 23);
    return sum_of_larger(w.h * f, w.l * f);
}

__device__ __forceinline__ float power2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ __forceinline__ uint32_t bits_of(const float *x) { return __float_as_uint(*x); }
__device__ __forceinline__ uint32_t bits_of(const __half *x) { return *reinterpret_cast<const uint16_t *>(x); }
__device__ __forceinline__ uint32_t bits_of(const __nv_bfloat16 *x) { return *reinterpret_cast<const uint16_t *>(x); }
// The low or the high 16 bits' number.
template <class T> __device__ __forceinline__ float half_of(uint32_t w, int high)
{
    if (std::is_same<T, __half>::value) return __half2float(__ushort_as_half((unsigned short)(high ? w >> 16 : w & 0xffff)));
    return __uint_as_float(high ? w & 0xffff0000u : w << 16);
}

// LONG: runs of which a lane has more than kShort elements, whose sums are closed on the way.  Of 128,256 tokens that is one
// block a request: 160 x 2 in 16 bits 234 us, 216 without.  (One kernel for all would take 1 x 5 x 32,000 17.5 us for 16.4 and
// 64 x 8 x 128,256 in 32 bits 146 for 137.)
constexpr int kShort = 256;

template <class T, bool LONG> struct Walk {
    using Sum = typename std::conditional<LONG, LongerSum, LongSum>::type;
    // A unit of a run: 16 bytes a lane.
    static constexpr int kEach = 16 / sizeof(T), kUnit = 32 * kEach, kStages = kRing / 1024;
    const VerifyParams &p;
    Shared &m;
    int lane, warp, rank, turn;
    int first, end;                              // this warp's run
    uint4 *ring;
    int ring_base;                               // the stage of the run's first unit
    bool ring_fresh;                             // nothing has come into the ring since the group's rows
    const T *x, *y;                              // the node's rows
    int64_t start;                               // the request's first row
    bool wide;                                   // 16-byte loads
    Two heat;                                    // 1 / T
    float x_top, y_top;                          // one of the largest of each
    Two run, block;                              // sums of this warp's run, and of the lane's block
    Two run_q, block_q;                          // split: of the draft's, beside p's, where p is above it
    float border;

    __device__ Walk(const VerifyParams &p, Shared &m, uint8_t *dynamic) : p(p), m(m), turn(0)
    {
        lane = threadIdx.x % 32, warp = threadIdx.x / 32, rank = blockIdx.x % p.split;
        ring = reinterpret_cast<uint4 *>(dynamic + warp * kRing);
        first = run_start(rank * kWarps + warp), end = run_start(rank * kWarps + warp + 1);
    }
    __device__ int run_start(int run) const
    {
        const int64_t units = ((int64_t)p.vocab + kUnit - 1) / kUnit;
        return (int)min(kUnit * (units * run / (kWarps * p.split)), (int64_t)p.vocab);
    }

    // What the lanes have, over the warp, the block and the cluster: join(k) takes in what lanes k apart
    // have, for powers of two below the lanes that there are.
    template <bool MORE = false, class F> __device__ __forceinline__ void exchange(Part &mine, F join)
    {
        auto over = [&](int lanes) {
#pragma unroll 1
            for (int k = 1; k < lanes; k *= 2) join(k);
        };
        over(32);
        run = mine.p;
        if (MORE) run = mine.p_more, run_q = mine.q_more;
        if (lane == 0) m.parts[warp] = mine;
        __syncthreads();
        mine = m.parts[lane % kWarps];
        over(kWarps);
        block = mine.p;
        if (MORE) block = mine.p_more, block_q = mine.q_more;
        if (p.split > 1) {
            if (warp == 0 && lane < p.split) {
                const uint32_t to = peer_addr(smem_addr(&m.blocks[turn][rank]), lane);
                peer_store4(to, make_float4(mine.p.h, mine.p.l, mine.q.h, mine.q.l));
                peer_store4(to + 16, make_float4(mine.p_top, mine.q_top, __int_as_float(mine.first), __int_as_float(mine.bad)));
                if (MORE) {
                    peer_store4(to + 32, make_float4(mine.p_more.h, mine.p_more.l, mine.q_more.h, mine.q_more.l));
                    peer_store4(to + 48, make_float4(mine.border, 0, 0, 0));
                }
            }
            cluster_barrier();
            mine = m.blocks[turn][lane % p.split];
            block = mine.p;
            if (MORE) block = mine.p_more, block_q = mine.q_more;
            over(p.split);
            turn ^= 1;
        } else {
            __syncthreads();                     // (the parts have been read)
        }
    }

    // A lane's elements of a unit.
    struct Lot {
        uint32_t w[4];
    };
    static __device__ __forceinline__ float element(const Lot &e, int j)
    {
        return sizeof(T) == 4 ? __uint_as_float(e.w[j]) : half_of<T>(e.w[j / 2], j % 2);
    }
    __device__ __forceinline__ Lot from_row(const T *row, int at) const
    {
        Lot e;
        if (wide) {
            const uint4 four = *reinterpret_cast<const uint4 *>(row + at + kEach * lane);
            e.w[0] = four.x, e.w[1] = four.y, e.w[2] = four.z, e.w[3] = four.w;
        } else {
            constexpr int kIn = 4 / sizeof(T);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                e.w[k] = bits_of(row + at + 32 * kIn * k + lane);
                if (kIn == 2) e.w[k] |= bits_of(row + at + 32 * kIn * k + 32 + lane) << 16;
            }
        }
        return e;
    }
    // A lane writes and reads its own 16 bytes of the ring only: [stage][row][32].
    __device__ __forceinline__ uint4 *ring_at(int stage, int row) const { return ring + (stage * 2 + row) * 32 + lane; }
    __device__ __forceinline__ void to_ring(const T *from, int stage, int which) const
    {
        copy_async16(smem_addr(ring_at(stage, which)), from, true);
    }
    __device__ __forceinline__ Lot from_ring(int stage, int which) const
    {
        const uint4 four = *ring_at(stage, which);
        return Lot{{four.x, four.y, four.z, four.w}};
    }

    __device__ __forceinline__ const T *row_of(const void *rows, int64_t stride, int node) const
    {
        return static_cast<const T *>(rows) + (start + node) * stride;
    }
    __device__ __forceinline__ void at_node(int node)
    {
        x = row_of(p.logits, p.logits_stride, node);
        y = p.draft ? row_of(p.draft, p.draft_stride, node) : x;
    }
    // This warp's run of the rows of the group's node `place` into the ring, where it holds them; which may be so still.
    __device__ __forceinline__ void fill_ring(bool both, int place, int count)
    {
        const int units = (end - first) / kUnit;
        ring_base = 0;
        if (!wide || units > kStages) return;
        if (ring_fresh && (count - place) * units <= kStages) {
            ring_base = place * units % kStages;
            return;
        }
        ring_fresh = false;
        for (int u = 0; u < units; ++u) {
            to_ring(x + first + u * kUnit + kEach * lane, u, 0);
            if (both) to_ring(y + first + u * kUnit + kEach * lane, u, 1);
        }
        copy_commit();
        copy_wait<0>();
    }

    // In 32 bits, of the group's nodes g < count: sums of 2^((x - top) log2 e / T), and of y's (bit g of `both`).  Lane g kWarps
    // has node g's.  The tops are the largest of a few of the row.  Rows come through the ring one after the other.
    __device__ __forceinline__ void estimate(int count, unsigned both, float &x_sum, float &y_sum)
    {
        const int units = (end - first) / kUnit;
        // (where the next copies come from: a node's next unit)
        int next_node = 0, next_unit = 0;
        const T *next_x = nullptr, *next_y = nullptr;
        ring_fresh = true;
        auto issue = [&](int stage) {
            if (next_node < count && units > 0) {
                if (next_unit == 0) {
                    next_x = row_of(p.logits, p.logits_stride, m.group[next_node]) + first + kEach * lane;
                    next_y = both >> next_node & 1 ? row_of(p.draft, p.draft_stride, m.group[next_node]) + first + kEach * lane : nullptr;
                }
                to_ring(next_x, stage, 0);
                next_x += kUnit;
                if (next_y) {
                    to_ring(next_y, stage, 1);
                    next_y += kUnit;
                }
                if (++next_unit == units) next_unit = 0, ++next_node;
            }
            copy_commit();
        };
        if (wide) {
#pragma unroll
            for (int k = 0; k < kStages; ++k) issue(k);
        }
        // the tops: a warp for each node's row
        static_assert(2 * kGroup == kWarps, "a warp for each row");
        {
            const int g = warp / 2;
            float a = -INFINITY;
            if (g < count && (warp % 2 == 0 || (both >> g & 1))) {
                const T *u = warp % 2 ? row_of(p.draft, p.draft_stride, m.group[g]) : row_of(p.logits, p.logits_stride, m.group[g]);
#pragma unroll
                for (int j = 0; j < 4; ++j) a = fmaxf(a, to_float(u[(int)((int64_t)p.vocab * (4 * lane + j) / 128)]));
#pragma unroll
                for (int k = 16; k; k /= 2) a = fmaxf(a, __shfl_xor_sync(~0u, a, k));
            }
            if (lane == 0) reinterpret_cast<float *>(m.tops)[warp] = a;
        }
        __syncthreads();
        const float2 *tops = m.tops;
        const float f = heat.h * 1.44269504f;
        // (a sum of n is off by n 2^-24 at most: 128 at a time, these with what rounding takes)
        constexpr int kClose = kShort / kEach;
        int stage = 0;
        // (a unit each, and all in the ring: two nodes side by side)
        const bool side_by_side = wide && end - first == kUnit && count > 1;
        if (side_by_side) {
            copy_wait<0>();
#pragma unroll 2
            for (int g = 0; g < count; ++g) {
                const float ca = tops[g].x * f, cb = tops[g].y * f;
                const Lot e = from_ring(g, 0), d = from_ring(g, 1);
                float sa[2] = {0, 0}, sb[2] = {0, 0};
#pragma unroll
                for (int j = 0; j < kEach; ++j)
                    sa[j % 2] += power2(__fmaf_rn(element(e, j), f, -ca)), sb[j % 2] += power2(__fmaf_rn(element(d, j), f, -cb));
                m.lane_sums[warp][g][lane] = make_float2(sa[0] + sa[1], both >> g & 1 ? sb[0] + sb[1] : 0.0f);
            }
        }
#pragma unroll 1
        for (int g = side_by_side ? count : 0; g < count; ++g) {
            const bool two = both >> g & 1;
            const float ca = tops[g].x * f, cb = tops[g].y * f;
            const T *u = row_of(p.logits, p.logits_stride, m.group[g]), *v = two ? row_of(p.draft, p.draft_stride, m.group[g]) : u;
            float sa[2] = {0, 0}, sb[2] = {0, 0};
            LongSum closed_a, closed_b;
            auto close = [&] {
                closed_a.add(Two{sa[0] + sa[1], 0}), closed_b.add(Two{sb[0] + sb[1], 0});
                sa[0] = sa[1] = sb[0] = sb[1] = 0;
            };
#pragma unroll 1
            for (int unit = 0; unit < units;) {
                if (LONG && unit > 0) close();
                const int until = LONG ? min(unit + kClose, units) : units;
#pragma unroll 1
                for (; unit < until; ++unit) {
                    Lot e, d;
                    if (wide) {
                        copy_wait<kStages - 1>();
                        e = from_ring(stage, 0);
                        if (two) d = from_ring(stage, 1);
                        issue(stage);
                    } else {
                        e = from_row(u, first + unit * kUnit);
                        if (two) d = from_row(v, first + unit * kUnit);
                    }
#pragma unroll
                    for (int j = 0; j < kEach; ++j) sa[j % 2] += power2(__fmaf_rn(element(e, j), f, -ca));
                    if (two) {
#pragma unroll
                        for (int j = 0; j < kEach; ++j) sb[j % 2] += power2(__fmaf_rn(element(d, j), f, -cb));
                    }
                    stage = stage == kStages - 1 ? 0 : stage + 1;
                }
            }
#pragma unroll 1
            for (int i = first + units * kUnit + lane; i < end; i += 32) {
                sa[0] += power2(__fmaf_rn(to_float(u[i]), f, -ca));
                if (two) sb[0] += power2(__fmaf_rn(to_float(v[i]), f, -cb));
            }
            if (LONG) {
                close();
                sa[0] = closed_a.value().h, sb[0] = closed_b.value().h;
            }
            m.lane_sums[warp][g][lane] = make_float2(sa[0] + sa[1], sb[0] + sb[1]);
        }
        // the warp's, the block's, the cluster's
        const int g = lane / kWarps, part = lane % kWarps;
        auto over = [&](float2 &sum) {
#pragma unroll
            for (int k = 1; k < kWarps; k *= 2) sum.x += __shfl_xor_sync(~0u, sum.x, k), sum.y += __shfl_xor_sync(~0u, sum.y, k);
        };
        __syncwarp();
        {
            float2 mine = make_float2(0, 0);
            if (g < count) {
#pragma unroll
                for (int k = 0; k < 32; k += kWarps) {
                    const float2 theirs = m.lane_sums[warp][g][part + k];
                    mine.x += theirs.x, mine.y += theirs.y;
                }
            }
            over(mine);
            if (part == 0) m.sums[warp][g] = mine;
        }
        __syncthreads();
        float2 sum = g < count ? m.sums[part][g] : make_float2(0, 0);
        over(sum);
        if (p.split > 1) {
            if (warp == 0) {
                for (int to = part; to < p.split; to += kWarps) {
                    const uint32_t at = peer_addr(smem_addr(&m.block_sums[turn][rank][g]), to);
                    asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(at), "f"(sum.x), "f"(sum.y) : "memory");
                }
            }
            cluster_barrier();
            sum = make_float2(0, 0);
            for (int from = part; from < p.split; from += kWarps) {
                const float2 theirs = m.block_sums[turn][from][g];
                sum.x += theirs.x, sum.y += theirs.y;
            }
            over(sum);
            turn ^= 1;
        } else {
            __syncthreads();                     // (the sums have been read)
        }
        x_sum = sum.x, y_sum = sum.y;
    }

    // Whether a token is one of these nodes'.
    __device__ __forceinline__ bool among(uint64_t nodes, int v) const
    {
        for (; nodes; nodes &= nodes - 1)
            if (m.ids[__ffsll(nodes) - 1] == v) return true;
        return false;
    }
    // The same run again, f(two elements of x, of y): a short loop, as f is long; close(times) after every 32 of a lane's
    // elements.  LEAVE: without the tokens of `out`'s nodes.
    template <bool BOTH, bool LEAVE = false, class F, class G> __device__ __forceinline__ void pairs(F f, G close, uint64_t out = 0) const
    {
        constexpr int kStep = sizeof(T) / 2;                              // words of two elements
        const int units = (end - first) / kUnit, rest = end - first - units * kUnit;
        const bool kept = wide && units <= kStages;
        const int leave = LEAVE && out ? m.ids[__ffsll(out) - 1] : -1;        // (a run has one at most, as a rule)
        Lot a, b;
        if (units > 0 && !kept) {
            a = from_row(x, first);
            if (BOTH) b = from_row(y, first);
        }
#pragma unroll 1
        for (int unit = 0; unit < units + (rest > 0); ++unit) {
            Lot u = a, v = b;
            const int at = first + unit * kUnit;
            if (kept && unit < units) {
                const int stage = ring_base + unit >= kStages ? ring_base + unit - kStages : ring_base + unit;
                u = from_ring(stage, 0);
                if (BOTH) v = from_ring(stage, 1);
            } else if (unit + 1 < units) {
                a = from_row(x, at + kUnit);
                if (BOTH) b = from_row(y, at + kUnit);
            }
#pragma unroll 1
            for (int k = 0; k < kEach / 2; ++k) {
                float c[2] = {element(u, 0), element(u, 1)}, d[2] = {0, 0};
                if (BOTH) d[0] = element(v, 0), d[1] = element(v, 1);
                if (unit == units) {                                          // (the rest of the row)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int i = at + 64 * k + 32 * e + lane;
                        c[e] = i < end ? to_float(x[i]) : -INFINITY;
                        if (BOTH) d[e] = i < end ? to_float(y[i]) : -INFINITY;
                    }
                }
                if (LEAVE && out) {
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int i = at + (wide && unit < units ? kEach * lane + 2 * k + e : 64 * k + 32 * e + lane);
                        if (i == leave || among(out & (out - 1), i)) c[e] = -INFINITY;
                    }
                }
                f(c, d);
#pragma unroll
                for (int w = 0; w + kStep < 4; ++w) {
                    u.w[w] = u.w[w + kStep];
                    if (BOTH) v.w[w] = v.w[w + kStep];
                }
            }
            constexpr int kClose = 32 / kEach;
            if (LONG && unit % kClose == kClose - 1) close(unit / kClose);
        }
    }

    // The largest of x (and of y): whether both rows have a distribution, and x's first largest.
    __device__ __forceinline__ bool tops(bool both, int &where)
    {
        Part mine{{0, 0}, {0, 0}, -INFINITY, -INFINITY, 0x7fffffff, 0};
        for (int i0 = first; i0 < end; i0 += kUnit)
#pragma unroll
            for (int j = 0; j < kEach; ++j) {
                const int i = i0 + 32 * j + lane;
                const float a = i < end ? to_float(x[i]) : -INFINITY, b = both && i < end ? to_float(y[i]) : -INFINITY;
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
        exchange(mine, [&](int k) {
            join(__shfl_xor_sync(~0u, mine.p_top, k), __shfl_xor_sync(~0u, mine.q_top, k), __shfl_xor_sync(~0u, mine.first, k),
                 __shfl_xor_sync(~0u, mine.bad, k));
        });
        x_top = mine.p_top, y_top = mine.q_top, where = mine.first;
        return !mine.bad && x_top > -INFINITY && (!both || y_top > -INFINITY);
    }

    // What P is of, of an element: w, or (w - the draft's)+.
    static __device__ __forceinline__ Two less_of(const Two &a, const Two &b)
    {
        const Two s = sum_of(a.h, -b.h);
        const Two d = sum_of_larger(s.h, s.l + (a.l - b.l));
        return d.h > 0 ? d : Two{0, 0};
    }
    // (the draft's weights carry their share in their table)
    __device__ __forceinline__ Two weight(int i, bool less, const Weigher of_x, const Weigher of_y) const
    {
        const Two a = of_x.of(to_float(x[i]), m.table);
        return less ? less_of(a, of_y.of(to_float(y[i]), m.shared_table)) : a;
    }
    // All threads of the block: from here on the draft's weights are times `share`.
    __device__ void set_share(const Two &share)
    {
        __syncthreads();
        for (int i = threadIdx.x; i < PowerTable::kSize; i += kThreads) {
            const Two w = Two{m.table[i].x, m.table[i].y} * share;
            m.shared_table[i] = float2{w.h, w.l};
        }
        __syncthreads();
    }

    // Sums by runs and whole: of x's weights, and of y's (LESS: of x's less y's share instead); x's without the tokens
    // of `out`'s nodes.
    template <bool BOTH, bool LESS> __device__ __forceinline__ Two sums(const Weigher of_x, const Weigher of_y, Two &q, uint64_t out = 0)
    {
        Sum a, b;
        if (out) {
            auto mine = [&](int c) { return __ballot_sync(~0u, out >> c & 1 && m.ids[c] >= first && m.ids[c] < end); };
            out = mine(lane) | (uint64_t)mine(lane + 32) << 32;
        }
        pairs<BOTH || LESS, !BOTH && !LESS>([&](const float (&u)[2], const float (&v)[2]) {
            Two w[2], d[2];
            of_x.of(u, m.table, w);
            if (BOTH || LESS) of_y.of(v, LESS ? m.shared_table : m.table, d);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                a.add(LESS ? less_of(w[j], d[j]) : w[j]);
                if (BOTH) b.add(d[j]);
            }
        }, [&](int times) {
            a.close(times);
            if (BOTH) b.close(times);
        }, out);
        Part mine{a.total(), BOTH ? b.total() : Two{0, 0}, 0, 0, 0, 0};
        exchange(mine, [&](int k) {
            mine.p = mine.p + shuffle_xor(mine.p, k);
            if (BOTH) mine.q = mine.q + shuffle_xor(mine.q, k);
        });
        q = mine.q;
        return mine.p;
    }

    // x's sum and y's, and by the way what (x - share y)+ sums to, for a share that is known to some 2^-20 only (`near`):
    // x and y are summed where x is above near y, which is where it is above share y but for elements within the
    // difference of the two, of which no more than that difference counts; `border` sums x within 2^-20 of it.
    __device__ __forceinline__ Two split(const Weigher of_x, const Weigher of_y, float near, Two &q)
    {
        Sum a[2], b[2];
        float edge = 0;
        pairs<true>([&](const float (&u)[2], const float (&v)[2]) {
            Two w[2], d[2];
            of_x.of(u, m.table, w);
            of_y.of(v, m.table, d);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const float over = __fmaf_rn(-near, d[j].h, w[j].h);
                const bool above = over > 0;
                if (fabsf(over) < 0x1p-20f * w[j].h) edge += w[j].h;
                LongSum x{above ? a[1].s : a[0].s, above ? a[1].c : a[0].c}, y{above ? b[1].s : b[0].s, above ? b[1].c : b[0].c};
                x.add(w[j]);
                y.add(d[j]);
                a[1].s = above ? x.s : a[1].s, a[1].c = above ? x.c : a[1].c, b[1].s = above ? y.s : b[1].s, b[1].c = above ? y.c : b[1].c;
                a[0].s = above ? a[0].s : x.s, a[0].c = above ? a[0].c : x.c, b[0].s = above ? b[0].s : y.s, b[0].c = above ? b[0].c : y.c;
            }
        }, [&](int times) { a[0].close(times), a[1].close(times), b[0].close(times), b[1].close(times); });
        Part mine{a[0].total(), b[0].total(), 0, 0, 0, 0, a[1].total(), b[1].total(), edge};
        exchange<true>(mine, [&](int k) {
            mine.p = mine.p + shuffle_xor(mine.p, k);
            mine.q = mine.q + shuffle_xor(mine.q, k);
            mine.p_more = mine.p_more + shuffle_xor(mine.p_more, k);
            mine.q_more = mine.q_more + shuffle_xor(mine.q_more, k);
            mine.border += __shfl_xor_sync(~0u, mine.border, k);
        });
        border = mine.border;
        q = mine.q + mine.q_more;
        return mine.p + mine.p_more;
    }
    // After it: run and block of (x - share y)+, and its sum; false where the border's part of it may be above 2^-37.
    // What is so little of x that it may be all rounding is nothing, so that whoever has something has an element with
    // something: sums of the two are off by 2^-36.8 each at worst, and a block that has something has a run that does.
    __device__ __forceinline__ bool take_split(const Two &share, float near, Two &sum)
    {
        auto of = [&](const Two &x, const Two &y, float least) {
            const Two d = x - share * y;
            return d.h > least * x.h ? d : Two{0, 0};
        };
        sum = warp_sum(lane < p.split ? of(block, block_q, 0x1p-34f) : Two{0, 0});
        // (2^-22: what the comparisons were rounded by)
        const float off = fabsf(__fdiv_rn((share - Two{near, 0}).h, near)) + 0x1p-22f;
        if (!(off < 0x1p-20f && off * border <= 0x1p-37f * sum.h)) return false;
        run = of(run, run_q, 0x1p-35f), block = of(block, block_q, 0x1p-34f);
        return true;
    }

    // The first v whose share of the sums in order passes u, in one warp of one block, which it
    // returns true to.  gone(i): tokens that P has lost.
    template <class F> __device__ __forceinline__ bool find(float u, bool less, const Weigher of_x, const Weigher of_y, F gone, int &answer)
    {
        // of `lanes` lanes' sums, one after the other, the first that passes the target: which one, and what is before it
        // (by rounding none may seem to: the last that has anything)
        Two target, base{0, 0};
        auto choose = [&](Two mine, int lanes) {
            if (lane >= lanes) mine = Two{0, 0};
            const Two up_to = base + warp_prefix(mine, lane);
            Two before{__shfl_up_sync(~0u, up_to.h, 1), __shfl_up_sync(~0u, up_to.l, 1)};
            if (lane == 0) before = base;
            const unsigned some = __ballot_sync(~0u, mine.h > 0), hit = __ballot_sync(~0u, mine.h > 0 && target < up_to);
            const int which = hit ? __ffs(hit) - 1 : some ? 31 - __clz(some) : 0;
            base = Two{__shfl_sync(~0u, before.h, which), __shfl_sync(~0u, before.l, which)};
            return which;
        };
        target = Two{u, 0} * warp_sum(lane < p.split ? block : Two{0, 0});
        if (choose(block, p.split) != rank) return false;
        if (lane == 0) m.sub[warp] = run;
        __syncthreads();
        const int found = rank * kWarps + choose(m.sub[lane % kWarps], kWarps);
        __syncthreads();
        // its parts, one a warp
        const int run_from = run_start(found), run_stop = run_start(found + 1);
        auto part_of = [&](int k) { return run_from + (int)((int64_t)(run_stop - run_from) * k / kWarps); };
        // a lane's share of them is side by side, too
        const int start = part_of(warp), stop = part_of(warp + 1), share = (stop - start + 31) / 32;
        Sum a;
#pragma unroll 1
        for (int k = 0, i = start + lane * share; k < share && i < stop; ++k, ++i) {
            if (!gone(i)) a.add(weight(i, less, of_x, of_y));
            if (LONG && k % 32 == 31) a.close(k / 32);
        }
        const Two mine = a.total(), sub = warp_sum(mine);
        if (lane == 0) m.sub[warp] = sub;
        __syncthreads();
        if (choose(m.sub[lane % kWarps], kWarps) != warp) return false;
        const int from = start + choose(mine, 32) * share, to = min(from + share, stop);
        // element by element
        answer = -1;
#pragma unroll 1
        for (int i0 = from; i0 < to; i0 += 32) {
            const int i = i0 + lane;
            const Two w = i < to && !gone(i) ? weight(i, less, of_x, of_y) : Two{0, 0};
            const Two sum = base + warp_prefix(w, lane);
            const unsigned some = __ballot_sync(~0u, w.h > 0), hit = __ballot_sync(~0u, w.h > 0 && target < sum);
            if (some) answer = i0 + (hit ? __ffs(hit) - 1 : 31 - __clz(some));
            if (hit) break;
            base = Two{__shfl_sync(~0u, sum.h, 31), __shfl_sync(~0u, sum.l, 31)};
        }
        return true;
    }
};

// (two kernels, as one for rows with and without the draft's keeps more than its registers)
template <class T, bool DRAFT, bool LONG> __global__ void __launch_bounds__(kThreads, 2) verify_kernel(const VerifyParams p)
{
    __shared__ Shared m;
    const int request = blockIdx.x / p.split;
    wait_before();
    allow_next();
    if (p.split > 1) asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory");
    extern __shared__ __align__(16) uint8_t dynamic[];
    Walk<T, LONG> walk(p, m, dynamic);
    const bool writer = walk.rank == 0 && threadIdx.x == 0;
    const int64_t start = p.starts[request], stop = p.starts[request + 1];
    const int n = start >= 0 && stop <= p.tokens ? (int)min(max(stop - start, (int64_t)0), (int64_t)p.max_new) : 0;
    for (int i = threadIdx.x; i < PowerTable::kSize; i += kThreads) m.table[i] = power_table.v[i];
    if (threadIdx.x < n) {
        m.ids[threadIdx.x] = p.ids[start + threadIdx.x];
        const int parent = p.parents[start + threadIdx.x];
        m.parents[threadIdx.x] = parent < (int)threadIdx.x ? parent : -1;
        const float u = p.uniforms[start + threadIdx.x];
        m.uniforms[threadIdx.x] = u > 0 ? fminf(u, 1.0f) : 0.0f;
    }
    __syncthreads();
    int32_t *nodes = p.nodes + (int64_t)request * p.max_new, *answer = p.answer + (int64_t)request * p.max_new;
    const float degree = p.temperature ? p.temperature[request] : 1.0f;
    const bool greedy = degree == 0, heated = degree > 0 && degree < INFINITY;
    walk.heat = heated ? Two{1, 0} / Two{fmaxf(degree, 0x1p-126f), 0} : Two{1, 0};
    auto inside = [&](int v) { return v >= 0 && v < p.vocab; };

    const int parent0 = walk.lane > 0 && walk.lane < n ? m.parents[walk.lane] : -1, parent1 = walk.lane + 32 < n ? m.parents[walk.lane + 32] : -1;

    walk.start = start;
    auto rows_at = [&](const void *rows, int64_t stride) {
        return reinterpret_cast<uintptr_t>(rows) | (start + n > 1 ? (uintptr_t)stride * sizeof(T) : 0);
    };
    walk.wide = (rows_at(p.logits, p.logits_stride) | (DRAFT ? rows_at(p.draft, p.draft_stride) : 0)) % 16 == 0;
    // (bit c: node c is a child)
    auto children_of = [&](int node) {
        return __ballot_sync(~0u, parent0 == node) | (uint64_t)__ballot_sync(~0u, parent1 == node) << 32;
    };
    auto first_of = [](uint64_t set) { return __ffsll(set) - 1; };
    // A node is looked at together with its first child, that one's first child, and so on, as long as the ring holds
    // them all: for small vocabularies, where a pass is latency, one does for up to four nodes.  (For larger ones, or
    // without the draft's rows, what is not accepted costs more: 8 x 16 x 128,256 40 us for 37.)
    const int runs = kWarps * p.split, run_units = ((p.vocab + Walk<T, LONG>::kUnit - 1) / Walk<T, LONG>::kUnit + runs - 1) / runs;
    const int at_once = DRAFT && walk.wide ? max(min(kGroup, Walk<T, LONG>::kStages / run_units), 1) : 1;
    int place = 0, count = 0;                             // of the node in its group; the group's nodes
    float x_sums = 0, y_sums = 0, child_value = 0;        // lane g kWarps: node g's; and the one after it: its first child's logits

    // (the cluster's blocks run, so that what goes to them has a place)
    if (p.split > 1) asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
    int here = 0, kept = n > 0;
    int token = -1;                                       // the token after the last, in the thread that knows it
    bool knows = writer;
    while (n > 0 && (greedy || heated)) {
        walk.at_node(here);
        const uint64_t children = children_of(here);
        const bool both = DRAFT && children && heated;
        int accepted = -1, first;
        if (greedy) {
            if (!walk.tops(false, first)) break;
            for (uint64_t set = children; set && accepted < 0; set &= set - 1)
                if (m.ids[first_of(set)] == first) accepted = first_of(set);
            if (accepted < 0) token = first;
        }
        float x_sum = 0, y_sum = 0, first_x = 0, first_y = 0;
        bool clear = false;
        if (!greedy) {
            // In 32 bits first: exponents are off by 2^-18 at most (of 64, and 2^-18 of that in f), sums by 2^-17,
            // so what is clear by one part in 2^14 is clear.
            constexpr float kClear = 0x1p-14f;
            const int child0 = children ? first_of(children) : 0;
            if (++place >= count || m.group[place] != here) {
                unsigned twos = 0;
                int node = here, my_node = 0, my_child = -1;
                place = count = 0;
                __syncthreads();
                for (uint64_t below = children;; below = children_of(node)) {
                    if (threadIdx.x == 0) m.group[count] = node;
                    if (DRAFT && below) twos |= 1u << count;
                    if (walk.lane / kWarps == count) my_node = node, my_child = below ? first_of(below) : -1;
                    if (++count == at_once || !below) break;
                    node = first_of(below);
                }
                // (the first children's logits are asked for now, looked at later)
                T value = from_float<T>(-INFINITY);
                const int v = my_child >= 0 ? m.ids[my_child] : -1;
                if (inside(v) && (walk.lane % kWarps == 0 || (walk.lane % kWarps == 1 && DRAFT)))
                    value = walk.lane % kWarps ? walk.row_of(p.draft, p.draft_stride, my_node)[v] : walk.row_of(p.logits, p.logits_stride, my_node)[v];
                __syncthreads();
                walk.estimate(count, twos, x_sums, y_sums);
                child_value = to_float(value);
            }
            first_x = __shfl_sync(~0u, child_value, place * kWarps), first_y = __shfl_sync(~0u, child_value, place * kWarps + 1);
            x_sum = __shfl_sync(~0u, x_sums, place * kWarps), y_sum = __shfl_sync(~0u, y_sums, place * kWarps);
            walk.x_top = m.tops[place].x, walk.y_top = m.tops[place].y;
            // (a NaN, or +inf, is in the sum; a sample without a token, or with none of the large ones, too)
            constexpr float kSome = 0.5f, kMost = 0x1p62f;
            clear = x_sum > kSome && x_sum < kMost && (!both || (y_sum > kSome && y_sum < kMost));
            if (!clear) {
                if (!walk.tops(both, first)) break;
            } else if (children) {
                const float f = walk.heat.h * 1.44269504f, cx = walk.x_top * f, cy = walk.y_top * f;
                if (DRAFT) {
                    const float w = power2(__fmaf_rn(first_x, f, -cx)) * y_sum, u = m.uniforms[child0];
                    const float asked = u * power2(__fmaf_rn(first_y, f, -cy)) * x_sum;
                    // (numbers that 32 bits do not hold are not clear)
                    if (w > 0x1p-60f && asked < w * (1 - kClear)) accepted = child0;
                } else {
                    float left = x_sum;
                    bool certain = true;
                    for (uint64_t set = children; set && certain && accepted < 0; set &= set - 1) {
                        const int c = first_of(set), v = m.ids[c];
                        if (!inside(v)) continue;
                        for (uint64_t done = children ^ set; done; done &= done - 1) certain &= m.ids[first_of(done)] != v;
                        const float w = power2(__fmaf_rn(c == child0 ? first_x : to_float(walk.x[v]), f, -cx)), asked = m.uniforms[c] * left;
                        if (!certain || !(w > 0x1p-60f)) certain = false;
                        else if (asked < w * (1 - kClear)) accepted = c;
                        else if (asked > w * (1 + kClear) && left - w > 0.25f * x_sum) left -= w;
                        else certain = false;
                    }
                }
            }
        }
        if (!greedy && accepted < 0) {
            walk.fill_ring(both, place, count);
            const Weigher of_x(walk.x_top, walk.heat), of_y(both ? walk.y_top : walk.x_top, walk.heat);
            const Two none{0, 0};
            Two q = none, A = none, B{1, 0};
            // (in 32 bits, of what the weights sum to here)
            float near = 0;
            if (both && clear) {
                const float f = walk.heat.h * 1.44269504f;
                const float wx = of_x.of(walk.x_top, m.table).h * x_sum * power2(__fmaf_rn(walk.y_top, f, -(walk.y_top * f)));
                const float wy = of_y.of(walk.y_top, m.table).h * y_sum * power2(__fmaf_rn(walk.x_top, f, -(walk.x_top * f)));
                near = __fdiv_rn(wx, wy);
            }
            // without the draft's rows: the children whose tokens are some, a thread each (its logit is asked for now)
            uint64_t drafted = 0;
            T value = from_float<T>(-INFINITY);
            if (!DRAFT && children) {
                const int a = walk.lane, b = walk.lane + 32, c = threadIdx.x;
                drafted = __ballot_sync(~0u, children >> a & 1 && inside(m.ids[a])) |
                          (uint64_t)__ballot_sync(~0u, children >> b & 1 && inside(m.ids[b])) << 32;
                if (c < E2_MAX_DRAFT && drafted >> c & 1) value = walk.x[m.ids[c]];
            }
            const Two all = near > 0 ? walk.split(of_x, of_y, near, q)
                            : both   ? walk.template sums<true, false>(of_x, of_y, q)
                                     : walk.template sums<false, false>(of_x, of_x, q, drafted);
            const bool parted = near > 0;
            // what P has: what is no child's, and the children's tokens that are not lost (bits k: this lane's nodes lane + 32 k)
            auto left_of = [&](unsigned out) {
                return all + warp_sum((out & 1 ? none : m.counted[walk.lane]) + (out & 2 ? none : m.counted[walk.lane + 32]));
            };
            unsigned out = 0;
            Two left = all;
            if (drafted) {
                const int c = threadIdx.x;
                if (c < E2_MAX_DRAFT) {
                    Two w = none, in_sums = none;
                    bool some = false;
                    if (drafted >> c & 1) {
                        int e;
                        some = of_x.wide(to_float(value), m.table, w, e);
                        w = scaled(w, some ? e : -127);
                        // (a token of several children is in the sums once)
                        if (!walk.among(drafted & ((1ull << c) - 1), m.ids[c])) in_sums = of_x.of(to_float(value), m.table);
                    }
                    m.asked[c] = w, m.counted[c] = in_sums, m.some[c] = some;
                }
                __syncthreads();
                left = left_of(out);
            }
            uint64_t lost = 0;                            // rejected children whose tokens P has lost
            bool less = false;
            auto gone = [&](int v) { return walk.among(lost, v); };
            for (uint64_t set = children; set; set &= set - 1) {
                const int c = first_of(set), v = m.ids[c];
                const bool in = inside(v);
                const float u = m.uniforms[c];
                if (DRAFT) {
                    // its weight, however small
                    Two w = none, wq = none;
                    int e = 0, eq = 0;
                    const bool known = c == first_of(children);
                    const bool some = in && of_x.wide(known ? first_x : to_float(walk.x[v]), m.table, w, e);
                    // u q(v) < P(v), times Z_p Z_q B and a power of two
                    const bool some_q = in && of_y.wide(known ? first_y : to_float(walk.y[v]), m.table, wq, eq);
                    const int most = some && some_q ? max(e, eq) : some ? e : eq;
                    w = scaled(w, some ? e - most : -127);
                    wq = scaled(wq, some_q ? eq - most : -127);
                    const Two mine = w * q - A * wq * all;
                    if ((u == 0 && !less && some) || Two{u, 0} * wq * all * B < (mine.h > 0 ? mine : none)) {
                        accepted = c;
                        break;
                    }
                    const Two run = walk.run, block = walk.block;
                    Two unused;
                    const Two more = A + B, share = more * all / q;
                    Two sum;
                    const bool enough = near > 0 && walk.take_split(share, near, sum);
                    walk.set_share(share);
                    if (!enough) sum = walk.template sums<false, true>(of_x, of_y, unused);
                    near = 0;                             // (the first child's only)
                    sum = sum / all;
                    if (sum.h > fmaxf(kNothing * B.h, kLeast)) {
                        A = more, B = sum, less = true;
                    } else {
                        // (p's own, which a split has not left)
                        if (parted && !less) walk.template sums<false, false>(of_x, of_x, unused);
                        else walk.run = run, walk.block = block;
                        walk.set_share(A * all / q);
                    }
                } else if (in && !gone(v)) {
                    const Two w = m.asked[c];
                    if ((u == 0 && m.some[c]) || Two{u, 0} * left < w) {
                        accepted = c;
                        break;
                    }
                    const unsigned more = out | (m.ids[walk.lane] == v) | (m.ids[walk.lane + 32] == v) << 1;
                    const Two rest = left_of(more);
                    if (m.some[c] && rest.h > kNothing * left.h) left = rest, out = more, lost |= 1ull << c;
                }
            }
            if (accepted < 0) {
                // the children's tokens that P has kept, in their runs and blocks
                for (uint64_t set = drafted; set; set &= set - 1) {
                    const int c = first_of(set), v = m.ids[c], owner = walk.lane % p.split;
                    if (gone(v)) continue;
                    if (v >= walk.first && v < walk.end) walk.run = walk.run + m.counted[c];
                    if (v >= walk.run_start(owner * kWarps) && v < walk.run_start((owner + 1) * kWarps)) walk.block = walk.block + m.counted[c];
                }
            }
            if (accepted < 0) knows = walk.find(m.uniforms[0], less, of_x, of_y, gone, token) && walk.lane == 0;
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
    // (what goes to other blocks goes before a barrier of the cluster, so blocks may end one by one)
}

// How many clusters of 2^i blocks run at once.
template <class T, bool DRAFT, bool LONG> int clusters_of(int i, int dev)
{
    static std::atomic<int> known[64][5];                    // one more
    int n = known[dev][i].load(std::memory_order_relaxed);
    if (n == 0) {
        cudaLaunchAttribute at{};
        at.id = cudaLaunchAttributeClusterDimension;
        at.val.clusterDim.x = 1u << i, at.val.clusterDim.y = at.val.clusterDim.z = 1;
        cudaLaunchConfig_t cfg{};
        cfg.gridDim = dim3(1u << 10);
        cfg.blockDim = dim3(kThreads);
        cfg.dynamicSmemBytes = kWarps * kRing;
        cfg.attrs = &at;
        cfg.numAttrs = 1;
        if (cudaFuncSetAttribute(verify_kernel<T, DRAFT, LONG>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess ||
            cudaFuncSetAttribute(verify_kernel<T, DRAFT, LONG>, cudaFuncAttributeMaxDynamicSharedMemorySize, kWarps * kRing) != cudaSuccess ||
            cudaOccupancyMaxActiveClusters(&n, verify_kernel<T, DRAFT, LONG>, &cfg) != cudaSuccess) {
            cudaGetLastError();
            n = 0;
        }
        known[dev][i].store(++n, std::memory_order_relaxed);
    }
    return n - 1;
}

// Requests over clusters, as large as all of them run at once, and as a warp's run is 256 elements.
template <class T, bool DRAFT, bool LONG> int launch_walks(VerifyParams p, const Device &dev, cudaStream_t s)
{
    constexpr int kUnit = Walk<T, LONG>::kUnit;
    int i = 4;
    while (i > 0 && (p.batch > clusters_of<T, DRAFT, LONG>(i, dev.id) || p.vocab < (kWarps * kUnit << i) / 2)) --i;
    p.split = 1 << i;
    if constexpr (!LONG) {
        const int runs = kWarps * p.split, run_units = ((p.vocab + kUnit - 1) / kUnit + runs - 1) / runs;
        if (run_units > kShort / Walk<T, LONG>::kEach) return launch_walks<T, DRAFT, true>(p, dev, s);
    }
    return launch<VerifyParams>(verify_kernel<T, DRAFT, LONG>, dim3((unsigned)p.batch * p.split), kThreads, kWarps * kRing, p.split, true, s, p);
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
    auto as = [&](auto draft) {
        constexpr bool kDraft = decltype(draft)::value;
        return a->dtype == E2_F16    ? launch_walks<__half, kDraft, false>(p, dev, s)
               : a->dtype == E2_BF16 ? launch_walks<__nv_bfloat16, kDraft, false>(p, dev, s)
                                     : launch_walks<float, kDraft, false>(p, dev, s);
    };
    return a->draft ? as(std::true_type{}) : as(std::false_type{});
}
