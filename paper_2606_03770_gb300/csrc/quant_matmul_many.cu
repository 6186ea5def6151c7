// quant_matmul_many.cu -- e2_quant_matmul for prompts.
//
// Bound by the fifth-generation tensor cores.  A block takes 128 weight rows (gated: 64 that
// gate and the 64 that they gate) and up to 256 tokens: D[rows][tokens] = W x^T, W and D
// in tensor memory, x in shared memory.  One warp copies x, prepared beforehand
// as the images of its stages (one bulk copy each), one issues the products, sixteen
// unpack weights, four a stage: a thread a row's 64 columns, to fp16 with their scale, one
// rounding (2^-11 of a weight; |W| up to 65504).  (Unpacked into shared memory instead, a
// stage took 520 ns whatever its tokens, and 370 with each thread loading its own row, a line a
// lane.)  Elements stay in the order that unpacking leaves (0, 4, 1, 5, 2, 6, 3, 7 of each
// eight), x is put into the same one.  Few rows are split over columns by the blocks of a
// cluster, whose sums are joined in a fixed order through shared memory.
//
// Measured with 1,152 tokens, us: 8192 x 28672 399 (1,356 TFLOP/s, 71% of the tensor cores'
// measured rate; 446 over weights of 300 MB in turn, 453 one call after another, where the power
// limit lowers the clock), 57344 x 8192 gated 853 (1,269), 10240 x 8192 163 (1,184), 4096 x 4096
// 49; 17 tokens 69, 118, 39 and 12.  Looking whether a stage's weights stay in range is 0 to 2% of it.
// Lost: turns that do not come
// out even on 152 multiprocessors, 430 cycles of unpacking a stage where the products of fewer
// than 215 tokens take less, and a block's start and end, when its products rest.
//
// Every wait ends: one that takes too long marks the block as failed, which then waits
// for its own copies, frees its tensor memory and writes NaN.
#include <algorithm>

#include "ops_tensor.cuh"
#include "quant_matmul.cuh"

namespace e2ops {
namespace {

constexpr int kTileRows = 128, kStageCols = 64, kTeams = 4, kUnpackWarps = 4 * kTeams, kThreads = 32 * (2 + kUnpackWarps);
constexpr int kMostSplit = 8;
constexpr int kChunkColumns = kTeams * kStageCols;           // codes are copied in chunks of a stage for each team
constexpr int kRaw = 3;                                      // chunks of codes in shared memory
// Tensor memory, all of it: sums first, then the stages of unpacked weights, 32 columns each.
constexpr int kColumns = 512, kWeightColumns = 256, kWeightStages = 8;

struct ManyParams {
    MatmulParams m;
    int outs, tile, row_tiles, split, stages, depth;         // tokens of a tile; stages in flight
    int first;                                               // of the blocks (row tiles in turn, then tokens'), this launch's
    int scales_by;                                           // scales copied by a chunk's row, by 4 bytes, or one by one (2)
    uint8_t *prepared;                                 // [tiles][cols / 64][tile][128 bytes], then scales per token
    float *unscale;
};

// Whether eight codes times d plus m stay within fp16's range, for two d and m (NaN: no).
template <bool MINS> __device__ __forceinline__ bool in_range(__half2 d, __half2 m)
{
    // (rounded as the weights are: what rounds to 65,504 here does there)
    const __half2 most = MINS ? __hfma2(__habs2(d), __float2half2_rn(15.0f), __habs2(m)) : __hmul2(__habs2(d), __float2half2_rn(8.0f));
    return __hble2(most, __float2half2_rn(65504.0f));
}

// Weights that became infinite are fp16's largest, unless d or m is not finite itself.
__device__ __forceinline__ void limit_weights(uint32_t *w, __half d, __half m)
{
    const __half largest(65504.0f);
    const __half2 most = __float2half2_rn(__hle(__habs(d), largest) && __hle(__habs(m), largest) ? 65504.0f : INFINITY);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const __half2 y = __hmin2_nan(__hmax2_nan(*reinterpret_cast<const __half2 *>(&w[i]), __hneg2(most)), most);
        w[i] = *reinterpret_cast<const uint32_t *>(&y);
    }
}

// A word's eight codes, less 8 where there are no minima, times d plus m.
template <bool MINS> __device__ __forceinline__ void scale_word(uint32_t *out, uint32_t w, __half2 d, __half2 m)
{
    const uint32_t v = w >> 8;
    const uint32_t q[4] = {(w & 0x000f000fu) | 0x64006400u, (w & 0x00f000f0u) | 0x64006400u, (v & 0x000f000fu) | 0x64006400u,
                           (v & 0x00f000f0u) | 0x64006400u};
    const __half2 low = __float2half2_rn(MINS ? -1024.0f : -1032.0f), sixteenth = __float2half2_rn(0.0625f);
    const __half2 high = __float2half2_rn(MINS ? -64.0f : -72.0f);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __half2 x = *reinterpret_cast<const __half2 *>(&q[i]);
        const __half2 c = i % 2 ? __hfma2(x, sixteenth, high) : __hadd2(x, low);
        const __half2 y = MINS ? __hfma2(c, d, m) : __hmul2(c, d);
        out[i] = *reinterpret_cast<const uint32_t *>(&y);
    }
}

// x as the images of its stages: a block per token.
template <class T> __global__ void __launch_bounds__(512) image_kernel(const ManyParams q)
{
    __shared__ unsigned largest;
    uint8_t *to = q.prepared;
    float *unscale = q.unscale;
    allow_next();
    const MatmulParams &p = q.m;
    const int tok = blockIdx.x, octets = q.stages * 8, row = tok % q.tile;
    if (threadIdx.x == 0) largest = 0;
    __syncthreads();
    const uint4 *x = reinterpret_cast<const uint4 *>(static_cast<const T *>(p.x) + tok * p.x_stride);
    unsigned m = 0;
    for (int o = threadIdx.x; o < p.cols / 8; o += blockDim.x) m = max(m, octet_largest(x[o]));
    m = __reduce_max_sync(~0u, m);
    if (threadIdx.x % 32 == 0) atomicMax(&largest, m);
    __syncthreads();
    const int k = power_for<T>(largest);
    const float f = power_of_two(k);
    uint8_t *tile = to + (size_t)(tok / q.tile) * q.stages * q.tile * 128;
    for (int o = threadIdx.x; o < octets; o += blockDim.x) {
        uint4 v{0, 0, 0, 0};
        if (o < p.cols / 8) v = octet_in_order<T>(x[o], f);
        *reinterpret_cast<uint4 *>(tile + ((size_t)(o / 8) * q.tile + row) * 128 + ((o % 8) ^ (row & 7)) * 16) = v;
    }
    if (threadIdx.x == 0) unscale[tok] = power_of_two(-k);
}

// A chunk of codes and scales as they lie in shared memory (rows 16 bytes apart in banks).
template <int G, bool MINS> struct Chunk {
    static constexpr int kPer = kChunkColumns / G, kRowBytes = kChunkColumns / 2 + 16, kCodes = kTileRows * kRowBytes;
    static constexpr int kBytes = kCodes + kTileRows * kPer * 2 * (MINS ? 2 : 1);
};

template <int G, bool MINS> __global__ void __launch_bounds__(kThreads, 1) many_kernel(const ManyParams q)
{
    extern __shared__ uint8_t dynamic[];
    uint8_t *smem = dynamic + (1024 - smem_addr(dynamic) % 1024) % 1024;     // (swizzled tiles start on 1024 bytes)
    __shared__ __align__(8) uint64_t barriers[2 * kWeightStages + 1];
    __shared__ uint32_t tensor_memory;
    __shared__ int failed;
    const MatmulParams &p = q.m;
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const int rank = blockIdx.x % q.split, block = (q.first + blockIdx.x / q.split) % q.row_tiles;
    const int tile = (q.first + blockIdx.x / q.split) / q.row_tiles;
    allow_next();
    const int rows_out = p.gated ? kTileRows / 2 : kTileRows;
    const uint32_t stage_bytes = (uint32_t)q.tile * 128;
    // this block's stages, whole chunks
    const int all_chunks = (q.stages + kTeams - 1) / kTeams;
    const int s0 = (int)((int64_t)all_chunks * rank / q.split) * kTeams;
    const int n = min((int)((int64_t)all_chunks * (rank + 1) / q.split) * kTeams, q.stages) - s0;
    // a stage is full when x and the unpacked weights are there, empty when its products are done
    const uint32_t ring = smem_addr(smem), full = smem_addr(barriers), empty = full + 8 * kWeightStages, done = empty + 8 * kWeightStages;
    if (threadIdx.x == 0) {
        for (int i = 0; i < q.depth; ++i) barrier_init(full + 8 * i, 1 + 4), barrier_init(empty + 8 * i, 1);
        barrier_init(done, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        failed = 0;
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&tensor_memory)), "r"(kColumns)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t d = *reinterpret_cast<volatile uint32_t *>(&tensor_memory), weights = d + kWeightColumns;

    if (warp == 0) {
        // x: a stage's image by one copy
        wait_before();
        const uint8_t *from = q.prepared + ((size_t)tile * q.stages + s0) * stage_bytes;
        int i = 0, slot = 0, phase = 1;
        for (; i < n; ++i) {
            if (!__all_sync(~0u, barrier_wait(empty + 8 * slot, phase))) break;
            if (elected()) {
                barrier_expect(full + 8 * slot, stage_bytes);
                asm volatile(
                    "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(ring + slot * stage_bytes),
                    "l"(from + (size_t)i * stage_bytes), "r"(stage_bytes), "r"(full + 8 * slot)
                    : "memory");
            }
            __syncwarp();
            if (++slot == q.depth) slot = 0, phase ^= 1;
        }
        if (i < n) {
            // the copies in flight have no waiter of their own: their stages are given up on after a while
            failed = 1;
            for (int j = i > q.depth ? i - q.depth : 0; j < i; ++j) barrier_wait(full + 8 * (j % q.depth), j / q.depth & 1);
        }
    } else if (warp == 1) {
        // products: the whole warp waits, one thread issues
        const uint32_t kind = product_kind(q.tile);
        bool ok = true, ready = false;
        int slot = 0, phase = 0;
        for (int i = 0; i < n; ++i) {
            if (!ready) ok = __all_sync(~0u, barrier_wait(full + 8 * slot, phase));
            if (!ok) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const int next = slot + 1 == q.depth ? 0 : slot + 1, next_phase = slot + 1 == q.depth ? phase ^ 1 : phase;
            ready = barrier_poll(full + 8 * next, next_phase);     // (its answer is there when these are issued)
            if (elected()) {
                const uint64_t b = operand(ring + slot * stage_bytes);
#pragma unroll
                for (int k = 0; k < kStageCols / 16; ++k)
                    issue_product(d, weights + slot * 32 + 8 * k, b + 2 * k, kind, i > 0 || k > 0);
                commit_products(empty + 8 * slot);
            }
            ready = __all_sync(~0u, ready);
            slot = next, phase = next_phase;
        }
        if (!ok) failed = 1;
        if (elected()) commit_products(done);
        __syncwarp();
        if (!__all_sync(~0u, barrier_wait(done, 0))) failed = 1;
    } else {
        // weights, in chunks: 128 rows of 256 columns, four stages.  The four warps of a quarter
        // of the rows copy it together, whole runs of a row; then each, of another team,
        // unpacks one stage, a thread a row.
        const int team = (warp - 2) / 4, quarter = warp % 4;
        using Ch = Chunk<G, MINS>;
        const int groups = p.cols / G, chunks = (n + kTeams - 1) / kTeams;
        uint8_t *raw = smem + q.depth * stage_bytes;
        // (past the last row the last one is read again, and its results are dropped)
        auto source = [&](int r) {
            const int half = p.gated && r >= kTileRows / 2;
            return (int64_t)min(block * rows_out + r - half * (kTileRows / 2), q.outs - 1) + (int64_t)half * q.outs;
        };
        constexpr int kPieces = kChunkColumns / 32, kRowsAtOnce = 32 / kPieces, kCopies = 8 / kRowsAtOnce;       // 16 bytes of codes
        const int part = lane % kPieces;
        const uint8_t *code_from[kCopies];
        uint32_t code_to[kCopies];
#pragma unroll
        for (int i = 0; i < kCopies; ++i) {
            const int r = 32 * quarter + team * 8 + i * kRowsAtOnce + lane / kPieces;
            code_from[i] = p.codes + source(r) * (p.cols / 2);
            code_to[i] = smem_addr(raw) + r * Ch::kRowBytes + part * 16;
        }
        // the rows' scales by the first team, minima by the second
        const int r = 32 * quarter + lane;
        const __half *scale_from = (MINS && team == 1 ? p.mins : p.scales) + source(r) * groups;
        const uint32_t scale_to = smem_addr(raw) + Ch::kCodes + (team * kTileRows + r) * (Ch::kPer * 2);
        auto copy = [&](int c, int place) {
            if (c < chunks) {
                const int col0 = (s0 + c * kTeams) * kStageCols, g0 = col0 / G;
                // (past the last column any codes will do: x is 0 there)
                const int at = col0 + part * 32 < p.cols ? col0 / 2 + part * 16 : 0;
#pragma unroll
                for (int i = 0; i < kCopies; ++i) copy_async16(code_to[i] + place * Ch::kBytes, code_from[i] + at, true);
                if (team < (MINS ? 2 : 1)) {
                    const uint32_t dst = scale_to + place * Ch::kBytes;
                    if (q.scales_by > 4) {
                        asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(dst), "l"(scale_from + g0), "n"(Ch::kPer * 2) : "memory");
                    } else {
#pragma unroll
                        for (int j = 0; j < Ch::kPer; j += 2) {
                            if (q.scales_by == 4) {
                                copy_async4(dst + 2 * j, g0 + j < groups ? scale_from + g0 + j : scale_from, g0 + j < groups);
                            } else {
                                const uint32_t lo = g0 + j < groups ? __half_as_ushort(scale_from[g0 + j]) : 0u;
                                const uint32_t hi = g0 + j + 1 < groups ? __half_as_ushort(scale_from[g0 + j + 1]) : 0u;
                                asm volatile("st.shared.u32 [%0], %1;" ::"r"(dst + 2 * j), "r"(lo | hi << 16) : "memory");
                            }
                        }
                    }
                }
            }
            copy_commit();
        };
        copy(0, 0);
        copy(1, 1);
        bool ok = true;
        int place = 0, slot = team, phase = 1;
        while (slot >= q.depth) slot -= q.depth, phase ^= 1;
        for (int c = 0; c < chunks; ++c) {
            copy_wait<1>();
            // the chunk is there, and the one before is done with, for the quarter's four warps
            asm volatile("bar.sync %0, 128;" ::"r"(1 + quarter) : "memory");
            copy(c + 2, place == 0 ? 2 : place - 1);
            const int i = c * kTeams + team, here = slot, round = phase;
            const uint8_t *chunk = raw + place * Ch::kBytes;
            place = place == 2 ? 0 : place + 1;
            slot += kTeams;
            while (slot >= q.depth) slot -= q.depth, phase ^= 1;
            ok = ok && !*reinterpret_cast<volatile int *>(&failed);
            ok = __all_sync(~0u, ok);
            if (i >= n || !ok) continue;
            const uint4 *w = reinterpret_cast<const uint4 *>(chunk + r * Ch::kRowBytes + team * 32);
            const uint4 w0 = w[0], w1 = w[1];
            const __half *sc = reinterpret_cast<const __half *>(chunk + Ch::kCodes + r * (Ch::kPer * 2));
            const __half *mn = sc + kTileRows * Ch::kPer;
            const int g0 = team * kStageCols / G, g1 = (team * kStageCols + 32) / G;
            const __half d0 = sc[g0], d1 = sc[g1], m0 = MINS ? mn[g0] : __half(0.0f), m1 = MINS ? mn[g1] : __half(0.0f);
            uint32_t v[32];
            {
                const __half2 ds = __half2half2(d0), ms = __half2half2(m0);
                scale_word<MINS>(&v[0], w0.x, ds, ms);
                scale_word<MINS>(&v[4], w0.y, ds, ms);
                scale_word<MINS>(&v[8], w0.z, ds, ms);
                scale_word<MINS>(&v[12], w0.w, ds, ms);
            }
            {
                const __half2 ds = __half2half2(d1), ms = __half2half2(m1);
                scale_word<MINS>(&v[16], w1.x, ds, ms);
                scale_word<MINS>(&v[20], w1.y, ds, ms);
                scale_word<MINS>(&v[24], w1.z, ds, ms);
                scale_word<MINS>(&v[28], w1.w, ds, ms);
            }
            if (!__all_sync(~0u, in_range<MINS>(__halves2half2(d0, d1), __halves2half2(m0, m1)))) {
                limit_weights(&v[0], d0, m0);
                limit_weights(&v[16], d1, m1);
            }
            ok = __all_sync(~0u, barrier_wait(empty + 8 * here, round));
            if (ok) {
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                store_columns(weights + ((uint32_t)(32 * quarter) << 16) + here * 32, v);
                asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                __syncwarp();
                if (lane == 0) barrier_arrive(full + 8 * here);
            } else if (lane == 0) {
                failed = 1;
            }
        }
        copy_wait<0>();
    }
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    wait_before();                  // (unscale comes from the kernel before, too)
    const bool bad = *reinterpret_cast<volatile int *>(&failed);

    // outputs: lanes are rows, columns tokens; the unpacking warps take them, four to 32 lanes.
    // A cluster's sums, and rows that are gated, go through shared memory: [tile][rows].
    const int token0 = tile * q.tile, live = min(q.tile, p.tokens - token0);
    const float nan = __int_as_float(0x7fc00000);
    float *sums = reinterpret_cast<float *>(smem);
    const int quarter = warp % 4, row = 32 * quarter + lane;
    auto columns = [&](auto take) {
        for (int c = (warp - 2) / 4 * 16; c < live; c += 16 * kTeams) {
            uint32_t v[16];
            load_columns(v, d + ((uint32_t)(32 * quarter) << 16) + c);
            loaded(v);
#pragma unroll
            for (int e = 0; e < 16; ++e) take(c + e, bad ? nan : __uint_as_float(v[e]));
        }
    };
    if (q.split > 1) {
        if (warp >= 2) columns([&](int c, float v) { sums[c * kTileRows + row] = v; });
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        __syncthreads();
        cluster_barrier();
        // each block of the cluster joins its share of the tokens, four rows a thread
        const uint32_t mine = smem_addr(smem);
        for (int at = rank * kThreads + threadIdx.x; at < live * (rows_out / 4); at += q.split * kThreads) {
            const int c = at / (rows_out / 4), r = at % (rows_out / 4) * 4, out = block * rows_out + r;
            auto joined = [&](int from) {
                float4 v[kMostSplit], sum{0, 0, 0, 0};
#pragma unroll
                for (int k = 0; k < kMostSplit; ++k)
                    if (k < q.split) v[k] = peer_load4(peer_addr(mine + (c * kTileRows + from) * 4, k));
#pragma unroll
                for (int k = 0; k < kMostSplit; ++k)
                    if (k < q.split) sum.x += v[k].x, sum.y += v[k].y, sum.z += v[k].z, sum.w += v[k].w;
                return sum;
            };
            const float4 g = joined(r), h = p.gated ? joined(r + kTileRows / 2) : g;
            const float f = q.unscale[token0 + c];
            if (out < q.outs) finish(p, token0 + c, out, g.x * f, h.x * f);
            if (out + 1 < q.outs) finish(p, token0 + c, out + 1, g.y * f, h.y * f);
            if (out + 2 < q.outs) finish(p, token0 + c, out + 2, g.z * f, h.z * f);
            if (out + 3 < q.outs) finish(p, token0 + c, out + 3, g.w * f, h.w * f);
        }
        cluster_barrier();                                               // (peers may still read)
    } else {
        if (p.gated && warp >= 2 && quarter >= 2) columns([&](int c, float v) { sums[c * (kTileRows / 2) + row - kTileRows / 2] = v; });
        if (p.gated) __syncthreads();
        const int out = block * rows_out + row;
        if (warp >= 2 && row < rows_out)
            columns([&](int c, float v) {
                if (c >= live || out >= q.outs) return;
                const float f = q.unscale[token0 + c];
                finish(p, token0 + c, out, v * f, p.gated ? sums[c * (kTileRows / 2) + row] * f : 0.0f);
            });
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    }
    __syncthreads();
    __syncwarp();
    if (warp == 1)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(d), "r"(kColumns) : "memory");
}

template <int G, bool MINS> int launch_many_as(const ManyParams &q, const ManyPlan &f, int dev, cudaStream_t s)
{
    static std::atomic<uint64_t> ready{0};                               // devices that have the attribute set
    auto kernel = many_kernel<G, MINS>;
    if (!(ready.load(std::memory_order_relaxed) >> dev & 1)) {
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemPerSm - 4096);
        if (e != cudaSuccess) return cuda_status(e);
        ready.fetch_or(1ull << dev, std::memory_order_relaxed);
    }
    if (int st = launch<ManyParams>(q.m.half ? image_kernel<__half> : image_kernel<__nv_bfloat16>,
                                    dim3((unsigned)q.m.tokens), 512, 0, 1, false, s, q))
        return st;
    // (never two blocks on a multiprocessor: tensor memory is for one)
    const size_t ring = (size_t)q.depth * q.tile * 128 + kRaw * Chunk<G, MINS>::kBytes + 1024;
    const size_t sums = q.split > 1 || f.rest_split > 1 ? (size_t)q.tile * kTileRows * 4 + 1024 : q.m.gated ? (size_t)q.tile * kTileRows * 2 + 1024 : 0;
    const size_t smem = std::max(std::max(ring, sums), (size_t)kSmemPerSm / 2);
    const int blocks = q.row_tiles * f.tiles;
    if (!f.whole) return launch<ManyParams>(kernel, dim3((unsigned)(blocks * f.split)), kThreads, smem, f.split, true, s, q);
    if (int st = launch<ManyParams>(kernel, dim3((unsigned)f.whole), kThreads, smem, 1, true, s, q)) return st;
    ManyParams rest = q;
    rest.first = f.whole;
    rest.split = f.rest_split;
    return launch<ManyParams>(kernel, dim3((unsigned)((blocks - f.whole) * f.rest_split)), kThreads, smem, f.rest_split, true, s, rest);
}

template <int G> int launch_many_group(const ManyParams &q, const ManyPlan &f, int dev, cudaStream_t s)
{
    return q.m.mins ? launch_many_as<G, true>(q, f, dev, s) : launch_many_as<G, false>(q, f, dev, s);
}

}  // namespace

// The tile of tokens (a multiple of 16, up to 256) and the split over columns that
// take the fewest turns of the multiprocessors times a turn's length: two cycles a token and
// stage, no fewer than unpacking takes, and a fixed part.  A last turn that would leave many
// multiprocessors idle is split over columns instead, by a second launch.  Measured, us (all
// alike / so): 8192 x 28672, 1,152 tokens 415 / 404 (one call after another 486 / 456), 28672 x 8192
// 431 / 415; 5000 x 8192, 1,000 tokens 94 / 74; 20000 x 4096, 250 tokens 63 / 47.
ManyPlan plan_many(int outs, bool gated, int cols, int tokens, int sms)
{
    ManyPlan best{};
    double least = 1e300;
    const int rows_out = gated ? kTileRows / 2 : kTileRows, row_tiles = (outs + rows_out - 1) / rows_out, stages = (cols + kStageCols - 1) / kStageCols;
    auto turn = [&](int tile, int split) {
        const double stage = 2.0 * tile > 430.0 ? 2.0 * tile : 430.0;
        return stage * ((stages + split - 1) / split) + 4000.0 + 12.0 * tile + (split > 1 ? 3000.0 + 16.0 * tile : 0.0);
    };
    auto consider = [&](double t, int tile, int tiles, int split, int whole, int rest) {
        if (t >= least) return;
        least = t;
        const int fit = 140 * 1024 / (tile * 128);
        best = ManyPlan{tile, tiles, row_tiles, split, stages, fit < kWeightStages ? fit : kWeightStages, whole, rest,
                        (size_t)tiles * stages * tile * 128, 0};
        best.workspace = best.image + (size_t)tokens * 4;
    };
    for (int tile = 32; tile <= 256; tile += 16) {
        const int tiles = (tokens + tile - 1) / tile;
        if (tile > 32 && (tokens + tiles - 1) / tiles <= tile - 16) continue;                  // (a smaller one does as well)
        for (int split = 1; split <= kMostSplit; split *= 2) {
            if (split > 1 && stages / split < 8) continue;
            const double t = (double)(((int64_t)row_tiles * tiles * split + sms - 1) / sms) * turn(tile, split);
            consider(t, tile, tiles, split, 0, 1);
        }
        // whole turns unsplit, then what is left split over all multiprocessors
        const int64_t blocks = (int64_t)row_tiles * tiles, whole = blocks / sms * sms;
        int rest = 1;
        while (rest < kMostSplit && (blocks - whole) * rest * 2 <= sms && stages / (rest * 2) >= 8) rest *= 2;
        if (whole > 0 && rest > 1 && blocks > whole)
            consider((double)(whole / sms) * turn(tile, 1) + turn(tile, rest) + 3000.0, tile, tiles, 1, (int)whole, rest);
    }
    return best;
}

int launch_many(const MatmulParams &m, const ManyPlan &f, void *workspace, int outs, int dev, cudaStream_t s)
{
    ManyParams q{m, outs, f.tile, f.row_tiles, f.split, f.stages, f.depth, 0, 0, static_cast<uint8_t *>(workspace),
                 reinterpret_cast<float *>(static_cast<uint8_t *>(workspace) + f.image)};
    // how a chunk's rows of scales are aligned
    const int wide = kChunkColumns / m.group * 2, groups = m.cols / m.group;
    auto all_aligned = [&](int to) { return groups * 2 % to == 0 && aligned(m.scales, to) && aligned(m.mins, to); };
    q.scales_by = m.cols % kChunkColumns == 0 && all_aligned(wide) ? 16 : all_aligned(4) ? 4 : 2;
    return m.group == 32   ? launch_many_group<32>(q, f, dev, s)
           : m.group == 64 ? launch_many_group<64>(q, f, dev, s)
                           : launch_many_group<128>(q, f, dev, s);
}

}  // namespace e2ops
