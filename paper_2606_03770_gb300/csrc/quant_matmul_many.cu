// quant_matmul_many.cu -- e2_quant_matmul for prompts.
//
// Bound by the fifth-generation tensor cores.  A block takes 128 weight rows (gated: 128
// that gate and the 128 that they gate) and up to 256 tokens (128): D[rows][tokens] = W
// x^T, W and D in tensor memory, x in shared memory.  One warp copies x, prepared beforehand
// as the images of its stages (one bulk copy each), one issues the products, eight
// unpack weights, four every other stage: a thread a row's 64 columns, from registers that
// are loaded stages ahead, to fp16 with their scale, one rounding (2^-11 of a weight;
// |W| up to 65504).  (Unpacked into shared memory instead, a stage took 520 ns whatever its
// tokens: the fence that the products need after such writes waits for the loads ahead as
// well.)  Elements stay in the order that unpacking leaves (0, 4, 1, 5, 2, 6, 3, 7 of each
// eight), x is put into the same one.  Few rows are split over columns by the blocks of a
// cluster, whose sums are joined in a fixed order through shared memory.
//
// Every wait ends: one that takes too long marks the block as failed, which then waits
// for its own copies, frees its tensor memory and writes NaN.
#include <algorithm>

#include "quant_matmul.cuh"

namespace e2ops {
namespace {

constexpr int kTileRows = 128, kStageCols = 64, kUnpackWarps = 8, kThreads = 32 * (2 + kUnpackWarps);
constexpr int kAhead = 3;                                    // a warp's stages of codes in registers
// Tensor memory, all of it: sums first, then the stages of unpacked weights, 32 columns each.
constexpr int kColumns = 512, kWeightColumns = 256, kWeightStages = 8;
constexpr int kMostX = 8;                                    // stages of x

struct ManyParams {
    MatmulParams m;
    int outs, tile, tiles, split, stages, depth;             // tokens of a tile; stages of x in shared memory
    const uint8_t *prepared;                                 // [tiles][cols / 64][tile][128 bytes], then scales per token
    const float *unscale;
};

__device__ __forceinline__ void barrier_init(uint32_t at, int count)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(at), "r"(count) : "memory");
}
__device__ __forceinline__ void barrier_arrive(uint32_t at)
{
    asm volatile("{\n.reg .b64 state;\nmbarrier.arrive.shared::cta.b64 state, [%0];\n}" ::"r"(at) : "memory");
}
__device__ __forceinline__ void barrier_expect(uint32_t at, uint32_t bytes)
{
    asm volatile("{\n.reg .b64 state;\nmbarrier.arrive.expect_tx.shared::cta.b64 state, [%0], %1;\n}" ::"r"(at), "r"(bytes) : "memory");
}
// Whether the phase ended, within a second or so (a million polls of up to a microsecond).
__device__ bool barrier_wait(uint32_t at, uint32_t parity)
{
    for (int i = 0; i < (1 << 20); ++i) {
        uint32_t done;
        asm volatile(
            "{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\nselp.u32 %0, 1, 0, p;\n}"
            : "=r"(done)
            : "r"(at), "r"(parity), "r"(1000u)
            : "memory");
        if (done) return true;
    }
    return false;
}

// A tile of 128-byte rows, swizzled by 128 bytes, columns contiguous: groups of eight rows
// 1024 bytes apart.
__device__ __forceinline__ uint64_t operand(uint32_t at)
{
    return (uint64_t)((at & 0x3ffff) >> 4) | (uint64_t)1 << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
__device__ __forceinline__ void issue_product(uint32_t d, uint32_t a, uint64_t b, uint32_t kind, bool add)
{
    asm volatile(
        "{\n.reg .pred p;\nsetp.ne.u32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}" ::"r"(d), "r"(a), "l"(b),
        "r"(kind), "r"((uint32_t)add)
        : "memory");
}
__device__ __forceinline__ void commit_products(uint32_t barrier)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(barrier) : "memory");
}
// 16 columns of this warp's 32 lanes.
__device__ __forceinline__ void load_columns(uint32_t (&v)[16], uint32_t at)
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]),
          "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
        : "r"(at)
        : "memory");
}

// 32 columns of this warp's 32 lanes.
__device__ __forceinline__ void store_columns(uint32_t at, const uint32_t (&v)[32])
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,"
        "%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};" ::"r"(at),
        "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]),
        "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(v[16]), "r"(v[17]), "r"(v[18]), "r"(v[19]), "r"(v[20]),
        "r"(v[21]), "r"(v[22]), "r"(v[23]), "r"(v[24]), "r"(v[25]), "r"(v[26]), "r"(v[27]), "r"(v[28]), "r"(v[29]), "r"(v[30]),
        "r"(v[31])
        : "memory");
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
template <class T> __global__ void __launch_bounds__(512) image_kernel(const ManyParams q, uint8_t *to, float *unscale)
{
    __shared__ unsigned largest;
    asm volatile("griddepcontrol.launch_dependents;");
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

template <int G, bool MINS, int MT> __global__ void __launch_bounds__(kThreads, 1) many_kernel(const ManyParams q)
{
    extern __shared__ uint8_t dynamic[];
    uint8_t *smem = dynamic + (1024 - smem_addr(dynamic) % 1024) % 1024;     // (swizzled tiles start on 1024 bytes)
    __shared__ __align__(8) uint64_t barriers[2 * kMostX + 2 * kWeightStages + 1];
    __shared__ uint32_t tensor_memory;
    __shared__ int failed;
    constexpr int kStep = kWeightColumns / MT, kDepthW = kWeightStages / MT;     // sums of a row tile; stages of weights
    const MatmulParams &p = q.m;
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const int rank = blockIdx.x % q.split, block = blockIdx.x / q.split;
    const uint32_t stage_bytes = (uint32_t)q.tile * 128;
    const int s0 = (int)((int64_t)q.stages * rank / q.split), s1 = (int)((int64_t)q.stages * (rank + 1) / q.split), n = s1 - s0;
    const uint32_t ring = smem_addr(smem), full_x = smem_addr(barriers), empty_x = full_x + 8 * kMostX;
    const uint32_t full_w = empty_x + 8 * kMostX, empty_w = full_w + 8 * kWeightStages, done = empty_w + 8 * kWeightStages;
    if (threadIdx.x == 0) {
        for (int i = 0; i < q.depth; ++i) barrier_init(full_x + 8 * i, 1), barrier_init(empty_x + 8 * i, 1);
        for (int i = 0; i < kDepthW; ++i) barrier_init(full_w + 8 * i, kUnpackWarps / 2), barrier_init(empty_w + 8 * i, 1);
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
        if (lane == 0) {
            asm volatile("griddepcontrol.wait;" ::: "memory");
            const uint8_t *from = q.prepared + ((size_t)blockIdx.y * q.stages + s0) * stage_bytes;
            int i = 0, slot = 0, phase = 1;
            for (; i < n; ++i) {
                if (!barrier_wait(empty_x + 8 * slot, phase)) break;
                barrier_expect(full_x + 8 * slot, stage_bytes);
                asm volatile(
                    "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(ring + slot * stage_bytes),
                    "l"(from + (size_t)i * stage_bytes), "r"(stage_bytes), "r"(full_x + 8 * slot)
                    : "memory");
                if (++slot == q.depth) slot = 0, phase ^= 1;
            }
            if (i < n) {
                failed = 1;
                for (int j = i > q.depth ? i - q.depth : 0; j < i; ++j) barrier_wait(full_x + 8 * (j % q.depth), j / q.depth & 1);
            }
        }
    } else if (warp == 1) {
        if (lane == 0) {
            const uint32_t kind = 1u << 4 | (uint32_t)(q.tile >> 3) << 17 | (uint32_t)(kTileRows >> 4) << 24;
            bool ok = true;
            int slot = 0, phase = 0;
            for (int i = 0; i < n; ++i) {
                const int w = i % kDepthW;
                ok = barrier_wait(full_x + 8 * slot, phase) && barrier_wait(full_w + 8 * w, i / kDepthW & 1);
                if (!ok) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const uint64_t b = operand(ring + slot * stage_bytes);
#pragma unroll
                for (int t = 0; t < MT; ++t)
#pragma unroll
                    for (int k = 0; k < kStageCols / 16; ++k)
                        issue_product(d + t * kStep, weights + (w * MT + t) * 32 + 8 * k, b + 2 * k, kind, i > 0 || k > 0);
                commit_products(empty_x + 8 * slot);
                commit_products(empty_w + 8 * w);
                if (++slot == q.depth) slot = 0, phase ^= 1;
            }
            if (!ok) failed = 1;
            commit_products(done);
            if (!barrier_wait(done, 0)) failed = 1;
        }
    } else {
        // weights: a thread a row; warps 2-5 even stages, 6-9 odd ones
        const int team = (warp - 2) / 4, quarter = warp % 4, r = 32 * quarter + lane;
        const int groups = p.cols / G;
        constexpr int kScales = G == 32 ? 2 : 1;
        const uint8_t *codes[MT];
        const __half *scales[MT], *mins[MT];
#pragma unroll
        for (int t = 0; t < MT; ++t) {
            // (past the last row the last one is read again, and its results are dropped)
            const int64_t row = min(block * kTileRows + r, q.outs - 1) + (int64_t)t * q.outs;
            codes[t] = p.codes + row * (p.cols / 2);
            scales[t] = p.scales + row * groups;
            mins[t] = MINS ? p.mins + row * groups : nullptr;
        }
        uint4 w[kAhead][MT][2];
        __half sc[kAhead][MT][kScales], mn[kAhead][MT][kScales];
        auto fetch = [&](int i, int at) {
            const int col = (s0 + i) * kStageCols;
            // (a last stage may have 32 columns; what is past them is 0, as x is)
            const bool in = i < n, whole = in && col + 32 < p.cols;
#pragma unroll
            for (int t = 0; t < MT; ++t) {
                w[at][t][0] = in ? *reinterpret_cast<const uint4 *>(codes[t] + col / 2) : uint4{0, 0, 0, 0};
                w[at][t][1] = whole ? *reinterpret_cast<const uint4 *>(codes[t] + col / 2 + 16) : uint4{0, 0, 0, 0};
#pragma unroll
                for (int j = 0; j < kScales; ++j) {
                    const bool there = j ? whole : in;
                    sc[at][t][j] = there ? scales[t][col / G + j] : __half(0.0f);
                    mn[at][t][j] = MINS && there ? mins[t][col / G + j] : __half(0.0f);
                }
            }
        };
#pragma unroll
        for (int a = 0; a < kAhead; ++a) fetch(team + 2 * a, a);
        bool ok = true;
        for (int i0 = team; i0 < n && ok; i0 += 2 * kAhead) {
#pragma unroll
            for (int a = 0; a < kAhead; ++a) {
                const int i = i0 + 2 * a, slot = i % kDepthW;
                if (i >= n || !ok) break;
                uint32_t v[MT][32];
#pragma unroll
                for (int t = 0; t < MT; ++t)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const __half2 ds = __half2half2(sc[a][t][kScales == 2 ? h : 0]), ms = __half2half2(mn[a][t][kScales == 2 ? h : 0]);
                        scale_word<MINS>(&v[t][16 * h], w[a][t][h].x, ds, ms);
                        scale_word<MINS>(&v[t][16 * h + 4], w[a][t][h].y, ds, ms);
                        scale_word<MINS>(&v[t][16 * h + 8], w[a][t][h].z, ds, ms);
                        scale_word<MINS>(&v[t][16 * h + 12], w[a][t][h].w, ds, ms);
                    }
                fetch(i + 2 * kAhead, a);
                ok = __all_sync(~0u, barrier_wait(empty_w + 8 * slot, (i / kDepthW & 1) ^ 1));
                if (ok) {
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll
                    for (int t = 0; t < MT; ++t)
                        store_columns(weights + ((uint32_t)(32 * quarter) << 16) + (slot * MT + t) * 32, v[t]);
                    asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
                    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) barrier_arrive(full_w + 8 * slot);
                } else if (lane == 0) {
                    failed = 1;
                }
            }
        }
    }
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");                  // (unscale comes from the kernel before, too)
    const bool bad = *reinterpret_cast<volatile int *>(&failed);

    // outputs: lanes are rows, columns tokens; the unpacking warps take them, two to 32 lanes
    const int token0 = blockIdx.y * q.tile, live = min(q.tile, p.tokens - token0);
    const float nan = __int_as_float(0x7fc00000);
    if (warp >= 2) {
        const int quarter = warp % 4, row = 32 * quarter + lane, out = block * kTileRows + row;
        for (int c = (warp - 2) / 4 * 16; c < live; c += 32) {
            uint32_t v[MT][16];
#pragma unroll
            for (int t = 0; t < MT; ++t) load_columns(v[t], d + ((uint32_t)(32 * quarter) << 16) + t * kStep + c);
            asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
            if (q.split > 1) {
                float *sums = reinterpret_cast<float *>(smem);           // [MT][tile][128]
#pragma unroll
                for (int t = 0; t < MT; ++t)
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        if (c + e < q.tile) sums[(t * q.tile + c + e) * kTileRows + row] = bad ? nan : __uint_as_float(v[t][e]);
            } else if (out < q.outs) {
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    if (c + e >= live) break;
                    const float f = bad ? nan : q.unscale[token0 + c + e];
                    finish(p, token0 + c + e, out, __uint_as_float(v[0][e]) * f, __uint_as_float(v[MT - 1][e]) * f);
                }
            }
        }
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    }
    if (q.split > 1) {
        __syncthreads();
        cluster_barrier();
        // each block of the cluster joins its share of the tokens
        const uint32_t mine = smem_addr(smem);
        for (int at = rank * kThreads + threadIdx.x; at < live * kTileRows; at += q.split * kThreads) {
            const int c = at / kTileRows, row = at % kTileRows, out = block * kTileRows + row;
            if (out >= q.outs) continue;
            float v[MT] = {};
            for (int k = 0; k < q.split; ++k)
#pragma unroll
                for (int t = 0; t < MT; ++t) v[t] += peer_load(peer_addr(mine + ((t * q.tile + c) * kTileRows + row) * 4, k));
            const float f = q.unscale[token0 + c];
            finish(p, token0 + c, out, v[0] * f, v[MT - 1] * f);
        }
        cluster_barrier();                                               // (peers may still read)
    }
    __syncthreads();
    __syncwarp();
    if (warp == 1)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(d), "r"(kColumns) : "memory");
}

template <int G, bool MINS, int MT> int launch_many_as(const ManyParams &q, const ManyPlan &f, int dev, cudaStream_t s)
{
    static std::atomic<uint64_t> ready{0};                               // devices that have the attribute set
    auto kernel = many_kernel<G, MINS, MT>;
    if (!(ready.load(std::memory_order_relaxed) >> dev & 1)) {
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemPerSm - 4096);
        if (e != cudaSuccess) return cuda_status(e);
        ready.fetch_or(1ull << dev, std::memory_order_relaxed);
    }
    uint8_t *to = const_cast<uint8_t *>(q.prepared);
    float *unscale = const_cast<float *>(q.unscale);
    if (q.m.half) image_kernel<__half><<<(unsigned)q.m.tokens, 512, 0, s>>>(q, to, unscale);
    else image_kernel<__nv_bfloat16><<<(unsigned)q.m.tokens, 512, 0, s>>>(q, to, unscale);
    cudaLaunchAttribute at[2]{};
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)((q.outs + kTileRows - 1) / kTileRows * q.split), (unsigned)q.tiles);
    cfg.blockDim = dim3(kThreads);
    // (never two blocks on a multiprocessor: tensor memory is for one)
    const size_t ring = (size_t)q.depth * q.tile * 128 + 1024, sums = q.split > 1 ? (size_t)MT * q.tile * kTileRows * 4 + 1024 : 0;
    cfg.dynamicSmemBytes = std::max(std::max(ring, sums), (size_t)kSmemPerSm / 2);
    cfg.stream = s;
    cfg.attrs = at;
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = (unsigned)f.split;
    at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cfg.numAttrs = f.split > 1 ? 2 : 1;
    return cuda_status(cudaLaunchKernelEx(&cfg, kernel, q));
}

template <int G> int launch_many_group(const ManyParams &q, const ManyPlan &f, int dev, cudaStream_t s)
{
    if (q.m.mins) return q.m.gated ? launch_many_as<G, true, 2>(q, f, dev, s) : launch_many_as<G, true, 1>(q, f, dev, s);
    return q.m.gated ? launch_many_as<G, false, 2>(q, f, dev, s) : launch_many_as<G, false, 1>(q, f, dev, s);
}

}  // namespace

// The tile of tokens (a multiple of 16, up to 256, gated 128) and the split over columns that
// take the fewest turns of the multiprocessors times a turn's length: two cycles a token and
// stage, no fewer than unpacking takes, and a fixed part.
ManyPlan plan_many(int outs, bool gated, int cols, int tokens, int sms)
{
    ManyPlan best{};
    double least = 1e300;
    const int mt = gated ? 2 : 1, row_tiles = (outs + kTileRows - 1) / kTileRows, stages = (cols + kStageCols - 1) / kStageCols;
    for (int tile = 32; tile <= 256 / mt; tile += 16) {
        const int tiles = (tokens + tile - 1) / tile;
        if (tile > 32 && (tokens + tiles - 1) / tiles <= tile - 16) continue;                  // (a smaller one does as well)
        for (int split = 1; split <= 8; split *= 2) {
            if (split > 1 && stages / split < 8) continue;
            const double turns = (double)(((int64_t)row_tiles * tiles * split + sms - 1) / sms);
            const double stage = mt * (2.0 * tile > 260.0 ? 2.0 * tile : 260.0);
            const double t = turns * (stage * ((stages + split - 1) / split) + 4000.0 + mt * 12.0 * tile + (split > 1 ? 2500.0 : 0.0));
            if (t < least) {
                least = t;
                const int fit = 200 * 1024 / (tile * 128);
                best = ManyPlan{tile, tiles, split, stages, fit < kMostX ? fit : kMostX, (size_t)tiles * stages * tile * 128, 0};
                best.workspace = best.image + (size_t)tokens * 4;
            }
        }
    }
    return best;
}

int launch_many(const MatmulParams &m, const ManyPlan &f, void *workspace, int outs, int dev, cudaStream_t s)
{
    ManyParams q{m, outs, f.tile, f.tiles, f.split, f.stages, f.depth, static_cast<const uint8_t *>(workspace),
                 reinterpret_cast<const float *>(static_cast<const uint8_t *>(workspace) + f.image)};
    return m.group == 32   ? launch_many_group<32>(q, f, dev, s)
           : m.group == 64 ? launch_many_group<64>(q, f, dev, s)
                           : launch_many_group<128>(q, f, dev, s);
}

}  // namespace e2ops
