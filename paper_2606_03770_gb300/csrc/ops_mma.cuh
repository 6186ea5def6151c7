// ops_mma.cuh -- PTX wrappers of the operators' warp-level products: 16 x 8 x 16
// multiply-accumulate, matrix loads from shared memory, asynchronous copies, and
// the unpacking of 4-bit codes into 16-bit pairs.
#pragma once

#include "ops_common.cuh"

namespace e2ops {

__device__ __forceinline__ uint32_t smem_addr(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }

// 16 bytes to shared memory, zeros instead when !take.
__device__ __forceinline__ void copy_async16(uint32_t dst, const void *src, bool take)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(take ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copy_async4(uint32_t dst, const void *src, bool take)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(take ? 4 : 0) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ void load_matrices(uint32_t (&w)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3])
                 : "r"(addr)
                 : "memory");
}
__device__ __forceinline__ void load_matrices_t(uint32_t (&w)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3])
                 : "r"(addr)
                 : "memory");
}

// d += a b, 32-bit sums, of fp16 or bf16 operands.
template <bool BF>
__device__ __forceinline__ void multiply(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1)
{
    if constexpr (BF)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t h2_sub(uint32_t a, uint32_t b)
{
    uint32_t d;
    asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
__device__ __forceinline__ uint32_t h2_fma(uint32_t a, uint32_t b, uint32_t c)
{
    uint32_t d;
    asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
    return d;
}
__device__ __forceinline__ uint32_t bf2_fma(uint32_t a, uint32_t b, uint32_t c)
{
    uint32_t d;
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
    return d;
}

// A word's eight codes less 8, exactly, as the pairs of nibbles (0,4), (1,5),
// (2,6), (3,7).  A code OR-ed into the low bits of 1024 (fp16: steps of 1) or of 128
// (bf16: steps of 1) is that number plus the code; in fp16 the next four bits count
// sixteens, which a multiply-add brings back without a shift.
template <bool BF> __device__ __forceinline__ void centred_codes(uint32_t w, uint32_t (&p)[4])
{
    if constexpr (BF) {
        const uint32_t one = 0x3f803f80u, off = 0xc308c308u;     // 1, -136
        p[0] = bf2_fma((w & 0x000f000fu) | 0x43004300u, one, off);
        p[1] = bf2_fma((w >> 4 & 0x000f000fu) | 0x43004300u, one, off);
        p[2] = bf2_fma((w >> 8 & 0x000f000fu) | 0x43004300u, one, off);
        p[3] = bf2_fma((w >> 12 & 0x000f000fu) | 0x43004300u, one, off);
    } else {
        const uint32_t low = 0x64086408u;                          // 1032
        const uint32_t sixteenth = 0x2c002c00u, high = 0xd480d480u; // 1/16, -72
        const uint32_t v = w >> 8;
        p[0] = h2_sub((w & 0x000f000fu) | 0x64006400u, low);
        p[1] = h2_fma((w & 0x00f000f0u) | 0x64006400u, sixteenth, high);
        p[2] = h2_sub((v & 0x000f000fu) | 0x64006400u, low);
        p[3] = h2_fma((v & 0x00f000f0u) | 0x64006400u, sixteenth, high);
    }
}

}  // namespace e2ops
