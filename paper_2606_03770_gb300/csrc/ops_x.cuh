// ops_x.cuh -- 16-bit activations as the operand that meets 4-bit codes: fp16
// times a power of two, in the order of the codes' nibbles.
#pragma once

#include <type_traits>

#include "ops_mma.cuh"

namespace e2ops {

// 2^k that brings the largest magnitude (16 bits of T) to 2^14..2^15, k within fp32's normal range.
template <class T> __device__ __forceinline__ int power_for(unsigned bits)
{
    T top;
    *reinterpret_cast<uint16_t *>(&top) = (uint16_t)bits;
    return bits ? min(14 + 127 - (int)(__float_as_uint(to_float(top)) >> 23), 126) : 0;
}
// Whether a magnitude is infinite or NaN.
template <class T> __device__ __forceinline__ bool not_finite(unsigned bits)
{
    return bits >= (std::is_same<T, __half>::value ? 0x7c00u : 0x7f80u);
}
__device__ __forceinline__ float power_of_two(int k) { return __uint_as_float((unsigned)(127 + k) << 23); }

// The larger 16-bit magnitude of an octet.
__device__ __forceinline__ unsigned octet_largest(const uint4 &v)
{
    const unsigned m = __vmaxu2(__vmaxu2(v.x & 0x7fff7fffu, v.y & 0x7fff7fffu), __vmaxu2(v.z & 0x7fff7fffu, v.w & 0x7fff7fffu));
    return max(m & 0xffffu, m >> 16);
}

// An octet times f in fp16, in the order of the codes' nibbles, those that meet high
// nibbles with 1/16; and its sum.
template <class T> __device__ __forceinline__ uint4 octet_convert(const uint4 &v, float f, float &sum)
{
    float x[8];
    unpack8<T>(v, x);
    sum = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        x[j] *= f;
        sum += x[j];
    }
    const __half2 h[4] = {__floats2half2_rn(x[0], x[4]), __floats2half2_rn(x[1] * 0.0625f, x[5] * 0.0625f),
                          __floats2half2_rn(x[2], x[6]), __floats2half2_rn(x[3] * 0.0625f, x[7] * 0.0625f)};
    return *reinterpret_cast<const uint4 *>(h);
}

// The same times f, all alike.
template <class T> __device__ __forceinline__ uint4 octet_in_order(const uint4 &v, float f)
{
    float x[8];
    unpack8<T>(v, x);
    const __half2 h[4] = {__floats2half2_rn(x[0] * f, x[4] * f), __floats2half2_rn(x[1] * f, x[5] * f),
                          __floats2half2_rn(x[2] * f, x[6] * f), __floats2half2_rn(x[3] * f, x[7] * f)};
    return *reinterpret_cast<const uint4 *>(h);
}

// A word's eight codes c as m + d c in fp16, rounded once, in the same order.  A code
// in the low bits of 1024's fp16 makes 1024 + c, in the next four 1024 + 16 c.  A value
// may pass fp16's range, by the rounding of d or in a cache that was not written here: it
// stays fp16's largest (NaN stays NaN), unless the caller knows that none does.
template <bool LIMIT = true> __device__ __forceinline__ uint4 unpack_word(uint32_t w, __half2 d, __half2 m)
{
    const uint32_t v = w >> 8;
    uint32_t q[4] = {(w & 0x000f000fu) | 0x64006400u, (w & 0x00f000f0u) | 0x64006400u, (v & 0x000f000fu) | 0x64006400u,
                     (v & 0x00f000f0u) | 0x64006400u};
    const __half2 off = __float2half2_rn(-1024.0f), sixteenth = __float2half2_rn(0.0625f), high = __float2half2_rn(-64.0f);
    const __half2 most = __float2half2_rn(65504.0f);
    uint4 out;
    __half2 *o = reinterpret_cast<__half2 *>(&out);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __half2 x = *reinterpret_cast<const __half2 *>(&q[i]);
        const __half2 c = i % 2 ? __hfma2(x, sixteenth, high) : __hadd2(x, off);
        o[i] = __hfma2(c, d, m);
        if (LIMIT) o[i] = __hmin2_nan(__hmax2_nan(o[i], __hneg2(most)), most);
    }
    return out;
}

}  // namespace e2ops
