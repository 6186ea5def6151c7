// ops_common.cuh -- what the operators of include/e2ops.h share: argument
// checks, element types, small device helpers.  Not part of the public ABI.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "e2ops.h"

namespace e2ops {

// Sets the calling thread's message (e2_ops_error) and returns the status.
int fail(int status, const char *text);
int cuda_status(cudaError_t e);

// The current device and its multiprocessors, looked up once per device.
struct Device {
    int id, sms;
};
int current_device(Device *d);

// Device memory of device `dev`, or managed memory.
bool on_device(const void *p, int dev);

inline bool aligned(const void *p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__half x) { return __half2float(x); }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
template <class T> __device__ __forceinline__ T from_float(float x);
template <> __device__ __forceinline__ float from_float<float>(float x) { return x; }
template <> __device__ __forceinline__ __half from_float<__half>(float x) { return __float2half_rn(x); }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

// Eight 16-bit elements as they lie in memory, in 32 bits.
template <class T> __device__ __forceinline__ void unpack8(const uint4 &w, float (&x)[8])
{
    const T *e = reinterpret_cast<const T *>(&w);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = to_float(e[i]);
}
template <class T> __device__ __forceinline__ uint4 pack8(const float (&x)[8])
{
    uint4 w;
    T *e = reinterpret_cast<T *>(&w);
#pragma unroll
    for (int i = 0; i < 8; ++i) e[i] = from_float<T>(x[i]);
    return w;
}

}  // namespace e2ops
