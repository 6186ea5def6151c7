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

// A kernel launched `early` is placed once all blocks of the one before it in its stream have
// called allow_next (or are gone); wait_before returns when that one is done and what it wrote
// can be seen.
__device__ __forceinline__ void wait_before() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void allow_next() { asm volatile("griddepcontrol.launch_dependents;"); }

// Launches a kernel in clusters of `cluster` blocks.
template <class P>
int launch(void (*kernel)(P), dim3 grid, int threads, size_t smem, int cluster, bool early, cudaStream_t s, const P &p)
{
    cudaLaunchAttribute at[2]{};
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cfg.attrs = at;
    if (early) {
        at[cfg.numAttrs].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        at[cfg.numAttrs++].val.programmaticStreamSerializationAllowed = 1;
    }
    if (cluster > 1) {
        at[cfg.numAttrs].id = cudaLaunchAttributeClusterDimension;
        at[cfg.numAttrs].val.clusterDim.x = (unsigned)cluster;
        at[cfg.numAttrs].val.clusterDim.y = at[cfg.numAttrs].val.clusterDim.z = 1;
        ++cfg.numAttrs;
    }
    return cuda_status(cudaLaunchKernelEx(&cfg, kernel, p));
}

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
