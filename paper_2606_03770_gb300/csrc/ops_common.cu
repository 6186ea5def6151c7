// ops_common.cu -- host-side checks and error text of the operators.
#include "ops_common.cuh"

#include <atomic>
#include <cstdio>

namespace e2ops {

namespace {
thread_local char g_error[256] = "";
constexpr int kMaxDevices = 64;
std::atomic<int> g_sms[kMaxDevices];
}  // namespace

int fail(int status, const char *text)
{
    std::snprintf(g_error, sizeof g_error, "%s", text);
    return status;
}

int cuda_status(cudaError_t e) { return e == cudaSuccess ? E2_OK : fail(E2_ECUDA, cudaGetErrorString(e)); }

int current_device(Device *d)
{
    cudaError_t e = cudaGetDevice(&d->id);
    if (e != cudaSuccess) return cuda_status(e);
    if (d->id < 0 || d->id >= kMaxDevices) return fail(E2_EINVAL, "device id beyond the supported range");
    d->sms = g_sms[d->id].load(std::memory_order_relaxed);
    if (d->sms == 0) {
        e = cudaDeviceGetAttribute(&d->sms, cudaDevAttrMultiProcessorCount, d->id);
        if (e != cudaSuccess) return cuda_status(e);
        g_sms[d->id].store(d->sms, std::memory_order_relaxed);
    }
    return E2_OK;
}

bool on_device(const void *p, int dev)
{
    cudaPointerAttributes a;
    if (cudaPointerGetAttributes(&a, p) != cudaSuccess) {
        cudaGetLastError();
        return false;
    }
    return a.type == cudaMemoryTypeManaged || (a.type == cudaMemoryTypeDevice && a.device == dev);
}

}  // namespace e2ops

extern "C" const char *e2_ops_error(void) { return e2ops::g_error; }
