// Host part that the operators on device tensors share.
#include "isc_ops.h"

#include <atomic>
#include <cstdio>
#include <cstdlib>

namespace isc {
namespace ops {

cudaError_t current_device(Device *out)
{
    static std::atomic<int> sms[kMostDevices];
    static std::atomic<void *> encoder[kMostDevices];
    int ordinal = 0;
    cudaError_t e = cudaGetDevice(&ordinal);
    if (e != cudaSuccess) return e;
    const int slot = ordinal < kMostDevices ? ordinal : kMostDevices - 1;
    int n = ordinal < kMostDevices ? sms[slot].load(std::memory_order_acquire) : 0;
    void *fn = encoder[slot].load(std::memory_order_acquire);
    if (!n) {
        e = cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, ordinal);
        if (e != cudaSuccess) return e;
        cudaDriverEntryPointQueryResult qr;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &qr) != cudaSuccess || qr != cudaDriverEntryPointSuccess) {
            fn = nullptr;
            cudaGetLastError();
        }
        encoder[slot].store(fn, std::memory_order_release);
        if (ordinal < kMostDevices) sms[slot].store(n, std::memory_order_release);
    }
    *out = Device{ordinal, n, fn};
    return cudaSuccess;
}

int status_of(cudaError_t e, const char *what)
{
    if (e == cudaSuccess) return ISC_OK;
    if (getenv("ISC_DEBUG_CUDA")) fprintf(stderr, "isc: %s: %s\n", what, cudaGetErrorString(e));
    cudaGetLastError();
    return e == cudaErrorMemoryAllocation ? ISC_ERR_NOMEM : ISC_ERR_CUDA;
}

}  // namespace ops
}  // namespace isc

extern "C" int isc_operator_status(void *cuda_stream)
{
    using namespace isc::ops;
    // what this thread has been told of: another thread's question takes nothing away from it
    static thread_local uint32_t told[kMostDevices][3];
    const cudaStream_t st = (cudaStream_t)cuda_stream;
    int ordinal = 0;
    uint32_t now[3] = {};
    cudaError_t e = cudaGetDevice(&ordinal);
    if (e == cudaSuccess) e = norm_timeouts(st, &now[0]);
    if (e == cudaSuccess) e = linear_timeouts(st, &now[1]);
    if (e == cudaSuccess) e = log_probs_timeouts(st, &now[2]);
    if (e != cudaSuccess) return status_of(e, "operator_status");
    uint32_t *const mine = told[ordinal < kMostDevices ? ordinal : kMostDevices - 1];
    bool more = false;
    for (int i = 0; i < 3; ++i) {
        more |= now[i] != mine[i];
        mine[i] = now[i];
    }
    return more ? ISC_ERR_TIMEOUT : ISC_OK;
}
