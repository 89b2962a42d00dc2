// Host part that the operators on device tensors share.
#include "isc_ops.h"

#include <atomic>
#include <cstdio>
#include <cstdlib>

namespace isc {
namespace ops {

cudaError_t current_device(Device *out)
{
    constexpr int kMost = 64;
    static std::atomic<int> sms[kMost];
    static std::atomic<void *> encoder[kMost];
    int ordinal = 0;
    cudaError_t e = cudaGetDevice(&ordinal);
    if (e != cudaSuccess) return e;
    const int slot = ordinal < kMost ? ordinal : kMost - 1;
    int n = ordinal < kMost ? sms[slot].load(std::memory_order_acquire) : 0;
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
        if (ordinal < kMost) sms[slot].store(n, std::memory_order_release);
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
    bool norm = false, linear = false, log_probs = false;
    cudaError_t e = norm_take_timeout((cudaStream_t)cuda_stream, &norm);
    if (e == cudaSuccess) e = linear_take_timeout((cudaStream_t)cuda_stream, &linear);
    if (e == cudaSuccess) e = log_probs_take_timeout((cudaStream_t)cuda_stream, &log_probs);
    if (e != cudaSuccess) return status_of(e, "operator_status");
    return norm || linear || log_probs ? ISC_ERR_TIMEOUT : ISC_OK;
}
