// What the operators on device tensors share on the host: element types, alignment, the current device's properties.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "isc.h"

namespace isc {
namespace ops {

inline bool is_float_type(int t) { return t == ISC_BF16 || t == ISC_F16 || t == ISC_F32; }
inline int type_bytes(int t) { return t == ISC_F32 ? 4 : t == ISC_I8 ? 1 : 2; }
inline bool aligned(const void *p, size_t to) { return ((uintptr_t)p & (to - 1)) == 0; }

// The current device as the operators' launches need it.  Filled once per device; a second thread that comes meanwhile fills it
// with the same values.
constexpr int kMostDevices = 64;          // whose properties are kept
struct Device {
    int ordinal, n_sms;
    void *encode;             // the driver's cuTensorMapEncodeTiled, or null
};
cudaError_t current_device(Device *out);

// How many bounded waits of the operators' kernels have run out on the current device; wait for `st`.
cudaError_t norm_timeouts(cudaStream_t st, uint32_t *count);
cudaError_t linear_timeouts(cudaStream_t st, uint32_t *count);
cudaError_t log_probs_timeouts(cudaStream_t st, uint32_t *count);

// A failed CUDA call as a status; clears the runtime's sticky copy of the error.
int status_of(cudaError_t e, const char *what);

}  // namespace ops
}  // namespace isc
