// Host helpers shared by the library's entry points.
#pragma once

#include <hip/hip_runtime.h>

namespace llc {

// Remembers a HIP error for ll_strerror in this thread and returns LL_ERR_HIP.
int hip_failed(hipError_t e);
// LL_OK, or the error of the launches just made.
int launch_status();
// Compute units of the current device.
int device_cus(int *cus);

}  // namespace llc
