// pc_host.h -- what the host files of the ABI share: the failure record of
// the calling thread (pc_last_error) and the checks around a launch.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace pcr {

// Records the message for pc_last_error and returns `code`.
int32_t fail(int32_t code, const char *fmt, ...);
int32_t ok();
int32_t hip_fail(hipError_t e, const char *what);

}  // namespace pcr
