// Status and detail text of the C entry points (defined in bitnet_api.hip).
#pragma once
#include <hip/hip_runtime.h>

namespace bitnet {

int fail(int status, const char* fmt, ...);               // sets the thread's detail text, returns status
int hip_status(hipError_t e, const char* what);           // BITNET_OK or BITNET_E_HIP with the error's text

}  // namespace bitnet
