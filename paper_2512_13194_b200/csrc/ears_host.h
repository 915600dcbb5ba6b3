// What the library's translation units share on the host side.
#pragma once
#include <cuda_runtime.h>

namespace ears {

// Records the text of a failing CUDA call for ears_last_cuda_error; -> EARS_ERR_CUDA.
int host_cuda_fail(cudaError_t e, const char* what);
// SM count of the current device (cached).
int host_device_sms(int* sms);

}  // namespace ears
