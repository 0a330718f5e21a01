// Status of a CUDA call as the entry points return it.
#pragma once

#include <cuda_runtime.h>

namespace gbmoe {

// GBMOE_OK, or GBMOE_ECUDA with the code kept for gbmoe_last_cuda_error
int cuda_status(cudaError_t e);

}  // namespace gbmoe
