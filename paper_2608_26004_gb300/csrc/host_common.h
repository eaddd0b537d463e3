// Host helpers shared by the C ABI's translation units.
#pragma once

#include <cuda_runtime.h>

#include <cstddef>
#include <cstdint>

namespace asymspec_impl {

// Records a failed CUDA call for asymspec_last_cuda_error; returns ASYMSPEC_ERR_CUDA.
int cuda_fail(cudaError_t e);

}  // namespace asymspec_impl
