// Host helpers of the operators around the step: alignment and types, launches.
#pragma once

#include <climits>
#include <cstdint>

#include "asymspec_serving.h"
#include "device_common.cuh"
#include "host_common.h"
#include "prepared.h"

namespace asymspec_impl {

constexpr int64_t kMax32 = INT32_MAX;

inline bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

inline int elt_size(int dtype) { return dtype == ASYMSPEC_FP32 ? 4 : 2; }

inline bool known_dtype(int dtype) { return dtype == ASYMSPEC_FP32 || dtype == ASYMSPEC_BF16; }

constexpr int kStaticSmem = 8192;  // what a kernel has beside its dynamic shared memory at most

inline Prepared g_prepared;

// Once per kernel and device: room for all the dynamic shared memory that it may ask for.
inline cudaError_t prepare(const void* fn, int device, int smem) {
  if (smem <= 48 * 1024 - kStaticSmem) return cudaSuccess;
  return static_cast<cudaError_t>(g_prepared.once(fn, device, [fn] {
    return static_cast<int>(cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxSmem - kStaticSmem));
  }));
}

// For numbers k below 2^30 and n <= 2^s, d = ceil(2^(31 + s) / n) gives k / n = k * d >> (31 + s): d n is less than n
// above 2^(31 + s), and k times that less than 2^(31 + s).
inline void divide_by(int n, unsigned* d, int* s) {
  *s = 0;
  while ((1ll << *s) < n) ++*s;
  *d = static_cast<unsigned>(((1ull << (31 + *s)) + n - 1) / n);
}

inline cudaError_t device_sms(int* device, int* sms) {
  const cudaError_t e = cudaGetDevice(device);
  return e == cudaSuccess ? cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, *device) : e;
}

inline int launch(const void* fn, dim3 grid, dim3 block, size_t smem, void* params, void* stream) {
  cudaError_t e = cudaSuccess;
  if (smem > 48 * 1024 - kStaticSmem) {
    int device = 0;
    e = cudaGetDevice(&device);
    if (e == cudaSuccess) e = prepare(fn, device, static_cast<int>(smem));
    if (e != cudaSuccess) return cuda_fail(e);
  }
  void* args[] = {params};
  e = cudaLaunchKernel(fn, grid, block, args, smem, static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? ASYMSPEC_OK : cuda_fail(e);
}

}  // namespace asymspec_impl
