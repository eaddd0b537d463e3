// Host helpers of the operators around the step: alignment and types, launches.
#pragma once

#include <climits>
#include <cstdint>
#include <mutex>

#include "asymspec_serving.h"
#include "device_common.cuh"
#include "host_common.h"

namespace asymspec_impl {

constexpr int64_t kMax32 = INT32_MAX;

inline bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

inline int elt_size(int dtype) { return dtype == ASYMSPEC_FP32 ? 4 : 2; }

inline bool known_dtype(int dtype) { return dtype == ASYMSPEC_FP32 || dtype == ASYMSPEC_BF16; }

constexpr int kStaticSmem = 8192;  // what a kernel has beside its dynamic shared memory at most

// Once per kernel and device: room for all the dynamic shared memory that it may ask for.
struct Prepared {
  const void* fn;
  int device;
};
inline std::mutex g_mu;
inline Prepared g_prepared[64];
inline int g_prepared_count = 0;

inline cudaError_t prepare(const void* fn, int device, int smem) {
  if (smem <= 48 * 1024 - kStaticSmem) return cudaSuccess;
  std::lock_guard<std::mutex> lock(g_mu);
  for (int i = 0; i < g_prepared_count; ++i)
    if (g_prepared[i].fn == fn && g_prepared[i].device == device) return cudaSuccess;
  const cudaError_t e = cudaFuncSetAttribute(fn, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxSmem - kStaticSmem);
  if (e == cudaSuccess && g_prepared_count < 64) g_prepared[g_prepared_count++] = {fn, device};
  return e;
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
