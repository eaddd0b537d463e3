// Attention of a few new tokens over a paged key-value cache (asymspec_cache_attend).
#pragma once

#include <cfloat>

#include "asymspec_serving.h"
#include "device_common.cuh"

namespace asymspec_impl {

struct AttendParams {
  const void *keys, *values, *q;
  void* out;
  float* lse;
  int64_t cks[3], cvs[3], qs[3], os[3];
  const int32_t *tables, *lens;
  int64_t table_ld;
  int B, Q, heads, kv_heads, D, num_blocks, block_size, table_width, window;
  float scale;
  uint32_t* err;
};

constexpr int kAThreads = 256;
constexpr int kAWarps = kAThreads / 32;

__device__ __forceinline__ void put(float* p, float y) { *p = y; }
__device__ __forceinline__ void put(__nv_bfloat16* p, float y) { *p = __float2bfloat16_rn(y); }

// One CTA per query and head: its warps take the keys in turn, a lane up to eight elements
// of a head, each warp with a running maximum and sum of its own; joined at the end.
template <typename T>
__global__ void __launch_bounds__(kAThreads) attend_kernel(const AttendParams p) {
  __shared__ float s_m[kAWarps], s_l[kAWarps], s_o[kAWarps][256];
  const int h = blockIdx.x, i = blockIdx.y, b = blockIdx.z;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int kh = h / (p.heads / p.kv_heads);
  const int len0 = p.lens[b];
  const int len = min(max(len0, 0), p.table_width * p.block_size);
  unsigned err = len != len0 ? ASYMSPEC_DATA_BAD_LENGTH : 0u;
  const int last = len - p.Q + i;
  const int first = p.window ? max(0, last - p.window + 1) : 0;
  const T* q = static_cast<const T*>(p.q) + b * p.qs[0] + i * p.qs[1] + h * p.qs[2];
  float x[8], o[8], m = -INFINITY, l = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int d = lane + 32 * e;
    x[e] = d < p.D ? to_f32(q[d]) * p.scale : 0.f;
    o[e] = 0.f;
  }
  for (int j = first + warp; j <= last; j += kAWarps) {
    const int page = p.tables[b * p.table_ld + j / p.block_size], at = j % p.block_size;
    if (static_cast<unsigned>(page) >= static_cast<unsigned>(p.num_blocks)) {
      err |= ASYMSPEC_DATA_BAD_INDEX;
      continue;
    }
    const T* k = static_cast<const T*>(p.keys) + page * p.cks[0] + at * p.cks[1] + kh * p.cks[2];
    const T* v = static_cast<const T*>(p.values) + page * p.cvs[0] + at * p.cvs[1] + kh * p.cvs[2];
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (lane + 32 * e < p.D) s = fmaf(x[e], to_f32(k[lane + 32 * e]), s);
#pragma unroll
    for (int d = 16; d; d >>= 1) s += __shfl_xor_sync(~0u, s, d);
    const float m2 = fmaxf(m, s), ref = m2 == -INFINITY ? 0.f : m2;
    const float f = expf(m - ref), w = expf(s - ref);
    m = m2;
    l = l * f + w;
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (lane + 32 * e < p.D) o[e] = fmaf(w, to_f32(v[lane + 32 * e]), o[e] * f);
  }
  if (lane == 0) s_m[warp] = m, s_l[warp] = l;
#pragma unroll
  for (int e = 0; e < 8; ++e) s_o[warp][lane + 32 * e] = o[e];
  __syncthreads();
  float M = -INFINITY, L = 0.f, O = 0.f;
  for (int w = 0; w < kAWarps; ++w) M = fmaxf(M, s_m[w]);
  for (int w = 0; w < kAWarps; ++w) {
    const float f = s_m[w] == -INFINITY ? 0.f : expf(s_m[w] - M);
    L += f * s_l[w];
    O += f == 0.f ? 0.f : f * s_o[w][threadIdx.x];
  }
  if (threadIdx.x < p.D)
    put(static_cast<T*>(p.out) + b * p.os[0] + i * p.os[1] + h * p.os[2] + threadIdx.x,
        L > 0.f ? O / L : (L == 0.f ? 0.f : L));
  if (threadIdx.x == 0 && p.lse)
    p.lse[(static_cast<int64_t>(b) * p.Q + i) * p.heads + h] = M + logf(L);
  if (err && p.err) atomicOr(p.err, err);
}

}  // namespace asymspec_impl
