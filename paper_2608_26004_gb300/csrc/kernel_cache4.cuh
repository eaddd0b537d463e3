// Writing and reading of a paged cache in 4 bits (asymspec_cache4_write, asymspec_cache4_read).
#pragma once

#include <cuda_fp16.h>

#include "asymspec_serving.h"
#include "device_common.cuh"

namespace asymspec_impl {

// Two codes, of a in the low and b in the high half of the byte; NaN and what is beyond 6 give 6.
__device__ __forceinline__ unsigned e2m1_pair(float a, float b) {
  unsigned r;
  asm("{.reg .b8 t, z; mov.b16 {z, z}, 0; cvt.rn.satfinite.e2m1x2.f32 t, %2, %1; mov.b32 %0, {t, z, z, z};}"
      : "=r"(r) : "f"(a), "f"(b));
  return r;
}
// The scale's byte, +448 at most; a NaN stays one.
__device__ __forceinline__ unsigned e4m3_byte(float a) {
  unsigned short r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(0.f), "f"(a));
  return r & 0xFFu;
}
// Two scales as fp16, which holds each of them.
__device__ __forceinline__ unsigned e4m3_to_f16(unsigned pair) {
  unsigned r;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"(static_cast<unsigned short>(pair)));
  return r;
}
// Eight codes as four pairs of fp16.
__device__ __forceinline__ void e2m1_to_f16(unsigned w, unsigned (&r)[4]) {
  asm("{.reg .b8 a, b, c, d; mov.b32 {a, b, c, d}, %4;\n\t"
      "cvt.rn.f16x2.e2m1x2 %0, a; cvt.rn.f16x2.e2m1x2 %1, b;\n\t"
      "cvt.rn.f16x2.e2m1x2 %2, c; cvt.rn.f16x2.e2m1x2 %3, d;}"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(w));
}
__device__ __forceinline__ unsigned mul_f16x2(unsigned a, unsigned b) {
  unsigned r;
  asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ float2 f16x2_to_f32(unsigned x) { return __half22float2(*reinterpret_cast<const __half2*>(&x)); }

struct Cache4Part {  // of keys, or of values
  char *codes, *scales;
  int64_t cs[3], ss[3];
  float scale, to_units;  // the pool's number, and 1 / (6 scale)
};

struct Cache4Params {
  Cache4Part part[2];
  void* x[2];  // keys and values outside the cache
  int64_t xs[2][2];
  const int64_t* slots;
  int T, num_blocks, block_size, kv_heads, groups;  // groups: of a head
  int per_token;                                    // groups of a token's keys and values
  uint32_t* err;
};

constexpr int k4Threads = 256;

// Copies, bound by their bytes: a thread takes 16 elements with one scale, neighbours those of a
// head, then of the token's heads, then of its values.  WIDE: the elements lie on 16-byte boundaries.
template <typename T, bool WIDE>
__global__ void __launch_bounds__(k4Threads) cache4_write_kernel(const __grid_constant__ Cache4Params p) {
  const int64_t total = static_cast<int64_t>(p.T) * p.per_token;
  const unsigned slots = static_cast<unsigned>(p.num_blocks) * static_cast<unsigned>(p.block_size);
  for (int64_t w = static_cast<int64_t>(blockIdx.x) * k4Threads + threadIdx.x; w < total;
       w += static_cast<int64_t>(gridDim.x) * k4Threads) {
    const int64_t t = w / p.per_token;
    const int e = static_cast<int>(w - t * p.per_token);
    const int64_t slot = p.slots[t];
    if (slot < 0) continue;
    if (slot >= slots) {
      if (e == 0 && p.err) atomicOr(p.err, ASYMSPEC_DATA_BAD_INDEX);
      continue;
    }
    const unsigned block = static_cast<unsigned>(slot) / static_cast<unsigned>(p.block_size);
    const unsigned at = static_cast<unsigned>(slot) - block * static_cast<unsigned>(p.block_size);
    const int head_of = e / p.groups, group = e - head_of * p.groups;
    const int which = head_of >= p.kv_heads, h = head_of - (which ? p.kv_heads : 0);
    const Cache4Part& c = p.part[which];
    const T* x = static_cast<const T*>(p.x[which]) + t * p.xs[which][0] + h * p.xs[which][1] + group * 16;
    float y[16];
    if constexpr (WIDE) {
      constexpr int N = 16 / sizeof(T);
      uint4 v[16 / N];
#pragma unroll
      for (int i = 0; i < 16 / N; ++i) v[i] = reinterpret_cast<const uint4*>(x)[i];
#pragma unroll
      for (int i = 0; i < 16; ++i) y[i] = to_f32(reinterpret_cast<const T*>(v)[i]);
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i) y[i] = to_f32(x[i]);
    }
    // (as whole numbers: a NaN is above every magnitude)
    unsigned most = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) most = max(most, __float_as_uint(y[i]) & 0x7FFFFFFFu);
    const unsigned s = e4m3_byte(__fmul_rn(__uint_as_float(most), c.to_units));
    const float step = __fmul_rn(f16x2_to_f32(e4m3_to_f16(s)).x, c.scale);
    const float r = step > 0.f ? __frcp_rn(step) : 0.f;
    unsigned code[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i)
      code[i >> 2] |= e2m1_pair(__fmul_rn(y[2 * i], r), __fmul_rn(y[2 * i + 1], r)) << (8 * (i & 3));
    *reinterpret_cast<uint2*>(c.codes + block * c.cs[0] + at * c.cs[1] + h * c.cs[2] + group * 8) =
        make_uint2(code[0], code[1]);
    c.scales[block * c.ss[0] + at * c.ss[1] + h * c.ss[2] + group] = static_cast<char>(s);
  }
}

template <typename T, bool WIDE>
__global__ void __launch_bounds__(k4Threads) cache4_read_kernel(const __grid_constant__ Cache4Params p) {
  const int64_t total = static_cast<int64_t>(p.T) * p.per_token;
  const unsigned slots = static_cast<unsigned>(p.num_blocks) * static_cast<unsigned>(p.block_size);
  for (int64_t w = static_cast<int64_t>(blockIdx.x) * k4Threads + threadIdx.x; w < total;
       w += static_cast<int64_t>(gridDim.x) * k4Threads) {
    const int64_t t = w / p.per_token;
    const int e = static_cast<int>(w - t * p.per_token);
    const int64_t slot = p.slots[t];
    const bool there = slot >= 0 && slot < slots;
    if (slot >= slots && e == 0 && p.err) atomicOr(p.err, ASYMSPEC_DATA_BAD_INDEX);
    const int head_of = e / p.groups, group = e - head_of * p.groups;
    const int which = head_of >= p.kv_heads, h = head_of - (which ? p.kv_heads : 0);
    const Cache4Part& c = p.part[which];
    unsigned code[2] = {0, 0}, s = 0;
    if (there) {
      const unsigned block = static_cast<unsigned>(slot) / static_cast<unsigned>(p.block_size);
      const unsigned at = static_cast<unsigned>(slot) - block * static_cast<unsigned>(p.block_size);
      const uint2 v = *reinterpret_cast<const uint2*>(c.codes + block * c.cs[0] + at * c.cs[1] + h * c.cs[2] + group * 8);
      code[0] = v.x, code[1] = v.y;
      s = static_cast<unsigned char>(c.scales[block * c.ss[0] + at * c.ss[1] + h * c.ss[2] + group]);
    }
    const unsigned s2 = e4m3_to_f16(s | s << 8);
    T* x = static_cast<T*>(p.x[which]) + t * p.xs[which][0] + h * p.xs[which][1] + group * 16;
    __align__(16) T y[16];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      unsigned f[4];
      e2m1_to_f16(code[k], f);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 v = f16x2_to_f32(mul_f16x2(f[i], s2));  // exact
        const float a = __fmul_rn(v.x, c.scale), b = __fmul_rn(v.y, c.scale);
        if constexpr (sizeof(T) == 4) y[8 * k + 2 * i] = a, y[8 * k + 2 * i + 1] = b;
        else y[8 * k + 2 * i] = __float2bfloat16_rn(a), y[8 * k + 2 * i + 1] = __float2bfloat16_rn(b);
      }
    }
    if constexpr (WIDE) {
#pragma unroll
      for (int i = 0; i < static_cast<int>(sizeof(T)); ++i)
        reinterpret_cast<uint4*>(x)[i] = reinterpret_cast<const uint4*>(y)[i];
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i) x[i] = y[i];
    }
  }
}

}  // namespace asymspec_impl
