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
  int T, num_blocks, block_size, kv_heads;
  int pairs;       // pairs of groups of 16 elements, of a head
  int per_token;   // and of a token's keys and values
  int log_lanes;   // 2^log_lanes threads take a token
  uint32_t* err;
};

constexpr int k4Threads = 256;

// Where a thread's pair of groups lies: of keys or values, the head, the pair.
struct Cache4Place {
  int which, h, pair;
};
__device__ __forceinline__ Cache4Place cache4_place(const Cache4Params& p, int e) {
  const unsigned head_of = static_cast<unsigned>(e) / static_cast<unsigned>(p.pairs);
  const int which = head_of >= static_cast<unsigned>(p.kv_heads);
  return {which, static_cast<int>(head_of) - (which ? p.kv_heads : 0), e - static_cast<int>(head_of) * p.pairs};
}
__device__ __forceinline__ void load_wide(unsigned (&r)[8], const void* p) {
  asm("ld.global.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]) : "l"(p));
}
__device__ __forceinline__ void store_wide(void* p, const unsigned (&r)[8]) {
  asm volatile("st.global.v8.b32 [%8], {%0,%1,%2,%3,%4,%5,%6,%7};" ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]),
               "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "l"(p) : "memory");
}

// Copies, bound by their bytes: a thread takes 32 elements with two scales, neighbours those of a head, then
// of the token's heads, then of its values.  WIDE: the elements lie on 32-byte boundaries.  16384 tokens of 8 heads of
// 128 bf16 written and read 32 us (a thread per 16 elements, 64-bit divisions: 46), the bytes 25; 100,003 read 98 = 5.4 TB/s.
// A write has five CTAs an SM where 48 registers hold 32 elements, as vectors of bf16, else four.  us of 16384 tokens
// written, with five and with four: fp32 32.0 and 30.8 (the bytes 22.6), off the boundaries bf16 65.7 and 62.8, fp32 121
// and 118 (with five 28 to 32 bytes a thread are spilled); vectors of bf16 18.4 with five.
template <typename T, bool WIDE>
constexpr int cache4_write_ctas() { return sizeof(T) == 2 && WIDE ? 5 : 4; }

template <typename T, bool WIDE>
__global__ void __launch_bounds__(k4Threads, (cache4_write_ctas<T, WIDE>())) cache4_write_kernel(const __grid_constant__ Cache4Params p) {
  const unsigned slots = static_cast<unsigned>(p.num_blocks) * static_cast<unsigned>(p.block_size);
  const int lanes = 1 << p.log_lanes, lane = threadIdx.x & (lanes - 1);
  const int64_t stride = static_cast<int64_t>(gridDim.x) * (k4Threads >> p.log_lanes);
  for (int64_t t = (static_cast<int64_t>(blockIdx.x) * k4Threads + threadIdx.x) >> p.log_lanes; t < p.T; t += stride) {
    const int64_t slot = p.slots[t];
    if (slot < 0) continue;
    if (slot >= slots) {
      if (lane == 0 && p.err) atomicOr(p.err, ASYMSPEC_DATA_BAD_INDEX);
      continue;
    }
    const unsigned block = static_cast<unsigned>(slot) / static_cast<unsigned>(p.block_size);
    const unsigned at = static_cast<unsigned>(slot) - block * static_cast<unsigned>(p.block_size);
    for (int e = lane; e < p.per_token; e += lanes) {
      const Cache4Place c = cache4_place(p, e);
      const Cache4Part& part = p.part[c.which];
      const T* x = static_cast<const T*>(p.x[c.which]) + t * p.xs[c.which][0] + c.h * p.xs[c.which][1] + c.pair * 32;
      float y[32];
      if constexpr (WIDE) {
        constexpr int N = 32 / sizeof(T);
        unsigned v[32 / N][8];
#pragma unroll
        for (int i = 0; i < 32 / N; ++i) load_wide(v[i], x + i * N);
#pragma unroll
        for (int i = 0; i < 32; ++i) {
          if constexpr (sizeof(T) == 4) y[i] = __uint_as_float(v[i / 8][i % 8]);
          else y[i] = __uint_as_float(i % 2 ? v[i / 16][i / 2 % 8] & 0xFFFF0000u : v[i / 16][i / 2 % 8] << 16);
        }
      } else {
#pragma unroll
        for (int i = 0; i < 32; ++i) y[i] = to_f32(x[i]);
      }
      unsigned code[4] = {0, 0, 0, 0}, scales = 0;
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        // (as whole numbers: a NaN is above every magnitude)
        unsigned most = 0;
#pragma unroll
        for (int i = 0; i < 16; ++i) most = max(most, __float_as_uint(y[16 * k + i]) & 0x7FFFFFFFu);
        const unsigned s = e4m3_byte(__fmul_rn(__uint_as_float(most), part.to_units));
        const float step = __fmul_rn(f16x2_to_f32(e4m3_to_f16(s)).x, part.scale);
        const float r = step > 0.f ? __frcp_rn(step) : 0.f;
        scales |= s << (8 * k);
#pragma unroll
        for (int i = 0; i < 8; ++i)
          code[2 * k + (i >> 2)] |= e2m1_pair(__fmul_rn(y[16 * k + 2 * i], r), __fmul_rn(y[16 * k + 2 * i + 1], r)) << (8 * (i & 3));
      }
      *reinterpret_cast<uint4*>(part.codes + block * part.cs[0] + at * part.cs[1] + c.h * part.cs[2] + c.pair * 16) =
          make_uint4(code[0], code[1], code[2], code[3]);
      *reinterpret_cast<uint16_t*>(part.scales + block * part.ss[0] + at * part.ss[1] + c.h * part.ss[2] + c.pair * 2) =
          static_cast<uint16_t>(scales);
    }
  }
}

template <typename T, bool WIDE>
__global__ void __launch_bounds__(k4Threads) cache4_read_kernel(const __grid_constant__ Cache4Params p) {
  const unsigned slots = static_cast<unsigned>(p.num_blocks) * static_cast<unsigned>(p.block_size);
  const int lanes = 1 << p.log_lanes, lane = threadIdx.x & (lanes - 1);
  const int64_t stride = static_cast<int64_t>(gridDim.x) * (k4Threads >> p.log_lanes);
  for (int64_t t = (static_cast<int64_t>(blockIdx.x) * k4Threads + threadIdx.x) >> p.log_lanes; t < p.T; t += stride) {
    const int64_t slot = p.slots[t];
    const bool there = slot >= 0 && slot < slots;
    if (slot >= slots && lane == 0 && p.err) atomicOr(p.err, ASYMSPEC_DATA_BAD_INDEX);
    const unsigned of = there ? static_cast<unsigned>(slot) : 0;
    const unsigned block = of / static_cast<unsigned>(p.block_size), at = of - block * static_cast<unsigned>(p.block_size);
    for (int e = lane; e < p.per_token; e += lanes) {
      const Cache4Place c = cache4_place(p, e);
      const Cache4Part& part = p.part[c.which];
      uint4 code = make_uint4(0, 0, 0, 0);
      unsigned scales = 0;
      if (there) {
        code = *reinterpret_cast<const uint4*>(part.codes + block * part.cs[0] + at * part.cs[1] + c.h * part.cs[2] + c.pair * 16);
        scales = *reinterpret_cast<const uint16_t*>(part.scales + block * part.ss[0] + at * part.ss[1] + c.h * part.ss[2] + c.pair * 2);
      }
      const unsigned both = e4m3_to_f16(scales);
      T* x = static_cast<T*>(p.x[c.which]) + t * p.xs[c.which][0] + c.h * p.xs[c.which][1] + c.pair * 32;
      const unsigned words[4] = {code.x, code.y, code.z, code.w};
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const unsigned s2 = __byte_perm(both, both, k ? 0x3232 : 0x1010);
        float y[16];
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          unsigned f[4];
          e2m1_to_f16(words[2 * k + w], f);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float2 v = f16x2_to_f32(mul_f16x2(f[i], s2));  // exact
            y[8 * w + 2 * i] = __fmul_rn(v.x, part.scale);
            y[8 * w + 2 * i + 1] = __fmul_rn(v.y, part.scale);
          }
        }
        if constexpr (WIDE) {
          constexpr int N = 32 / sizeof(T);
#pragma unroll
          for (int i = 0; i < 16 / N; ++i) {
            unsigned v[8];
#pragma unroll
            for (int d = 0; d < 8; ++d) {
              if constexpr (sizeof(T) == 4) v[d] = __float_as_uint(y[8 * i + d]);
              else asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(v[d]) : "f"(y[2 * d + 1]), "f"(y[2 * d]));
            }
            store_wide(x + 16 * k + i * N, v);
          }
        } else {
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            if constexpr (sizeof(T) == 4) x[16 * k + i] = y[i];
            else x[16 * k + i] = __float2bfloat16_rn(y[i]);
          }
        }
      }
    }
  }
}

}  // namespace asymspec_impl
