// Queries and keys turned by their positions (asymspec_rotary).
#pragma once

#include "asymspec_serving.h"
#include "device_common.cuh"

namespace asymspec_impl {

struct RotaryHeads {
  const void* in;
  void* out;
  int64_t is[2], os[2];
  int heads, units;  // a head's units of work (see below)
  unsigned divide;   // n / units is the high half of 2 n * divide, shifted
  int shift;
};

struct RotaryParams {
  RotaryHeads x[2];  // queries, keys
  int T, head_dim, rot;
  int turning;       // a head's units that turn; the others copy
  int all_units;     // of a token
  unsigned divide;   // the same for n / all_units
  int shift;
  int tokens, each;  // of a CTA: tokens, and units of each
  bool transpose;
  float magnitude;
  const int32_t* positions;
  const uint64_t* steps;
};

constexpr int kRThreads = 128;
constexpr int kRBatch = 3;       // units that a thread has on their way together
constexpr int kRTable = 1024;    // cosines and sines of a CTA's tokens at most
constexpr int kRTokens = 256;    // tokens of a CTA at most

__device__ __forceinline__ float2 turned(float2 cs, float a, float b) {
  return make_float2(cs.x * a - cs.y * b, cs.y * a + cs.x * b);
}
// Two bf16 numbers of a word.
__device__ __forceinline__ float2 unpacked(unsigned w) {
  return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
}
__device__ __forceinline__ unsigned packed(float a, float b) {
  unsigned r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
  return r;
}
__device__ __forceinline__ unsigned divided(int n, unsigned divide, int shift) {
  return __umulhi(2u * static_cast<unsigned>(n), divide) >> shift;
}

// A copy with three operations an element: bound by its bytes.  A CTA takes a few tokens' heads: it
// computes their cosines and sines once, into shared memory, while its threads' first loads are
// on their way.  A unit is what a thread moves at once: the same vector of both halves
// (or two neighbours, interleaved: one vector, or a pair), or a vector past rotary_dim.
// A vector's pairs lie in the table two by two (chunks of 16 bytes), the same two of all vectors next to one another, so
// that lanes meet no bank twice.  16384 tokens of 40 heads of 128 bf16 take 52 us = 6.4 TB/s (one after another in the
// table, 64-bit reads that met banks four times, divisions: 66), 4099 of 40 heads of 64 9.3 us, 5 of 24 heads 2.4.
// CTAs of 256 threads: 53 and 10.2 us; of two units a thread, six an SM, 53.5 and 9.1.
// U: 16 bytes, or one element where something is not on the 16-byte boundaries.
template <typename T, typename U, bool INTER>
__global__ void __launch_bounds__(kRThreads, 8) rotary_kernel(const __grid_constant__ RotaryParams p) {
  constexpr int N = sizeof(U) / sizeof(T);
  constexpr bool kOne = INTER && N > 1;  // a turning unit is one vector
  constexpr int kPairs = kOne ? N / 2 : N;  // of a unit
  __shared__ __align__(16) float2 s_turn[kRTable];
  __shared__ int s_pos[kRTokens];
  const int tid = threadIdx.x, half = p.rot / 2;
  const int t0 = blockIdx.x * p.tokens, nt = min(p.tokens, p.T - t0);
  const int e0 = blockIdx.y * p.each, ne = min(p.each, p.all_units - e0);
  const int total = nt * ne;

  U a[kRBatch], b[kRBatch];
  int64_t to[kRBatch];  // element of the output; below 0: nothing to do
  int info[kRBatch];    // token, unit of the head, which tensor
  auto load = [&](int first) {
#pragma unroll
    for (int i = 0; i < kRBatch; ++i) {
      const int w = first + i * kRThreads;
      to[i] = -1;
      if (w >= total) continue;
      const int t = p.tokens > 1 ? divided(w, p.divide, p.shift) : 0;  // (then ne is all_units)
      int e = e0 + w - t * ne;
      const int which = e >= p.x[0].heads * p.x[0].units;
      const RotaryHeads& x = p.x[which];
      if (which) e -= p.x[0].heads * p.x[0].units;
      const int h = divided(e, x.divide, x.shift), u = e - h * x.units;
      const bool turns = u < p.turning;
      const int at = turns ? u * (kOne ? N : INTER ? 2 : N) : p.rot + (u - p.turning) * N;
      const T* in = static_cast<const T*>(x.in) + (t0 + t) * x.is[0] + h * x.is[1] + at;
      to[i] = (t0 + t) * x.os[0] + h * x.os[1] + at;
      info[i] = t << 20 | u << 1 | which;
      a[i] = *reinterpret_cast<const U*>(in);
      if (turns && !kOne) b[i] = *reinterpret_cast<const U*>(in + (INTER ? 1 : half));
    }
  };
  load(tid);
  for (int i = tid; i < nt * half; i += kRThreads) {
    const int t = i / half, pair = i - t * half;
    const int pos = p.positions[t0 + t];
    if (pair == 0) s_pos[t] = pos;
    // the phase: a fraction of a turn, modulo one, exact but for the step's own rounding; and what
    // is left of it within an eighth of a turn of a quarter (fp32 rounds it by 2^-28 turns at most)
    const unsigned phase = static_cast<unsigned>((p.steps[pair] * static_cast<uint64_t>(max(pos, 0))) >> 32);
    const unsigned quarter = (phase + (1u << 29)) >> 30;
    float s, c;
    sincospif(static_cast<float>(static_cast<int>(phase - (quarter << 30))) * 0x1p-31f, &s, &c);
    const float y = p.magnitude * (quarter & 1 ? c : s), x = p.magnitude * (quarter & 1 ? -s : c);
    const bool back = quarter & 2;
    const int u = pair / kPairs, k = pair % kPairs;
    s_turn[kPairs == 1 ? i : t * half + (k / 2 * p.turning + u) * 2 + (k & 1)] =
        make_float2(back ? -x : x, back != p.transpose ? -y : y);
  }
  __syncthreads();
  for (int first = tid;;) {
#pragma unroll
    for (int i = 0; i < kRBatch; ++i) {
      if (to[i] < 0) continue;
      const int t = info[i] >> 20, u = (info[i] >> 1) & 0x7FFFF, which = info[i] & 1;
      const RotaryHeads& x = p.x[which];
      T* out = static_cast<T*>(x.out) + to[i];
      const bool live = s_pos[t] >= 0;
      if (!live && x.in == x.out) continue;
      const bool turns = u < p.turning;
      if (turns && live) {
        if constexpr (N == 1) {
          T* const one = reinterpret_cast<T*>(a + i);
          T* const two = reinterpret_cast<T*>(b + i);
          const float2 y = turned(s_turn[t * half + u], to_f32(*one), to_f32(*two));
          if constexpr (sizeof(T) == 4) *one = y.x, *two = y.y;
          else *one = __float2bfloat16_rn(y.x), *two = __float2bfloat16_rn(y.y);
        } else {
          const float4* table = reinterpret_cast<const float4*>(s_turn + t * half) + u;
          unsigned* va = reinterpret_cast<unsigned*>(a + i);
          unsigned* vb = reinterpret_cast<unsigned*>(b + i);
#pragma unroll
          for (int k = 0; k < kPairs / 2; ++k) {
            const float4 both = table[k * p.turning];
            const float2 cs0 = make_float2(both.x, both.y), cs1 = make_float2(both.z, both.w);
            if constexpr (sizeof(T) == 2 && kOne) {  // a pair to a word
              const float2 x0 = unpacked(va[2 * k]), x1 = unpacked(va[2 * k + 1]);
              const float2 y0 = turned(cs0, x0.x, x0.y), y1 = turned(cs1, x1.x, x1.y);
              va[2 * k] = packed(y0.x, y0.y);
              va[2 * k + 1] = packed(y1.x, y1.y);
            } else if constexpr (sizeof(T) == 2) {
              const float2 xa = unpacked(va[k]), xb = unpacked(vb[k]);
              const float2 y0 = turned(cs0, xa.x, xb.x), y1 = turned(cs1, xa.y, xb.y);
              va[k] = packed(y0.x, y1.x);
              vb[k] = packed(y0.y, y1.y);
            } else {
              unsigned* const other = kOne ? va : vb;
              const int at[4] = {kOne ? 4 * k : 2 * k, kOne ? 4 * k + 1 : 2 * k, kOne ? 4 * k + 2 : 2 * k + 1,
                                 kOne ? 4 * k + 3 : 2 * k + 1};
              const float2 y0 = turned(cs0, __uint_as_float(va[at[0]]), __uint_as_float(other[at[1]]));
              const float2 y1 = turned(cs1, __uint_as_float(va[at[2]]), __uint_as_float(other[at[3]]));
              va[at[0]] = __float_as_uint(y0.x), other[at[1]] = __float_as_uint(y0.y);
              va[at[2]] = __float_as_uint(y1.x), other[at[3]] = __float_as_uint(y1.y);
            }
          }
        }
      }
      *reinterpret_cast<U*>(out) = a[i];
      if (turns && !kOne) *reinterpret_cast<U*>(out + (INTER ? 1 : half)) = b[i];
    }
    first += kRThreads * kRBatch;
    if (first >= total) break;
    load(first);
  }
}

}  // namespace asymspec_impl
