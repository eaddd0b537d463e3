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
};

struct RotaryParams {
  RotaryHeads x[2];  // queries, keys
  int T, head_dim, rot;
  int turning;       // a head's units that turn; the others copy
  int all_units;     // of a token
  int tokens, each;  // of a CTA: tokens, and units of each
  bool transpose;
  float magnitude;
  const int32_t* positions;
  const uint64_t* steps;
};

constexpr int kRThreads = 256;
constexpr int kRBatch = 3;       // units that a thread has on their way together
constexpr int kRTable = 2048;    // cosines and sines of a CTA's tokens at most
constexpr int kRTokens = 256;    // tokens of a CTA at most

template <typename T, typename U>
struct RotaryVector {
  static constexpr int N = sizeof(U) / sizeof(T);
  U u;
  __device__ __forceinline__ float get(int i) const { return to_f32(reinterpret_cast<const T*>(&u)[i]); }
  __device__ __forceinline__ void set(int i, float y) {
    if constexpr (sizeof(T) == 4) reinterpret_cast<T*>(&u)[i] = y;
    else reinterpret_cast<T*>(&u)[i] = __float2bfloat16_rn(y);
  }
};

// A copy with three operations an element: bound by its bytes.  A CTA takes a few tokens' heads: it
// computes their cosines and sines once, into shared memory, while its threads' first loads are
// on their way.  A unit is what a thread moves at once: the same vector of both halves
// (or two neighbours, interleaved: one vector, or a pair), or a vector past rotary_dim.
// 16384 tokens of 40 heads of 128 bf16: 66 us = 5.1 TB/s (three units of a thread at once; two 72, four 67; CTAs of
// 128 threads the same), 5 tokens of 24 heads 2.7 us.
// U: 16 bytes, or one element where something is not on the 16-byte boundaries.
template <typename T, typename U, bool INTER>
__global__ void __launch_bounds__(kRThreads) rotary_kernel(const __grid_constant__ RotaryParams p) {
  using V = RotaryVector<T, U>;
  constexpr int N = V::N;
  constexpr bool kOne = INTER && N > 1;  // a turning unit is one vector
  __shared__ float2 s_turn[kRTable];
  __shared__ int s_pos[kRTokens];
  const int tid = threadIdx.x, half = p.rot / 2;
  const int t0 = blockIdx.x * p.tokens, nt = min(p.tokens, p.T - t0);
  const int e0 = blockIdx.y * p.each, ne = min(p.each, p.all_units - e0);
  const int total = nt * ne;

  V a[kRBatch], b[kRBatch];
  int64_t to[kRBatch];  // element of the output; below 0: nothing to do
  int info[kRBatch];    // token, unit of the head, which tensor
  auto load = [&](int first) {
#pragma unroll
    for (int i = 0; i < kRBatch; ++i) {
      const int w = first + i * kRThreads;
      to[i] = -1;
      if (w >= total) continue;
      const int t = w / ne;
      int e = e0 + w - t * ne;
      const int which = e >= p.x[0].heads * p.x[0].units;
      const RotaryHeads& x = p.x[which];
      if (which) e -= p.x[0].heads * p.x[0].units;
      const int h = e / x.units, u = e - h * x.units;
      const bool turns = u < p.turning;
      const int at = turns ? u * (kOne ? N : INTER ? 2 : N) : p.rot + (u - p.turning) * N;
      const T* in = static_cast<const T*>(x.in) + (t0 + t) * x.is[0] + h * x.is[1] + at;
      to[i] = (t0 + t) * x.os[0] + h * x.os[1] + at;
      info[i] = t << 20 | u << 1 | which;
      a[i].u = *reinterpret_cast<const U*>(in);
      if (turns && !kOne) b[i].u = *reinterpret_cast<const U*>(in + (INTER ? 1 : half));
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
    s_turn[i] = make_float2(back ? -x : x, back != p.transpose ? -y : y);
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
        const float2* table = s_turn + t * half + u * (kOne ? N / 2 : INTER ? 1 : N);
        if constexpr (kOne) {
#pragma unroll
          for (int k = 0; k < N / 2; ++k) {
            const float y = a[i].get(2 * k), z = a[i].get(2 * k + 1);
            const float2 cs = table[k];
            a[i].set(2 * k, cs.x * y - cs.y * z);
            a[i].set(2 * k + 1, cs.y * y + cs.x * z);
          }
        } else {
#pragma unroll
          for (int k = 0; k < N; ++k) {
            const float y = a[i].get(k), z = b[i].get(k);
            const float2 cs = table[k];
            a[i].set(k, cs.x * y - cs.y * z);
            b[i].set(k, cs.y * y + cs.x * z);
          }
        }
      }
      *reinterpret_cast<U*>(out) = a[i].u;
      if (turns && !kOne) *reinterpret_cast<U*>(out + (INTER ? 1 : half)) = b[i].u;
    }
    first += kRThreads * kRBatch;
    if (first >= total) break;
    load(first);
  }
}

}  // namespace asymspec_impl
