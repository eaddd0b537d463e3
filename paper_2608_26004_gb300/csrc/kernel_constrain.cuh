// Penalties, biases and grammar masks on a round's logits (asymspec_constrain_logits).
#pragma once

#include <cfloat>

#include "asymspec_serving.h"
#include "device_common.cuh"

namespace asymspec_impl {

struct CParams {
  asymspec_constraints c;
  const void* logits;
  void* out;
  int64_t ld, out_ld;
  int B, P, V;
  uint32_t* err;
};

constexpr int kCThreads = 256;
constexpr int kCSlice = 4096;           // vocabulary entries of a CTA
constexpr unsigned kCPrompt = 1u << 31;  // the token is in the prompt; below: its output count

__device__ __forceinline__ float type_max(float) { return FLT_MAX; }
__device__ __forceinline__ float type_max(__nv_bfloat16) { return __uint_as_float(0x7F7F0000u); }
__device__ __forceinline__ void store1(float* p, float y) { *p = y; }
__device__ __forceinline__ void store1(__nv_bfloat16* p, float y) { *p = __float2bfloat16_rn(y); }

// One CTA per slice of the vocabulary and request: the history's counts of its slice in
// shared memory, then the request's rows in order, each draft counted after its row.
template <typename T>
__global__ void __launch_bounds__(kCThreads) constrain_kernel(const CParams p) {
  extern __shared__ unsigned c_smem[];
  unsigned* cnt = c_smem;
  int* bias_at = reinterpret_cast<int*>(c_smem + kCSlice);  // 1 + the entry of a biased token
  const asymspec_constraints& c = p.c;
  const int b = blockIdx.y, v0 = blockIdx.x * kCSlice, n = min(kCSlice, p.V - v0);
  const int tid = threadIdx.x;
  unsigned err = 0;
  for (int i = tid; i < kCSlice; i += kCThreads) {
    cnt[i] = 0;
    if (c.bias_offsets) bias_at[i] = 0;
  }
  __syncthreads();
  if (c.history) {
    const int len0 = c.history_len[b], len = min(max(len0, 0), c.history_width);
    const int pl0 = c.prompt_len ? c.prompt_len[b] : 0, pl = min(max(pl0, 0), len);
    if (len != len0 || pl != pl0) err |= ASYMSPEC_DATA_BAD_LENGTH;
    const int32_t* h = c.history + b * c.history_ld;
    for (int i = tid; i < len; i += kCThreads) {
      const int v = h[i];
      if (static_cast<unsigned>(v) >= static_cast<unsigned>(p.V)) err |= ASYMSPEC_DATA_BAD_TOKEN;
      else if (v >= v0 && v < v0 + n) {
        if (i < pl) atomicOr(&cnt[v - v0], kCPrompt);
        else atomicAdd(&cnt[v - v0], 1u);
      }
    }
  }
  if (c.bias_offsets) {
    const int a0 = c.bias_offsets[b], e0 = c.bias_offsets[b + 1];
    const int a = min(max(a0, 0), c.bias_count), e = min(max(e0, a), c.bias_count);
    if (a != a0 || e != e0) err |= ASYMSPEC_DATA_BAD_LENGTH;
    for (int i = a + tid; i < e; i += kCThreads) {
      const int v = c.bias_tokens[i];
      if (static_cast<unsigned>(v) >= static_cast<unsigned>(p.V)) err |= ASYMSPEC_DATA_BAD_TOKEN;
      else if (v >= v0 && v < v0 + n) atomicMax(&bias_at[v - v0], i + 1);
    }
  }
  float rep = c.repetition ? c.repetition[b] : 1.f, freq = c.frequency ? c.frequency[b] : 0.f,
        pres = c.presence ? c.presence[b] : 0.f;
  if (!(rep > 0.f && rep <= FLT_MAX && fabsf(freq) <= FLT_MAX && fabsf(pres) <= FLT_MAX)) {
    err |= ASYMSPEC_DATA_BAD_PENALTY;
    rep = 1.f;
    freq = pres = 0.f;
  }
  const float top = type_max(T());
  const float low = fminf(fmaxf(c.mask_value, -top), top);
  for (int k = 0; k < p.P; ++k) {
    __syncthreads();
    const int64_t r = static_cast<int64_t>(b) * p.P + k;
    const T* x = static_cast<const T*>(p.logits) + r * p.ld + v0;
    T* y = static_cast<T*>(p.out) + r * p.out_ld + v0;
    const uint32_t* mask = nullptr;
    bool none = false;
    if (c.mask) {
      const int at = c.mask_rows ? c.mask_rows[r] : static_cast<int>(r);
      none = at < -1 || at >= c.mask_count;
      if (none) err |= ASYMSPEC_DATA_BAD_INDEX;
      if (!none && at >= 0) mask = c.mask + at * c.mask_ld;
    }
    for (int i = tid; i < n; i += kCThreads) {
      const unsigned w = cnt[i];
      const int bi = c.bias_offsets ? bias_at[i] : 0;
      const T raw = x[i];
      if (none || (mask && !((mask[(v0 + i) >> 5] >> ((v0 + i) & 31)) & 1u))) store1(y + i, low);
      else if (w == 0 && bi == 0) y[i] = raw;
      else {
        const float z = to_f32(raw);
        float s = z;
        if (w) {
          const float m = static_cast<float>(w & ~kCPrompt);
          s = z > 0.f ? z / rep : z * rep;
          s -= freq * m;
          s -= m > 0.f ? pres : 0.f;
        }
        if (bi) s += c.bias_values[bi - 1];
        if (fabsf(z) <= FLT_MAX) s = fminf(fmaxf(s, -top), top);
        store1(y + i, s);
      }
    }
    if (k + 1 < p.P && c.drafts) {
      __syncthreads();
      const int v = c.drafts[b * c.drafts_ld + k];
      if (static_cast<unsigned>(v) >= static_cast<unsigned>(p.V)) err |= ASYMSPEC_DATA_BAD_TOKEN;
      else if (tid == 0 && v >= v0 && v < v0 + n) ++cnt[v - v0];
    }
  }
  if (err && p.err) atomicOr(p.err, err);
}

}  // namespace asymspec_impl
