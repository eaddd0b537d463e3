// Host side of the rotary positions declared in include/asymspec_serving.h.
#include <algorithm>
#include <cfloat>
#include <cmath>

#include "kernel_rotary.cuh"
#include "serving_host.h"

namespace {

using namespace asymspec_impl;

constexpr double kTurn = 6.283185307179586476925;

// Units of a CTA: what its threads have on their way at once.
constexpr int kRUnits = kRThreads * kRBatch;

const void* rotary_pick(int dtype, bool wide, bool inter) {
  if (dtype == ASYMSPEC_FP32) {
    if (wide) return inter ? reinterpret_cast<const void*>(&rotary_kernel<float, uint4, true>)
                           : reinterpret_cast<const void*>(&rotary_kernel<float, uint4, false>);
    return inter ? reinterpret_cast<const void*>(&rotary_kernel<float, float, true>)
                 : reinterpret_cast<const void*>(&rotary_kernel<float, float, false>);
  }
  using B = __nv_bfloat16;
  if (wide) return inter ? reinterpret_cast<const void*>(&rotary_kernel<B, uint4, true>)
                         : reinterpret_cast<const void*>(&rotary_kernel<B, uint4, false>);
  return inter ? reinterpret_cast<const void*>(&rotary_kernel<B, uint16_t, true>)
               : reinterpret_cast<const void*>(&rotary_kernel<B, uint16_t, false>);
}

// The pair that turns `turns` times within `length` positions.
double pair_of(double turns, int length, int rotary_dim, double base) {
  return rotary_dim * std::log(length / (turns * kTurn)) / (2 * std::log(base));
}

}  // namespace

extern "C" {

int asymspec_rotary_steps(int rotary_dim, double base, const asymspec_rotary_scaling* scaling,
                          const double* frequencies, uint64_t* out_steps, float* out_magnitude) {
  if (!out_steps || !out_magnitude || rotary_dim < 2 || rotary_dim % 2 != 0) return ASYMSPEC_ERR_INVALID_ARG;
  const int kind = scaling ? scaling->kind : ASYMSPEC_ROTARY_NONE;
  if (frequencies ? kind != ASYMSPEC_ROTARY_NONE : !(base > 1.0 && base <= DBL_MAX)) return ASYMSPEC_ERR_INVALID_ARG;
  if (kind < ASYMSPEC_ROTARY_NONE || kind > ASYMSPEC_ROTARY_WAVELENGTH) return ASYMSPEC_ERR_INVALID_ARG;
  const double f = kind == ASYMSPEC_ROTARY_NONE ? 1.0 : scaling->factor;
  if (!(f >= 1.0 && f <= DBL_MAX) || (kind == ASYMSPEC_ROTARY_BASE && rotary_dim < 4)) return ASYMSPEC_ERR_INVALID_ARG;
  const bool parts = kind == ASYMSPEC_ROTARY_RAMP || kind == ASYMSPEC_ROTARY_WAVELENGTH;
  if (parts && (scaling->original_length < 1 || !(scaling->slow > 0.0) || !(scaling->fast > scaling->slow) ||
                !(scaling->fast <= DBL_MAX)))
    return ASYMSPEC_ERR_INVALID_ARG;
  if (frequencies)
    for (int i = 0; i < rotary_dim / 2; ++i)
      if (!(std::fabs(frequencies[i]) <= DBL_MAX)) return ASYMSPEC_ERR_INVALID_ARG;
  if (kind == ASYMSPEC_ROTARY_BASE) {
    base *= std::pow(f, static_cast<double>(rotary_dim) / (rotary_dim - 2));
    if (!(base <= DBL_MAX)) return ASYMSPEC_ERR_INVALID_ARG;
  }
  double first = 0.0, last = 0.0;  // RAMP: the pairs where it begins and ends
  if (kind == ASYMSPEC_ROTARY_RAMP) {
    const int length = scaling->original_length;
    first = std::max(std::floor(pair_of(scaling->fast, length, rotary_dim, base)), 0.0);
    last = std::min(std::ceil(pair_of(scaling->slow, length, rotary_dim, base)), rotary_dim - 1.0);
  }
  for (int i = 0; i < rotary_dim / 2; ++i) {
    double w = frequencies ? frequencies[i] : std::pow(base, -2.0 * i / rotary_dim);
    if (kind == ASYMSPEC_ROTARY_LINEAR) w /= f;
    if (parts) {
      const double r = kind == ASYMSPEC_ROTARY_RAMP
                           ? 1.0 - (i - first) / std::max(last - first, 0.001)
                           : (scaling->original_length * w / kTurn - scaling->slow) / (scaling->fast - scaling->slow);
      const double kept = std::min(std::max(r, 0.0), 1.0);
      w = w / f * (1.0 - kept) + w * kept;
    }
    const double turns = w / kTurn, part = turns - std::floor(turns);
    // (a part that rounds to one whole turn is none)
    out_steps[i] = part < 1.0 ? static_cast<uint64_t>(std::ldexp(part, 64)) : 0;
  }
  *out_magnitude = kind == ASYMSPEC_ROTARY_RAMP && f > 1.0 ? static_cast<float>(0.1 * std::log(f) + 1.0) : 1.0f;
  return ASYMSPEC_OK;
}

int asymspec_rotary(const asymspec_rotary_heads* q, const asymspec_rotary_heads* k, int T, int head_dim,
                    int rotary_dim, int interleaved, int transpose, const int32_t* positions,
                    const uint64_t* steps, float magnitude, int dtype, void* stream) {
  if (!known_dtype(dtype)) return ASYMSPEC_ERR_UNSUPPORTED;
  if (!q || T < 0 || head_dim < 1 || rotary_dim < 2 || rotary_dim % 2 != 0 || rotary_dim > head_dim ||
      !(std::fabs(magnitude) <= FLT_MAX))
    return ASYMSPEC_ERR_INVALID_ARG;
  if (head_dim > ASYMSPEC_ROTARY_MAX_D) return ASYMSPEC_ERR_UNSUPPORTED;
  const asymspec_rotary_heads* both[2] = {q, k};
  for (const asymspec_rotary_heads* x : both) {
    if (!x) continue;
    if (x->heads < 1) return ASYMSPEC_ERR_INVALID_ARG;
    if (x->heads > 65536) return ASYMSPEC_ERR_TOO_LARGE;
    const int extents[2] = {T, x->heads};
    for (int i = 0; i < 2; ++i) {
      if (x->in_strides[i] < 0 || x->out_strides[i] < 0 || (x->out_strides[i] == 0 && extents[i] > 1))
        return ASYMSPEC_ERR_INVALID_ARG;
      if (x->in == x->out && x->in_strides[i] != x->out_strides[i] && extents[i] > 1) return ASYMSPEC_ERR_INVALID_ARG;
    }
  }
  if (T == 0) return ASYMSPEC_OK;
  if (!positions || !steps) return ASYMSPEC_ERR_INVALID_ARG;
  for (const asymspec_rotary_heads* x : both)
    if (x && (!x->in || !x->out)) return ASYMSPEC_ERR_INVALID_ARG;
  // (a swap in place, too: one's outputs would be the other's inputs)
  if (k && (q->out == k->out || q->out == k->in || k->out == q->in)) return ASYMSPEC_ERR_INVALID_ARG;
  const int elt = elt_size(dtype), per = 16 / elt;
  if (!aligned(positions, 4) || !aligned(steps, 8)) return ASYMSPEC_ERR_MISALIGNED;
  bool wide = (interleaved ? rotary_dim : rotary_dim / 2) % per == 0 && head_dim % per == 0;
  for (const asymspec_rotary_heads* x : both) {
    if (!x) continue;
    if (!aligned(x->in, elt) || !aligned(x->out, elt)) return ASYMSPEC_ERR_MISALIGNED;
    wide = wide && aligned(x->in, 16) && aligned(x->out, 16);
    for (int i = 0; i < 2; ++i) wide = wide && x->in_strides[i] % per == 0 && x->out_strides[i] % per == 0;
  }
  RotaryParams p = {};
  p.T = T;
  p.head_dim = head_dim;
  p.rot = rotary_dim;
  p.turning = wide ? rotary_dim / (interleaved ? per : 2 * per) : rotary_dim / 2;
  p.transpose = transpose != 0;
  p.magnitude = magnitude;
  p.positions = positions;
  p.steps = steps;
  int64_t units = 0;
  for (int i = 0; i < 2; ++i) {
    const asymspec_rotary_heads* x = both[i];
    if (!x) continue;
    RotaryHeads& y = p.x[i];
    y.in = x->in;
    y.out = x->out;
    for (int s = 0; s < 2; ++s) y.is[s] = x->in_strides[s], y.os[s] = x->out_strides[s];
    y.heads = x->heads;
    y.units = p.turning + (x->in == x->out ? 0 : (head_dim - rotary_dim) / (wide ? per : 1));
    divide_by(y.units, &y.divide, &y.shift);
    units += static_cast<int64_t>(y.heads) * y.units;
  }
  p.all_units = static_cast<int>(units);  // (2^27 at most)
  divide_by(p.all_units, &p.divide, &p.shift);
  int device = 0, sms = 0;
  const cudaError_t e = device_sms(&device, &sms);
  if (e != cudaSuccess) return cuda_fail(e);
  // a thread's batch of units to a CTA, but first enough CTAs for the chip
  p.tokens = std::max(1, std::min({kRUnits / p.all_units, kRTable / (rotary_dim / 2), kRTokens, T / (2 * sms)}));
  const int64_t tiles = (static_cast<int64_t>(T) + p.tokens - 1) / p.tokens;
  int each = std::min(p.all_units, kRUnits);
  while (each > kRThreads && tiles * ((p.all_units + each - 1) / each) < 2 * sms) each = (each + 1) / 2;
  p.each = p.tokens > 1 ? p.all_units : std::max({each, kRThreads, (p.all_units + 65534) / 65535});
  const unsigned slices = static_cast<unsigned>((p.all_units + p.each - 1) / p.each);
  return launch(rotary_pick(dtype, wide, interleaved != 0), dim3(static_cast<unsigned>(tiles), slices),
                dim3(kRThreads), 0, &p, stream);
}

}  // extern "C"
