// Host side of the paged cache in 4 bits declared in include/asymspec_serving.h: argument checks and
// launches.
//
//   cache4_write_kernel, cache4_read_kernel  (kernel_cache4.cuh)
//   attend4_split  (kernel_attend4.cuh) attention over it, the keys split evenly over the chip;
//                  attend4_join joins the parts of a request's keys
#include <algorithm>
#include <cfloat>
#include <climits>
#include <cmath>

#include "k_attend.h"
#include "kernel_attend4.cuh"
#include "kernel_cache4.cuh"
#include "serving_host.h"

namespace {

using namespace asymspec_impl;

// CTAs of a read at most: 100,003 tokens 98 us with a token's threads to each, 112 with 1216 (and no fewer with a
// slot looked up a token ahead, 114).  A write takes what an SM has room for on each of 152: 16384 tokens written and
// read of 8 heads of 128 bf16 31.9 us with 760, 32.8 with twice that.
constexpr int kReadCtas = 1 << 20;

AttendKernels attend4_kernels(int dtype, int D, int rows, bool fast) {
  return dtype == ASYMSPEC_FP32 ? attend4_kernels_f32(D, rows) : attend4_kernels_bf16(D, rows, fast);
}

int check_cache4(const asymspec_cache4* c) {
  if (!c || !c->key_codes || !c->key_scales || !c->value_codes || !c->value_scales) return ASYMSPEC_ERR_INVALID_ARG;
  if (c->num_blocks < 1 || c->block_size < 1 || c->kv_heads < 1 || c->head_dim < 1) return ASYMSPEC_ERR_INVALID_ARG;
  if (c->head_dim % 32 != 0 || c->head_dim > ASYMSPEC_CACHE_MAX_D) return ASYMSPEC_ERR_UNSUPPORTED;
  for (const float s : {c->key_scale, c->value_scale})
    if (!(s >= 0x1p-64f && s <= 0x1p64f)) return ASYMSPEC_ERR_INVALID_ARG;
  for (int i = 0; i < 3; ++i) {
    const int64_t codes[2] = {c->key_code_strides[i], c->value_code_strides[i]};
    const int64_t scales[2] = {c->key_scale_strides[i], c->value_scale_strides[i]};
    for (int k = 0; k < 2; ++k) {
      if (codes[k] < 0 || scales[k] < 0) return ASYMSPEC_ERR_INVALID_ARG;
      if (codes[k] % 16 != 0 || scales[k] % 2 != 0) return ASYMSPEC_ERR_MISALIGNED;
    }
  }
  if (!aligned(c->key_codes, 16) || !aligned(c->value_codes, 16) || !aligned(c->key_scales, 2) ||
      !aligned(c->value_scales, 2))
    return ASYMSPEC_ERR_MISALIGNED;
  if (static_cast<int64_t>(c->num_blocks) * c->block_size > kMax32 || c->kv_heads > 65536) return ASYMSPEC_ERR_TOO_LARGE;
  return ASYMSPEC_OK;
}

template <typename T, bool WIDE>
const void* write_pick(int* most_ctas) {
  *most_ctas = cache4_write_ctas<T, WIDE>() * kASms;
  return reinterpret_cast<const void*>(&cache4_write_kernel<T, WIDE>);
}

// What a write and a read have in common.
int move(const asymspec_cache4* c, const void* k, const void* v, int dtype, const int64_t* k_strides,
         const int64_t* v_strides, const int64_t* slots, int T, uint32_t* err, bool read, void* stream) {
  const int st = check_cache4(c);
  if (st != ASYMSPEC_OK) return st;
  if (!known_dtype(dtype)) return ASYMSPEC_ERR_UNSUPPORTED;
  if (T < 0 || !k_strides || !v_strides) return ASYMSPEC_ERR_INVALID_ARG;
  const int extents[2] = {T, c->kv_heads};
  for (int i = 0; i < 2; ++i) {
    if (k_strides[i] < 0 || v_strides[i] < 0) return ASYMSPEC_ERR_INVALID_ARG;
    if (read && extents[i] > 1 && (k_strides[i] == 0 || v_strides[i] == 0)) return ASYMSPEC_ERR_INVALID_ARG;
  }
  if (T == 0) return ASYMSPEC_OK;
  if (!k || !v || !slots || (read && k == v)) return ASYMSPEC_ERR_INVALID_ARG;
  const int elt = elt_size(dtype), per = 32 / elt;
  if (!aligned(k, elt) || !aligned(v, elt) || !aligned(slots, 8) || !aligned(err, 4)) return ASYMSPEC_ERR_MISALIGNED;
  bool wide = aligned(k, 32) && aligned(v, 32);
  for (int i = 0; i < 2; ++i) wide = wide && k_strides[i] % per == 0 && v_strides[i] % per == 0;
  Cache4Params p = {};
  p.part[0] = {static_cast<char*>(c->key_codes), static_cast<char*>(c->key_scales)};
  p.part[1] = {static_cast<char*>(c->value_codes), static_cast<char*>(c->value_scales)};
  for (int i = 0; i < 3; ++i) {
    p.part[0].cs[i] = c->key_code_strides[i], p.part[0].ss[i] = c->key_scale_strides[i];
    p.part[1].cs[i] = c->value_code_strides[i], p.part[1].ss[i] = c->value_scale_strides[i];
  }
  p.part[0].scale = c->key_scale, p.part[1].scale = c->value_scale;
  for (Cache4Part& part : p.part) part.to_units = static_cast<float>(1.0 / (6.0 * static_cast<double>(part.scale)));
  p.x[0] = const_cast<void*>(k), p.x[1] = const_cast<void*>(v);
  for (int i = 0; i < 2; ++i) p.xs[0][i] = k_strides[i], p.xs[1][i] = v_strides[i];
  p.slots = slots;
  p.T = T;
  p.num_blocks = c->num_blocks;
  p.block_size = c->block_size;
  p.kv_heads = c->kv_heads;
  p.pairs = c->head_dim / 32;
  p.per_token = 2 * c->kv_heads * p.pairs;
  while ((1 << p.log_lanes) < std::min(p.per_token, k4Threads)) ++p.log_lanes;
  p.err = err;
  using B = __nv_bfloat16;
  const void* fn;
  int most = kReadCtas;
  if (read)
    fn = elt == 4 ? (wide ? reinterpret_cast<const void*>(&cache4_read_kernel<float, true>)
                          : reinterpret_cast<const void*>(&cache4_read_kernel<float, false>))
                  : (wide ? reinterpret_cast<const void*>(&cache4_read_kernel<B, true>)
                          : reinterpret_cast<const void*>(&cache4_read_kernel<B, false>));
  else if (elt == 4)
    fn = wide ? write_pick<float, true>(&most) : write_pick<float, false>(&most);
  else
    fn = wide ? write_pick<B, true>(&most) : write_pick<B, false>(&most);
  const int64_t ctas = (static_cast<int64_t>(T) + (k4Threads >> p.log_lanes) - 1) / (k4Threads >> p.log_lanes);
  return launch(fn, dim3(static_cast<unsigned>(std::min<int64_t>(ctas, most))), dim3(k4Threads), 0, &p, stream);
}

}  // namespace

extern "C" {

int asymspec_cache4_write(const asymspec_cache4* cache, const void* k, const void* v, int dtype,
                          const int64_t* k_strides, const int64_t* v_strides, const int64_t* slots, int T,
                          uint32_t* out_error_word, void* stream) {
  return move(cache, k, v, dtype, k_strides, v_strides, slots, T, out_error_word, false, stream);
}

int asymspec_cache4_read(const asymspec_cache4* cache, const int64_t* slots, int T, void* k, void* v, int dtype,
                         const int64_t* k_strides, const int64_t* v_strides, uint32_t* out_error_word,
                         void* stream) {
  return move(cache, k, v, dtype, k_strides, v_strides, slots, T, out_error_word, true, stream);
}

size_t asymspec_cache4_attend_workspace_bytes(int B, int Q, int heads, int kv_heads, int head_dim) {
  if (B < 1 || Q < 1 || heads < 1 || kv_heads < 1 || head_dim < 1 || heads % kv_heads != 0 || head_dim % 32 != 0 ||
      head_dim > ASYMSPEC_CACHE_MAX_D || B > ASYMSPEC_CACHE_MAX_B || static_cast<int64_t>(Q) * heads > (1 << 20))
    return 0;
  // any number of queries up to Q: fewer rows may have more CTAs
  size_t most = 0;
  const int rows = Q * (heads / kv_heads);
  for (const int r : {rows, 32, 16, 8}) {
    if (r > rows) continue;
    for (const AttendKernels& k : {attend4_kernels_bf16(head_dim, r, true), attend4_kernels_f32(head_dim, r)})
      most = std::max(most, attend_ws_bytes(k.rows, k.DP, k.most_ctas));
  }
  return most;
}

int asymspec_cache4_attend(const asymspec_cache4* cache, const void* q, int dtype, const int64_t* q_strides,
                           int B, int Q, int heads, const int32_t* block_tables, int64_t table_ld,
                           int table_width, const int32_t* lens, float scale, int window, void* out,
                           const int64_t* out_strides, float* out_lse, void* workspace,
                           size_t workspace_bytes, uint32_t* out_error_word, void* stream) {
  const int st = check_cache4(cache);
  if (st != ASYMSPEC_OK) return st;
  if (!known_dtype(dtype)) return ASYMSPEC_ERR_UNSUPPORTED;
  if (B < 0 || Q < 0 || heads < 1 || heads % cache->kv_heads != 0 || table_width < 1 || table_ld < table_width ||
      !(std::fabs(scale) <= FLT_MAX) || window < 0 || !q_strides || !out_strides)
    return ASYMSPEC_ERR_INVALID_ARG;
  const int extents[3] = {B, Q, heads};
  for (int i = 0; i < 3; ++i)
    if (q_strides[i] < 0 || out_strides[i] < 0 || (out_strides[i] == 0 && extents[i] > 1)) return ASYMSPEC_ERR_INVALID_ARG;
  if (B > ASYMSPEC_CACHE_MAX_B || static_cast<int64_t>(Q) * heads > (1 << 20) ||
      static_cast<int64_t>(table_width) * cache->block_size > (1 << 30))
    return ASYMSPEC_ERR_TOO_LARGE;
  if (B == 0 || Q == 0) return ASYMSPEC_OK;
  if (!q || !block_tables || !lens || !out) return ASYMSPEC_ERR_INVALID_ARG;
  const int elt = elt_size(dtype);
  if (!aligned(q, elt) || !aligned(out, elt) || !aligned(block_tables, 4) || !aligned(lens, 4) ||
      !aligned(out_lse, 4) || !aligned(out_error_word, 4))
    return ASYMSPEC_ERR_MISALIGNED;
  const size_t need = asymspec_cache4_attend_workspace_bytes(B, Q, heads, cache->kv_heads, cache->head_dim);
  if (!workspace || !aligned(workspace, 256) || workspace_bytes < need) return ASYMSPEC_ERR_WORKSPACE;
  if (q == out) return ASYMSPEC_ERR_INVALID_ARG;  // (one CTA of a request may read what another has written)
  const double scale2 = static_cast<double>(scale) * cache->key_scale * 1.4426950408889634;
  if (!(std::fabs(scale2) <= FLT_MAX)) return ASYMSPEC_ERR_INVALID_ARG;
  Attend4Params P = {};
  AttendParams& p = P.a;
  p.q = q;
  p.out = out;
  p.lse = out_lse;
  for (int i = 0; i < 3; ++i) p.qs[i] = q_strides[i], p.os[i] = out_strides[i];
  p.tables = block_tables;
  p.lens = lens;
  p.table_ld = table_ld;
  p.B = B;
  p.Q = Q;
  p.heads = heads;
  p.kv_heads = cache->kv_heads;
  p.D = cache->head_dim;
  p.num_blocks = cache->num_blocks;
  p.block_size = cache->block_size;
  p.table_width = table_width;
  p.window = attend_window(window, table_width, cache->block_size);
  p.group = heads / cache->kv_heads;
  p.rows = Q * p.group;
  AttendKernels k = attend4_kernels(dtype, p.D, p.rows, true);
  p.row_tiles = (p.rows + k.rows - 1) / k.rows;
  p.scale2 = static_cast<float>(scale2);
  p.out_vec = aligned(out, 4 * elt);
  for (int i = 0; i < 3; ++i) p.out_vec = p.out_vec && out_strides[i] % 4 == 0;
  p.ws = static_cast<char*>(workspace);
  p.err = out_error_word;
  P.codes[0] = static_cast<const char*>(cache->key_codes), P.codes[1] = static_cast<const char*>(cache->value_codes);
  P.scales[0] = static_cast<const char*>(cache->key_scales), P.scales[1] = static_cast<const char*>(cache->value_scales);
  const int64_t* codes[2] = {cache->key_code_strides, cache->value_code_strides};
  const int64_t* scales[2] = {cache->key_scale_strides, cache->value_scale_strides};
  const size_t scale_row = k.DP / 16;
  P.wide_scales = P.wide_codes = p.D == k.DP;
  for (int w = 0; w < 2; ++w) {
    P.head_codes[w] = codes[w][2], P.head_scales[w] = scales[w][2];
    for (int i = 0; i < 2; ++i) {
      if (codes[w][i] > kMax32 || scales[w][i] > kMax32) return ASYMSPEC_ERR_TOO_LARGE;
      P.codes_of[w][i] = static_cast<unsigned>(codes[w][i]), P.scales_of[w][i] = static_cast<unsigned>(scales[w][i]);
    }
    P.wide_scales = P.wide_scales && aligned(P.scales[w], scale_row);
    P.wide_codes = P.wide_codes && aligned(P.codes[w], 32);
    for (int i = 0; i < 3; ++i) {
      P.wide_scales = P.wide_scales && scales[w][i] % static_cast<int64_t>(scale_row) == 0;
      P.wide_codes = P.wide_codes && codes[w][i] % 32 == 0;
    }
  }
  divide_by(p.block_size, &P.divide, &P.shift);
  divide_by(p.group, &P.divide_rows, &P.shift_rows);
  if (!P.wide_scales || !P.wide_codes) k = attend4_kernels(dtype, p.D, p.rows, false);
  P.value_scale = cache->value_scale;
  int device = 0, sms = 0;
  cudaError_t e = device_sms(&device, &sms);
  if (e == cudaSuccess) e = prepare(k.split, device, k.smem);
  if (e != cudaSuccess) return cuda_fail(e);
  // as many CTAs as fit on the chip, but no more than there may be units of work (see attend_tiles)
  const int64_t most = static_cast<int64_t>(table_width) * p.block_size / k.tile + 1 + kAItem;
  int ctas = static_cast<int>(std::min<int64_t>(std::min(k.most_ctas, sms * k.ctas_per_sm), B * most * p.kv_heads * p.row_tiles));
  const cudaStream_t st_ = static_cast<cudaStream_t>(stream);
  void* args[] = {&P};
  e = cudaLaunchKernel(k.split, dim3(ctas), dim3(k.threads), args, k.smem, st_);
  if (e != cudaSuccess) return cuda_fail(e);
  if (ctas == 1) return ASYMSPEC_OK;
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  const int join_rows = std::min(p.rows, k.rows);
  cfg.gridDim = join_rows <= 16 ? dim3(ctas - 1, join_rows) : dim3(std::min(4 * sms, (ctas - 1) * join_rows));
  cfg.blockDim = dim3(kAJoinThreads);
  cfg.stream = st_;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  void* join_args[] = {&p, &ctas};
  e = cudaLaunchKernelExC(&cfg, k.join, join_args);
  return e == cudaSuccess ? ASYMSPEC_OK : cuda_fail(e);
}

}  // extern "C"
