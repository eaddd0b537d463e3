// Host side of the C ABI declared in include/asymspec_serving.h: argument checks and
// launches of the operators around the verification step.
//
//   constrain_rows      (kernel_constrain.cuh) penalties, biases and masks on logits;
//                       constrain_in_place where they are (no masks)
//   cache_plan_kernel   (kernel_cache.cuh) block tables and slot maps
//   cache_write_kernel  (kernel_cache.cuh) new keys and values into the cache
//   attend_split        (kernel_attend.cuh) attention over the cache, the keys split evenly
//                       over the chip; attend_join joins the parts of a request's keys
#include <algorithm>
#include <climits>
#include <cmath>

#include "host_common.h"
#include "k_attend.h"
#include "kernel_attend.cuh"
#include "kernel_cache.cuh"
#include "kernel_constrain.cuh"
#include "serving_host.h"

namespace {

using namespace asymspec_impl;

constexpr int kWriteCtas = 1216;  // CTAs of the write at most: eight on each SM

// Slots above which the plan takes a cluster: two goes of one CTA (512 slots: 4.9 us, 7.1 in a
// cluster; 115,000: 17.3 in a cluster, 120 in one CTA).
constexpr int kPlanTokens = 2048;

// A CTA's slice of the vocabulary in 16-byte vectors, and the vectors that a thread has at
// least, of one row or of several.  us, kVectors = 256 / 512: 64x8 bf16 50.6 / 52.6, 32x9 with
// histories to 65536 51.3 / 56.5; kThreadVectors = 1 / 2 / 4 / 8: 64x1 29.6 / 17.9 / 15.0 / 16.4.
constexpr int kVectors = 256;
constexpr int kThreadVectors = 4;

// Where histories may be this long, the grid's last CTAs, those that are resident together at its
// end, take the requests with the longest histories first, so that none of those begins last.
// us, in the grid's order / with the last CTAs ordered / with all (each waits for the lengths then):
// 32x9 with histories to 8192 35.0 / 34.7 / 38.0, 32768 40.1 / 38.5 / 39.6, 65536 48.2 / 44.9 / 42.9;
// 64x8 to 8192 47.8 / 48.7 / 53.9, 16384 49.8 / 49.9 / 55.5, 32768 53.7 / 51.4 / 57.0.  (The host knows
// how long they may be, not how long they are: short ones with room for long ones pay those 2 %.)
constexpr int kOrderWidth = 16384;
constexpr int kOrderCtas = 4;  // on an SM
template <typename T>
const void* constrain_pick(bool in_place, bool edges) {
  if (in_place) return reinterpret_cast<const void*>(&constrain_in_place<T>);
  return edges ? reinterpret_cast<const void*>(&constrain_rows<T, true>)
               : reinterpret_cast<const void*>(&constrain_rows<T, false>);
}

AttendKernels attend_kernels(int dtype, int D, int rows) {
  return dtype == ASYMSPEC_FP32 ? attend_kernels_f32(D, rows) : attend_kernels_bf16(D, rows);
}

int check_constraints(const asymspec_constraints& c, int B, int P, int V) {
  if (c.history && (!c.history_len || c.history_ld < 0 || c.history_width < 0))
    return ASYMSPEC_ERR_INVALID_ARG;
  if (!c.history && (c.history_len || c.prompt_len)) return ASYMSPEC_ERR_INVALID_ARG;
  if (c.drafts && c.drafts_ld < 0) return ASYMSPEC_ERR_INVALID_ARG;
  if (c.bias_offsets && (c.bias_count < 0 || (c.bias_count > 0 && (!c.bias_tokens || !c.bias_values))))
    return ASYMSPEC_ERR_INVALID_ARG;
  if (!c.bias_offsets && (c.bias_tokens || c.bias_values)) return ASYMSPEC_ERR_INVALID_ARG;
  if (c.mask) {
    if (c.mask_count < 0 || c.mask_ld * 32 < V || !(std::fabs(c.mask_value) <= FLT_MAX))
      return ASYMSPEC_ERR_INVALID_ARG;
    if (!c.mask_rows && c.mask_count < static_cast<int64_t>(B) * P) return ASYMSPEC_ERR_INVALID_ARG;
  } else if (c.mask_rows) {
    return ASYMSPEC_ERR_INVALID_ARG;
  }
  for (const void* q : {static_cast<const void*>(c.history), static_cast<const void*>(c.history_len),
                        static_cast<const void*>(c.prompt_len), static_cast<const void*>(c.drafts),
                        static_cast<const void*>(c.repetition), static_cast<const void*>(c.frequency),
                        static_cast<const void*>(c.presence), static_cast<const void*>(c.bias_offsets),
                        static_cast<const void*>(c.bias_tokens), static_cast<const void*>(c.bias_values),
                        static_cast<const void*>(c.mask), static_cast<const void*>(c.mask_rows)})
    if (!aligned(q, 4)) return ASYMSPEC_ERR_MISALIGNED;
  return ASYMSPEC_OK;
}

int check_cache(const asymspec_cache* c) {
  if (!c || !c->keys || !c->values) return ASYMSPEC_ERR_INVALID_ARG;
  if (!known_dtype(c->dtype)) return ASYMSPEC_ERR_UNSUPPORTED;
  if (c->num_blocks < 1 || c->block_size < 1 || c->kv_heads < 1 || c->head_dim < 1)
    return ASYMSPEC_ERR_INVALID_ARG;
  for (int i = 0; i < 3; ++i)
    if (c->key_strides[i] < 0 || c->value_strides[i] < 0) return ASYMSPEC_ERR_INVALID_ARG;
  if (static_cast<int64_t>(c->num_blocks) * c->block_size > kMax32 ||
      static_cast<int64_t>(c->kv_heads) * c->head_dim > kMax32)
    return ASYMSPEC_ERR_TOO_LARGE;
  const int elt = elt_size(c->dtype);
  if (!aligned(c->keys, elt) || !aligned(c->values, elt)) return ASYMSPEC_ERR_MISALIGNED;
  return ASYMSPEC_OK;
}

}  // namespace

extern "C" {

int asymspec_constrain_logits(const asymspec_constraints* c, const void* logits, int64_t ld,
                              void* out, int64_t out_ld, int B, int P, int V, int dtype,
                              uint32_t* out_error_word, void* stream) {
  if (!known_dtype(dtype)) return ASYMSPEC_ERR_UNSUPPORTED;
  if (!c || B < 0 || P < 0 || V < 2 || ld < V || out_ld < V) return ASYMSPEC_ERR_INVALID_ARG;
  if (P > ASYMSPEC_CONSTRAIN_MAX_P || B > 65535 || V > (1 << 25)) return ASYMSPEC_ERR_TOO_LARGE;
  const int st = check_constraints(*c, B, P, V);
  if (st != ASYMSPEC_OK) return st;
  if (B == 0 || P == 0) return ASYMSPEC_OK;
  if (!logits || !out || (logits == out && ld != out_ld)) return ASYMSPEC_ERR_INVALID_ARG;
  const int elt = elt_size(dtype);
  if (!aligned(logits, elt) || !aligned(out, elt) || !aligned(out_error_word, 4))
    return ASYMSPEC_ERR_MISALIGNED;
  CParams p = {*c, logits, out, ld, out_ld, B, P, V, 0, P, 0, INT_MAX, 0, out_error_word};
  int device = 0, sms = 0;
  cudaError_t e = device_sms(&device, &sms);
  if (e != cudaSuccess) return cuda_fail(e);
  const int per = 16 / elt;
  const bool edges = !aligned(logits, 16) || !aligned(out, 16) || ld % per != 0 || out_ld % per != 0 || V % per != 0;
  // a slice: more of the vocabulary where there are few rows
  int vectors = kVectors;
  for (int rows = P; rows < kThreadVectors && vectors < 1024; rows *= 2) vectors *= 2;
  p.W = vectors * per;
  const int64_t slices = (V + p.W - 1) / p.W;
  // enough CTAs for the chip: fewer rows each
  while (p.group_rows > 1 && slices * B * ((P + p.group_rows - 1) / p.group_rows) < 2 * sms)
    p.group_rows = (p.group_rows + 1) / 2;
  const int groups = (P + p.group_rows - 1) / p.group_rows;
  // batches of one size, kCSlots vectors of a thread at most
  const int most = kCSlots * kCThreads / vectors, batches = (p.group_rows + most - 1) / most;
  p.batch_rows = (p.group_rows + batches - 1) / batches;
  const bool in_place = logits == out && !c->mask;
  const size_t smem = constrain_list_bytes(p.W) +
                      (in_place ? 0 : static_cast<size_t>(p.batch_rows) * constrain_pitch(p.W, elt));
  const void* fn = dtype == ASYMSPEC_FP32 ? constrain_pick<float>(in_place, edges)
                                          : constrain_pick<__nv_bfloat16>(in_place, edges);
  e = prepare(fn, device, static_cast<int>(smem));
  if (e != cudaSuccess) return cuda_fail(e);
  if (c->history && c->history_width >= kOrderWidth && B > 1 && B <= kCOrdered) {
    p.ordered_from = static_cast<int>(std::max<int64_t>(slices - (kOrderCtas * sms + B - 1) / B, 0));
    while (c->history_width >> kCStepBits >> p.length_bits) ++p.length_bits;
  }
  void* args[] = {&p};
  e = cudaLaunchKernel(fn, dim3(B, static_cast<unsigned>(slices), groups), dim3(kCThreads), args, smem,
                       static_cast<cudaStream_t>(stream));
  return e == cudaSuccess ? ASYMSPEC_OK : cuda_fail(e);
}

int asymspec_cache_plan(const int32_t* lens, const int32_t* accepted, const int32_t* grow,
                        int grow_all, int B, int block_size, int num_blocks,
                        int32_t* block_tables, int64_t table_ld, int table_width,
                        const int32_t* held, int32_t* free_list, const int32_t* free_count,
                        int32_t* out_start, int32_t* out_len, int32_t* out_held,
                        int32_t* out_free_count, int32_t* out_offsets, int64_t* out_slots,
                        int32_t* out_positions, int64_t capacity, uint32_t* out_error_word,
                        void* stream) {
  if (B < 0 || block_size < 1 || num_blocks < 1 || table_width < 1 || table_ld < table_width ||
      capacity < 0 || (!grow && grow_all < 0))
    return ASYMSPEC_ERR_INVALID_ARG;
  if (B > ASYMSPEC_CACHE_MAX_B || static_cast<int64_t>(B) * table_width > kMax32 ||
      static_cast<int64_t>(num_blocks) * block_size > kMax32 ||
      static_cast<int64_t>(table_width) * block_size > kMax32 || capacity > kMax32)
    return ASYMSPEC_ERR_TOO_LARGE;
  if (!free_list || !free_count || !out_free_count || !out_offsets || (capacity > 0 && !out_slots) ||
      (B > 0 && (!lens || !held || !block_tables || !out_start || !out_len || !out_held)))
    return ASYMSPEC_ERR_INVALID_ARG;
  for (const void* q : {static_cast<const void*>(lens), static_cast<const void*>(accepted),
                        static_cast<const void*>(grow), static_cast<const void*>(block_tables),
                        static_cast<const void*>(held), static_cast<const void*>(free_list),
                        static_cast<const void*>(free_count), static_cast<const void*>(out_start),
                        static_cast<const void*>(out_len), static_cast<const void*>(out_held),
                        static_cast<const void*>(out_free_count), static_cast<const void*>(out_offsets),
                        static_cast<const void*>(out_positions), static_cast<const void*>(out_error_word)})
    if (!aligned(q, 4)) return ASYMSPEC_ERR_MISALIGNED;
  if (!aligned(out_slots, 8)) return ASYMSPEC_ERR_MISALIGNED;
  PlanParams p = {lens, accepted, grow, held, free_count, grow_all, B, block_size, num_blocks,
                  table_width, block_tables, free_list, table_ld, out_start, out_len, out_held,
                  out_free_count, out_offsets, out_positions, out_slots, capacity, out_error_word};
  // a cluster where there is more than a CTA does in one or two goes
  const bool clusters = capacity > kPlanTokens;
  const void* fn = clusters ? reinterpret_cast<const void*>(&cache_plan_kernel<true>)
                            : reinterpret_cast<const void*>(&cache_plan_kernel<false>);
  const size_t smem = plan_smem_bytes(B);
  int device = 0;
  cudaError_t e = cudaSuccess;
  if (smem > 48 * 1024 - kStaticSmem) e = cudaGetDevice(&device);
  if (e == cudaSuccess) e = prepare(fn, device, static_cast<int>(smem));
  if (e != cudaSuccess) return cuda_fail(e);
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = kPCluster;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.gridDim = dim3(clusters ? kPCluster : 1);
  cfg.blockDim = dim3(kPThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = static_cast<cudaStream_t>(stream);
  cfg.attrs = attr;
  cfg.numAttrs = clusters ? 1 : 0;
  void* args[] = {&p};
  e = cudaLaunchKernelExC(&cfg, fn, args);
  return e == cudaSuccess ? ASYMSPEC_OK : cuda_fail(e);
}

int asymspec_cache_write(const asymspec_cache* cache, const void* k, const void* v,
                         const int64_t* k_strides, const int64_t* v_strides, const int64_t* slots,
                         int T, uint32_t* out_error_word, void* stream) {
  const int st = check_cache(cache);
  if (st != ASYMSPEC_OK) return st;
  if (T < 0 || !k_strides || !v_strides) return ASYMSPEC_ERR_INVALID_ARG;
  for (int i = 0; i < 2; ++i)
    if (k_strides[i] < 0 || v_strides[i] < 0) return ASYMSPEC_ERR_INVALID_ARG;
  if (T == 0) return ASYMSPEC_OK;
  if (!k || !v || !slots) return ASYMSPEC_ERR_INVALID_ARG;
  const int elt = elt_size(cache->dtype);
  if (!aligned(k, elt) || !aligned(v, elt) || !aligned(slots, 8) || !aligned(out_error_word, 4))
    return ASYMSPEC_ERR_MISALIGNED;
  const int per = 16 / elt;
  bool wide = aligned(k, 16) && aligned(v, 16) && aligned(cache->keys, 16) &&
              aligned(cache->values, 16) && cache->head_dim % per == 0;
  for (int i = 0; i < 3; ++i)
    wide = wide && cache->key_strides[i] % per == 0 && cache->value_strides[i] % per == 0;
  for (int i = 0; i < 2; ++i) wide = wide && k_strides[i] % per == 0 && v_strides[i] % per == 0;
  const int u = wide ? per : 1;
  WriteParams p = {};
  p.k = k;
  p.v = v;
  p.keys = cache->keys;
  p.values = cache->values;
  for (int i = 0; i < 2; ++i) p.ks[i] = k_strides[i] / u, p.vs[i] = v_strides[i] / u;
  for (int i = 0; i < 3; ++i)
    p.cks[i] = cache->key_strides[i] / u, p.cvs[i] = cache->value_strides[i] / u;
  p.slots = slots;
  p.T = T;
  p.num_blocks = cache->num_blocks;
  p.block_size = cache->block_size;
  p.kv_heads = cache->kv_heads;
  p.head_dim = cache->head_dim / u;
  p.err = out_error_word;
  const int per_token = p.kv_heads * p.head_dim;
  while (p.log_lanes < 5 && (1 << p.log_lanes) < per_token) ++p.log_lanes;
  const int64_t ctas = (static_cast<int64_t>(T) + (kWThreads >> p.log_lanes) - 1) / (kWThreads >> p.log_lanes);
  const void* fn = wide ? reinterpret_cast<const void*>(&cache_write_kernel<uint4>)
                   : elt == 4 ? reinterpret_cast<const void*>(&cache_write_kernel<uint32_t>)
                              : reinterpret_cast<const void*>(&cache_write_kernel<uint16_t>);
  return launch(fn, dim3(static_cast<unsigned>(std::min<int64_t>(ctas, kWriteCtas))), dim3(kWThreads), 0, &p,
                stream);
}

size_t asymspec_cache_attend_workspace_bytes(int B, int Q, int heads, int kv_heads, int head_dim) {
  if (B < 1 || Q < 1 || heads < 1 || kv_heads < 1 || head_dim < 1 || heads % kv_heads != 0 ||
      head_dim > ASYMSPEC_CACHE_MAX_D || B > ASYMSPEC_CACHE_MAX_B ||
      static_cast<int64_t>(Q) * heads > (1 << 20))
    return 0;
  const int rows = Q * (heads / kv_heads);
  const AttendKernels a = attend_kernels_bf16(head_dim, rows), b = attend_kernels_f32(head_dim, rows);
  return std::max(attend_ws_bytes(a.rows, a.DP, a.most_ctas), attend_ws_bytes(b.rows, b.DP, b.most_ctas));
}

int asymspec_cache_attend(const asymspec_cache* cache, const void* q, const int64_t* q_strides,
                          int B, int Q, int heads, const int32_t* block_tables, int64_t table_ld,
                          int table_width, const int32_t* lens, float scale, int window, void* out,
                          const int64_t* out_strides, float* out_lse, void* workspace,
                          size_t workspace_bytes, uint32_t* out_error_word, void* stream) {
  const int st = check_cache(cache);
  if (st != ASYMSPEC_OK) return st;
  if (cache->head_dim > ASYMSPEC_CACHE_MAX_D) return ASYMSPEC_ERR_UNSUPPORTED;
  if (B < 0 || Q < 0 || heads < 1 || heads % cache->kv_heads != 0 || table_width < 1 ||
      table_ld < table_width || !(std::fabs(scale) <= FLT_MAX) || window < 0 || !q_strides || !out_strides)
    return ASYMSPEC_ERR_INVALID_ARG;
  for (int i = 0; i < 3; ++i)
    if (q_strides[i] < 0 || out_strides[i] < 0) return ASYMSPEC_ERR_INVALID_ARG;
  const int extents[3] = {B, Q, heads};
  for (int i = 0; i < 3; ++i)
    if (out_strides[i] == 0 && extents[i] > 1) return ASYMSPEC_ERR_INVALID_ARG;
  if (B > ASYMSPEC_CACHE_MAX_B || static_cast<int64_t>(Q) * heads > (1 << 20) ||
      static_cast<int64_t>(table_width) * cache->block_size > (1 << 30))
    return ASYMSPEC_ERR_TOO_LARGE;
  if (B == 0 || Q == 0) return ASYMSPEC_OK;
  if (!q || !block_tables || !lens || !out) return ASYMSPEC_ERR_INVALID_ARG;
  const int elt = elt_size(cache->dtype), per = 16 / elt;
  if (!aligned(q, elt) || !aligned(out, elt) || !aligned(block_tables, 4) || !aligned(lens, 4) ||
      !aligned(out_lse, 4) || !aligned(out_error_word, 4) || !aligned(cache->keys, 16) ||
      !aligned(cache->values, 16) || cache->head_dim % per != 0)
    return ASYMSPEC_ERR_MISALIGNED;
  for (int i = 0; i < 3; ++i)
    if (cache->key_strides[i] % per != 0 || cache->value_strides[i] % per != 0)
      return ASYMSPEC_ERR_MISALIGNED;
  const size_t need =
      asymspec_cache_attend_workspace_bytes(B, Q, heads, cache->kv_heads, cache->head_dim);
  if (!workspace || !aligned(workspace, 256) || workspace_bytes < need) return ASYMSPEC_ERR_WORKSPACE;
  if (q == out) return ASYMSPEC_ERR_INVALID_ARG;  // (one CTA of a request may read what another has written)
  AttendParams p = {};
  p.keys = cache->keys;
  p.values = cache->values;
  p.q = q;
  p.out = out;
  p.lse = out_lse;
  for (int i = 0; i < 3; ++i) {
    p.cks[i] = cache->key_strides[i];
    p.cvs[i] = cache->value_strides[i];
    p.qs[i] = q_strides[i];
    p.os[i] = out_strides[i];
  }
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
  const AttendKernels k = attend_kernels(cache->dtype, p.D, p.rows);
  p.row_tiles = (p.rows + k.rows - 1) / k.rows;
  p.scale2 = scale * kLog2e;
  p.q_vec = aligned(q, 16);
  p.out_vec = aligned(out, 4 * elt);
  for (int i = 0; i < 3; ++i) {
    p.q_vec = p.q_vec && q_strides[i] % per == 0;
    p.out_vec = p.out_vec && out_strides[i] % 4 == 0;
  }
  p.whole_steps = cache->block_size % kAKeys == 0;
  for (int i = 0; i < 2; ++i) {
    const int64_t* strides = i == 0 ? cache->key_strides : cache->value_strides;
    p.whole_steps = p.whole_steps && strides[0] * elt <= kMax32 && strides[1] * elt * kAKeys <= kMax32;
    p.block_bytes[i] = static_cast<int>(strides[0] * elt);
    p.token_bytes[i] = static_cast<int>(strides[1] * elt);
  }
  p.ws = static_cast<char*>(workspace);
  p.err = out_error_word;
  int device = 0, sms = 0;
  cudaError_t e = device_sms(&device, &sms);
  if (e == cudaSuccess) e = prepare(k.split, device, k.smem);
  if (e != cudaSuccess) return cuda_fail(e);
  int ctas = std::min(kAMaxCtas, sms * k.ctas_per_sm);
  const cudaStream_t st_ = static_cast<cudaStream_t>(stream);
  void* args[] = {&p, &ctas};
  e = cudaLaunchKernel(k.split, dim3(ctas), dim3(k.threads), args, k.smem, st_);
  if (e != cudaSuccess) return cuda_fail(e);
  if (ctas == 1) return ASYMSPEC_OK;
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.gridDim = dim3(ctas - 1, std::min(p.rows, k.rows));
  cfg.blockDim = dim3(kAJoinThreads);
  cfg.stream = st_;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  e = cudaLaunchKernelExC(&cfg, k.join, args);
  return e == cudaSuccess ? ASYMSPEC_OK : cuda_fail(e);
}

}  // extern "C"
