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
  int W;           // vocabulary entries of a CTA, a power of two from 1024 on
  int group_rows;  // rows of a CTA (blockIdx.z: which)
  int batch_rows;  // rows that come into shared memory together
  int ordered_from;  // the slice from which on the longest histories come first
  int length_bits;   // of the histories' lengths in steps of 2^kCStepBits
  uint32_t* err;
};

constexpr int kCThreads = 256;
constexpr int kCAhead = 2;     // 16-byte loads of the history that a thread has on their way
constexpr int kCSlots = 12;    // vectors of a thread in a batch of rows at most
constexpr int kCOrdered = 64;  // requests that are taken in the order of their lengths at most: two a lane of a warp
constexpr int kCStepBits = 8;      // in steps of so many tokens (a power of two)
constexpr int kCBiases = 256;  // a slice's bias entries that shared memory holds
constexpr int kCPart = 2 * kCBiases;  // tokens of a part of a slice with more of them: divides every W
// A token's word: in the prompt, among the drafts, biased, and how often in the output.
constexpr unsigned kCPrompt = 1u << 31, kCDraft = 1u << 30, kCBias = 1u << 29, kCCount = kCBias - 1;

// Dynamic shared memory: the words and the list of those that are not zero; then the rows
// of the slice at hand, each with room for the 16-byte boundaries around it.
__host__ __device__ constexpr size_t constrain_list_bytes(int W) { return static_cast<size_t>(W) * 6; }
__host__ __device__ constexpr int constrain_pitch(int W, int elt) { return W * elt + 32; }

__device__ __forceinline__ float type_max(float) { return FLT_MAX; }
__device__ __forceinline__ float type_max(__nv_bfloat16) { return __uint_as_float(0x7F7F0000u); }
__device__ __forceinline__ float from_f32(float y, float) { return y; }
__device__ __forceinline__ __nv_bfloat16 from_f32(float y, __nv_bfloat16) { return __float2bfloat16_rn(y); }

// 16 bytes of consecutive entries off the 16-byte boundaries.
__device__ __forceinline__ uint4 gather16(const float* p) {
  return make_uint4(__float_as_uint(p[0]), __float_as_uint(p[1]), __float_as_uint(p[2]), __float_as_uint(p[3]));
}
__device__ __forceinline__ uint4 gather16(const __nv_bfloat16* q) {
  const uint16_t* p = reinterpret_cast<const uint16_t*>(q);
  return make_uint4(p[0] | static_cast<unsigned>(p[1]) << 16, p[2] | static_cast<unsigned>(p[3]) << 16,
                    p[4] | static_cast<unsigned>(p[5]) << 16, p[6] | static_cast<unsigned>(p[7]) << 16);
}

// The entries whose bit is not set become `low` (a word of the type's entries).
template <typename T>
__device__ __forceinline__ uint4 masked16(uint4 v, unsigned bits, unsigned low) {
  if constexpr (sizeof(T) == 4)
    return make_uint4(bits & 1u ? v.x : low, bits & 2u ? v.y : low, bits & 4u ? v.z : low, bits & 8u ? v.w : low);
  // bf16: a byte permutation a word, its selector from the bits of four entries at once
  // (each bit to a byte of its own; a half's bytes are numbered 4 less in v than in low)
  const unsigned a = 0x76547654u - (((bits & 15u) * 0x204081u) & 0x01010101u) * 0x44u;
  const unsigned b = 0x76547654u - (((bits >> 4) * 0x204081u) & 0x01010101u) * 0x44u;
  return make_uint4(__byte_perm(v.x, low, a), __byte_perm(v.y, low, a >> 16), __byte_perm(v.z, low, b),
                    __byte_perm(v.w, low, b >> 16));
}

// The mask bits of the 16 / sizeof(T) tokens from v on.
template <typename T>
__device__ __forceinline__ unsigned mask_bits(const uint32_t* mask, int v) {
  constexpr int VE = 16 / sizeof(T);
  const int sh = v & 31;
  const uint32_t lo = mask[v >> 5], hi = sh + VE > 32 ? mask[(v >> 5) + 1] : 0u;
  return __funnelshift_r(lo, hi, sh) & ((1u << VE) - 1u);
}

template <int N>
__device__ __forceinline__ void cp_async_at(unsigned smem, const void* gmem) {
  if constexpr (N == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem), "l"(gmem) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(smem), "l"(gmem) : "memory");
}

// Entries of a row's slice before its first 16-byte boundary.
template <typename T>
__device__ __forceinline__ int entries_before(const T* p) {
  return static_cast<int>((16u - (reinterpret_cast<uintptr_t>(p) & 15u)) & 15u) / static_cast<int>(sizeof(T));
}

// What the CTA's slice of the vocabulary needs of the request: words and the list of those
// that are not zero, and the slice's biases.
struct Slice {
  unsigned* words;
  uint16_t* list;
  int2* bias;  // [kCBiases]: entry of the slice, entry of the biases (more: last_biases')
  int *listed, *biases;
  int b, v0, n, W;
};

// The request that comes `q`-th when the longest histories (in steps of 2^kCStepBits tokens) come
// first, by bisection of the lengths; for kCOrdered requests at most.  Ends at a barrier.
__device__ __forceinline__ int ordered_request(const CParams& p, int q, int* found) {
  if (threadIdx.x < 32) {
    const int lane = threadIdx.x;
    const int32_t* len = p.c.history_len;
    const int a = lane < p.B ? min(max(len[lane], 0), p.c.history_width) >> kCStepBits : -1;
    const int b = lane + 32 < p.B ? min(max(len[lane + 32], 0), p.c.history_width) >> kCStepBits : -1;
    int key = 0;  // of the q-th: the largest that more than q have or exceed
    for (int bit = p.length_bits - 1; bit >= 0; --bit) {
      const int more = key | 1 << bit;
      if (__popc(__ballot_sync(~0u, a >= more)) + __popc(__ballot_sync(~0u, b >= more)) > q) key = more;
    }
    const unsigned ea = __ballot_sync(~0u, a == key), eb = __ballot_sync(~0u, b == key), below = (1u << lane) - 1u;
    q -= __popc(__ballot_sync(~0u, a > key)) + __popc(__ballot_sync(~0u, b > key));
    if (a == key && __popc(ea & below) == q) *found = lane;
    if (b == key && __popc(ea) + __popc(eb & below) == q) *found = lane + 32;
  }
  __syncthreads();
  return *found;
}

// A request's numbers, all on their way together before the CTA's first barrier.
struct Request {
  int len0, prompt0, bias0, bias1, draft;
  float rep, freq, pres;
  __device__ __forceinline__ Request(const CParams& p, int b) {
    const asymspec_constraints& c = p.c;
    len0 = c.history ? c.history_len[b] : 0;
    prompt0 = c.prompt_len ? c.prompt_len[b] : 0;
    bias0 = c.bias_offsets ? c.bias_offsets[b] : 0;
    bias1 = c.bias_offsets ? c.bias_offsets[b + 1] : 0;
    const int tid = threadIdx.x;  // (P - 1 is at most the CTA's threads)
    draft = c.drafts && tid < p.P - 1 ? c.drafts[b * c.drafts_ld + tid] : 0;
    rep = c.repetition ? c.repetition[b] : 1.f;
    freq = c.frequency ? c.frequency[b] : 0.f;
    pres = c.presence ? c.presence[b] : 0.f;
  }
};
static_assert(ASYMSPEC_CONSTRAIN_MAX_P - 1 <= kCThreads, "a thread per draft");

// A thread's first tokens of the history (four a load from the first 16-byte boundary on, one
// before and one after them) and its first bias, on their way before that barrier too.
struct Tokens {
  const int4* fours;
  int len, prompt, head, count, end, before, after, bias_first, bias_end, bias;
  int4 v[kCAhead];
  __device__ __forceinline__ void load(int4 (&to)[kCAhead], int i0) const {
#pragma unroll
    for (int e = 0; e < kCAhead; ++e)
      if (i0 + e * kCThreads < count) to[e] = fours[i0 + e * kCThreads];
  }
  __device__ __forceinline__ Tokens(const CParams& p, const Request& r, int b, unsigned& err) {
    const asymspec_constraints& c = p.c;
    const int tid = threadIdx.x;
    len = min(max(r.len0, 0), c.history_width);
    prompt = min(max(r.prompt0, 0), len);
    if (len != r.len0 || prompt != r.prompt0) err |= ASYMSPEC_DATA_BAD_LENGTH;
    const int32_t* h = c.history + b * c.history_ld;
    head = min(entries_before(h), len);
    count = (len - head) / 4;
    end = head + count * 4;
    fours = reinterpret_cast<const int4*>(h + head);
    before = tid < head ? h[tid] : 0;
    after = tid < len - end ? h[end + tid] : 0;
    load(v, tid);
    bias_first = min(max(r.bias0, 0), c.bias_count);
    bias_end = min(max(r.bias1, bias_first), c.bias_count);
    if (bias_first != r.bias0 || bias_end != r.bias1) err |= ASYMSPEC_DATA_BAD_LENGTH;
    bias = bias_first + tid < bias_end ? c.bias_tokens[bias_first + tid] : 0;
  }
};

// The tokens of the history are counted in shared memory: each CTA reads all of it (from
// the L2) and counts its slice's.  Ends at a barrier; the words are zero at the start,
// which a barrier before says.  (Clusters whose CTAs read a share each and count a token
// where its slice is, by remote atomics: 92 us for 32 requests of 65,536 tokens each against
// 117, but 61 against 47 at 8,000 and 66 against 60 at 20,000.)
__device__ __forceinline__ unsigned count_slice(const CParams& p, const Slice& s, const Request& r, Tokens& t) {
  const int v0 = s.v0, n = s.n, tid = threadIdx.x;
  unsigned err = 0;
  auto here = [&](int v) {
    if (static_cast<unsigned>(v) >= static_cast<unsigned>(p.V)) err |= ASYMSPEC_DATA_BAD_TOKEN;
    return static_cast<unsigned>(v - v0) < static_cast<unsigned>(n);
  };
  auto count = [&](int v, int i) {
    if (!here(v)) return;
    if (i < t.prompt) atomicOr(&s.words[v - v0], kCPrompt);
    else atomicAdd(&s.words[v - v0], 1u);
  };
  if (tid < t.head) count(t.before, tid);
  if (tid < t.len - t.end) count(t.after, t.end + tid);
  for (int i0 = tid; i0 < t.count; i0 += kCThreads * kCAhead) {
    int4 next[kCAhead];
    t.load(next, i0 + kCThreads * kCAhead);
#pragma unroll
    for (int e = 0; e < kCAhead; ++e) {
      if (i0 + e * kCThreads >= t.count) break;
      const int i = t.head + (i0 + e * kCThreads) * 4;
      count(t.v[e].x, i);
      count(t.v[e].y, i + 1);
      count(t.v[e].z, i + 2);
      count(t.v[e].w, i + 3);
    }
#pragma unroll
    for (int e = 0; e < kCAhead; ++e) t.v[e] = next[e];
  }
  if (p.c.drafts && tid < p.P - 1 && here(r.draft)) atomicOr(&s.words[r.draft - v0], kCDraft);
  for (int i = t.bias_first + tid; i < t.bias_end; i += kCThreads) {
    const int v = i == t.bias_first + tid ? t.bias : p.c.bias_tokens[i];
    if (!here(v)) continue;
    atomicOr(&s.words[v - v0], kCBias);
    const int at = atomicAdd(s.biases, 1);
    if (at < kCBiases) s.bias[at] = make_int2(v - v0, i);
  }
  __syncthreads();
  return err;
}

// The list of the words that are not zero (in any order); a barrier has to follow.
__device__ __forceinline__ void list_slice(const Slice& s) {
  for (int i0 = threadIdx.x * 8; i0 < s.W; i0 += kCThreads * 8) {
    const uint4 f = *reinterpret_cast<const uint4*>(s.words + i0);
    const uint4 g = *reinterpret_cast<const uint4*>(s.words + i0 + 4);
    if ((f.x | f.y | f.z | f.w | g.x | g.y | g.z | g.w) == 0) continue;
    const unsigned w[8] = {f.x, f.y, f.z, f.w, g.x, g.y, g.z, g.w};
    int at = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) at += w[e] != 0;
    at = atomicAdd(s.listed, at);
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (w[e] != 0) s.list[at++] = static_cast<uint16_t>(i0 + e);
  }
}

// Where a slice has more than kCBiases bias entries, its tokens take theirs in parts of kCPart: the
// last entry of each token of a part, plus one (0: none), by a sweep of the request's list.  (A
// search of the list for each token would take the square of the biases: 64 requests of 16,000 each
// 3096 us, 337 so; of all 128,256 180 ms.)  Begins and ends at a barrier.
__device__ __forceinline__ void last_biases(const asymspec_constraints& c, int b, int first, int n, int* last) {
  __syncthreads();
  for (int i = threadIdx.x; i < kCPart; i += kCThreads) last[i] = 0;
  __syncthreads();
  const int a = min(max(c.bias_offsets[b], 0), c.bias_count);
  const int e = min(max(c.bias_offsets[b + 1], a), c.bias_count);
#pragma unroll 4
  for (int j = a + threadIdx.x; j < e; j += kCThreads) {
    const unsigned i = static_cast<unsigned>(c.bias_tokens[j]) - static_cast<unsigned>(first);
    if (i < static_cast<unsigned>(n)) atomicMax(last + i, j + 1);
  }
  __syncthreads();
}

struct Penalties {
  float rep, freq, pres, top;
  __device__ __forceinline__ Penalties(const Request& r, float top_, unsigned& err)
      : rep(r.rep), freq(r.freq), pres(r.pres), top(top_) {
    if (!(rep > 0.f && rep <= FLT_MAX && fabsf(freq) <= FLT_MAX && fabsf(pres) <= FLT_MAX)) {
      err |= ASYMSPEC_DATA_BAD_PENALTY;
      rep = 1.f;
      freq = pres = 0.f;
    }
  }
};

// One entry of the list: its word, bias, and how often its token came up to a row.
struct Touched {
  int v;
  unsigned w, count;
  float bias;
  __device__ __forceinline__ Touched(const CParams& p, const Slice& s, int i, int k0)
      : v(s.v0 + i), w(s.words[i]), count(w & kCCount), bias(0.f) {
    const asymspec_constraints& c = p.c;
    if (w & kCBias) {
      int last = -1;
      if (*s.biases <= kCBiases) {
        for (int j = 0; j < *s.biases; ++j)
          if (s.bias[j].x == i) last = max(last, s.bias[j].y);
      } else {
        last = reinterpret_cast<const int*>(s.bias)[i % kCPart] - 1;
      }
      bias = c.bias_values[last];
    }
    if (w & kCDraft)
      for (int j = 0; j < k0; ++j) count += c.drafts[s.b * c.drafts_ld + j] == v;
  }
  __device__ __forceinline__ float value(const Penalties& r, float z) const {
    float f = z;
    if (count != 0 || (w & kCPrompt)) f = f > 0.f ? f / r.rep : f * r.rep;
    if (count != 0) f = (f - r.freq * static_cast<float>(count)) - r.pres;
    if (w & kCBias) f += bias;
    return fabsf(z) <= FLT_MAX && bias == bias ? fminf(fmaxf(f, -r.top), r.top) : f;  // (fmaxf drops a NaN)
  }
  // past row k
  __device__ __forceinline__ void past(const CParams& p, const Slice& s, int k) {
    if ((w & kCDraft) && k < p.P - 1) count += p.c.drafts[s.b * p.c.drafts_ld + k] == v;
  }
};

// The mask of row r: its row of bits, -1: none, -2: it allows nothing.
__device__ __forceinline__ int mask_of(const CParams& p, int64_t r, unsigned& err) {
  if (!p.c.mask) return -1;
  const int at = p.c.mask_rows ? p.c.mask_rows[r] : static_cast<int>(r);
  if (at >= -1 && at < p.c.mask_count) return at;
  err |= ASYMSPEC_DATA_BAD_INDEX;
  return -2;
}

// The constrained rows, in another place than the logits or (masks) in theirs: one CTA per
// slice of the vocabulary, request and group of rows.  The rows' slices and their masks' words
// come into shared memory by cp.async while the history is counted; the entries that a penalty
// or a bias touches, gathered in a list so that no lane is idle, are computed there (in
// registers on the way of a copy each held up the 255 others of its warp, scattered over the
// rows in global memory they took longer than the rows); then the rows leave under their
// masks.  The slices of the lowest token ids, which a vocabulary gives to the most frequent
// tokens, come first in the grid: theirs are the most entries to compute.
// Bound by HBM, a row in and out; 64x8 rows of V=128256 bf16, half of them masked, histories to
// 8192: 47 us = 5.6 TB/s (43 with nothing to do but copy); 32x9 rows of V=151936, histories to
// 65536: 45 us, issuing instructions for the histories (34 without).
template <typename T, bool EDGES>
__global__ void __launch_bounds__(kCThreads, 4) constrain_rows(const CParams p) {
  extern __shared__ __align__(16) unsigned c_smem[];
  __shared__ int2 s_bias[kCBiases];
  __shared__ uint32_t s_mask[kCSlots * kCThreads / 4];  // the rows' masks, the slice's words of each
  __shared__ int s_at[kCSlots];                         // which, -1: none, -2: one that allows nothing
  __shared__ int s_listed, s_biases;
  constexpr int VE = 16 / sizeof(T);
  constexpr unsigned kAll = (1u << VE) - 1u;
  const asymspec_constraints& c = p.c;
  __shared__ int s_request;
  int b = blockIdx.x, at_slice = blockIdx.y;
  if (at_slice >= p.ordered_from) {
    const int last = static_cast<int>(gridDim.y) - p.ordered_from, i = (at_slice - p.ordered_from) * p.B + b;
    at_slice = p.ordered_from + i % last;
    b = ordered_request(p, i / last, &s_request);
  }
  const int W = p.W, v0 = at_slice * W, n = min(W, p.V - v0), tid = threadIdx.x;
  const Slice slice = {c_smem, reinterpret_cast<uint16_t*>(c_smem + W), s_bias, &s_listed, &s_biases, b, v0, n, W};
  const int pitch = constrain_pitch(W, sizeof(T));
  unsigned char* tile = reinterpret_cast<unsigned char*>(c_smem) + constrain_list_bytes(W);
  const int k_end = min((static_cast<int>(blockIdx.z) + 1) * p.group_rows, p.P);
  const int k0 = blockIdx.z * p.group_rows;
  unsigned err = 0;
  const T* x = static_cast<const T*>(p.logits) + (static_cast<int64_t>(b) * p.P + k0) * p.ld + v0;
  T* y = static_cast<T*>(p.out) + (static_cast<int64_t>(b) * p.P + k0) * p.out_ld + v0;
  auto misplaced = [&](const T* row) {  // bytes from the 16-byte boundary at or before it
    return EDGES ? static_cast<int>(reinterpret_cast<uintptr_t>(row) & 15u) : 0;
  };

  // A batch of rows, and their masks' words, on the way into shared memory
  const int batch = p.batch_rows, row_words = W / 32;
  const unsigned tile_at = smem_u32(tile);
  auto load_rows = [&](int first_row, int rows) {
    const T* from = x + static_cast<int64_t>(first_row) * p.ld;
    if constexpr (!EDGES) {
      for (int i = tid; i * VE < n; i += kCThreads) {
        const T* src = from + i * VE;
        unsigned dst = tile_at + i * 16;
#pragma unroll 4
        for (int k = 0; k < rows; ++k) {
          cp_async_at<16>(dst, src);
          src += p.ld;
          dst += pitch;
        }
      }
    } else {
      for (int k = 0; k < rows; ++k) {
        const T* row = from + k * p.ld;
        const int off = misplaced(row), first = off / static_cast<int>(sizeof(T));
        for (int j = tid; j * VE - first < n; j += kCThreads) {
          const int e0 = j * VE - first;
          if (e0 < 0 || e0 + VE > n) {
            for (int e = max(e0, 0); e < min(e0 + VE, n); ++e)
              *reinterpret_cast<T*>(tile + k * pitch + off + e * sizeof(T)) = row[e];
          } else {
            cp_async_at<16>(tile_at + k * pitch + j * 16, row + e0);
          }
        }
      }
    }
  };
  auto load_masks = [&](int first_row, int rows) {
    if (c.mask) {  // a warp a row
      const int words = min(row_words, (n + 31) / 32);
      for (int k = tid / 32; k < rows; k += kCThreads / 32) {
        const int at = mask_of(p, static_cast<int64_t>(b) * p.P + k0 + first_row + k, err);
        if (tid % 32 == 0) s_at[k] = at;
        if (at < 0) continue;
        const uint32_t* src = c.mask + at * c.mask_ld + (v0 >> 5);
        for (int w = tid % 32; w < words; w += 32) cp_async_at<4>(smem_u32(s_mask + k * row_words + w), src + w);
      }
    } else if (tid < rows) {
      s_at[tid] = -1;
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };

  load_rows(0, min(batch, k_end - k0));
  const Request request(p, b);
  if (tid == 0) s_listed = s_biases = 0;
  for (int i = tid; i < W / 4; i += kCThreads) reinterpret_cast<uint4*>(c_smem)[i] = make_uint4(0, 0, 0, 0);
  load_masks(0, min(batch, k_end - k0));
  Tokens tokens(p, request, b, err);
  __syncthreads();
  err |= count_slice(p, slice, request, tokens);
  list_slice(slice);
  const float top = type_max(T());
  const T low = from_f32(fminf(fmaxf(c.mask_value, -top), top), T());
  unsigned low_word;
  if constexpr (sizeof(T) == 4) low_word = __float_as_uint(low);
  else low_word = __bfloat16_as_ushort(low) * 0x10001u;
  const Penalties penalties(request, top, err);
  for (int first_row = 0;;) {
    const int rows = min(batch, k_end - k0 - first_row);
    const T* xt = x + static_cast<int64_t>(first_row) * p.ld;
    T* yt = y + static_cast<int64_t>(first_row) * p.out_ld;
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    __syncthreads();
    const int listed = s_listed;
    // an entry's rows by one thread, or, where entries are fewer than threads, by one each
    const int each = listed * rows <= 2 * kCThreads ? 1 : rows;
    auto touch = [&](int q) {
      const int i = slice.list[q % listed], first = q / listed;
      Touched u(p, slice, i, k0 + first_row + first);
#pragma unroll 4
      for (int k = first; k < first + each; ++k) {
        T* cell = reinterpret_cast<T*>(tile + k * pitch + misplaced(xt + k * p.ld)) + i;
        *cell = from_f32(u.value(penalties, to_f32(*cell)), T());
        u.past(p, slice, k0 + first_row + k);
      }
    };
    const int touches = listed * (rows / each);
    if (s_biases <= kCBiases) {
      for (int q = tid; q < touches; q += kCThreads) touch(q);
    } else {
      for (int part = 0; part < n; part += kCPart) {
        last_biases(c, b, v0 + part, min(kCPart, n - part), reinterpret_cast<int*>(s_bias));
        for (int q = tid; q < touches; q += kCThreads)
          if (slice.list[q % listed] / kCPart == part / kCPart) touch(q);
      }
    }
    if (listed > 0) __syncthreads();
    if constexpr (!EDGES) {
      for (int i = tid; i * VE < n; i += kCThreads) {
        const unsigned char* src = tile + i * 16;
        T* dst = yt + i * VE;
#pragma unroll 4
        for (int k = 0; k < rows; ++k) {
          uint4 v = *reinterpret_cast<const uint4*>(src);
          const int at = s_at[k];
          if (at != -1) {
            const uint8_t* mask = reinterpret_cast<const uint8_t*>(s_mask + k * row_words);
            const unsigned on = at < 0 ? 0u : VE == 8 ? mask[i] : (mask[i >> 1] >> ((i & 1) * 4)) & kAll;
            v = masked16<T>(v, on, low_word);
          }
          *reinterpret_cast<uint4*>(dst) = v;
          src += pitch;
          dst += p.out_ld;
        }
      }
    } else {
      for (int k = 0; k < rows; ++k) {
        T* row = yt + k * p.out_ld;
        const T* from = reinterpret_cast<const T*>(tile + k * pitch + misplaced(xt + k * p.ld));
        const int first = misplaced(row) / static_cast<int>(sizeof(T)), at = s_at[k];
        const uint32_t* mask = s_mask + k * row_words;
        for (int j = tid; j * VE - first < n; j += kCThreads) {
          const int e0 = j * VE - first;
          if (e0 < 0 || e0 + VE > n) {
            for (int e = max(e0, 0); e < min(e0 + VE, n); ++e)
              row[e] = at == -1 || (at >= 0 && ((mask[e >> 5] >> (e & 31)) & 1u)) ? from[e] : low;
          } else {
            uint4 v = reinterpret_cast<uintptr_t>(from + e0) % 16 == 0
                          ? *reinterpret_cast<const uint4*>(from + e0) : gather16(from + e0);
            if (at != -1) v = masked16<T>(v, at < 0 ? 0u : mask_bits<T>(mask, e0), low_word);
            *reinterpret_cast<uint4*>(row + e0) = v;
          }
        }
      }
    }
    first_row += rows;
    if (k0 + first_row >= k_end) break;
    __syncthreads();
    load_rows(first_row, min(batch, k_end - k0 - first_row));
    load_masks(first_row, min(batch, k_end - k0 - first_row));
  }
  if (err && p.err) atomicOr(p.err, err);
}

// The logits penalised and biased where they are, without masks: nothing but the entries
// that something touches is read or written, each where it lies (64x8 rows of V=128256 bf16
// with histories to 8192: 24 us, 45 through constrain_rows; with masks on half of the rows,
// when those were overwritten here too, 64 against 48: a call with masks takes constrain_rows
// in place).
template <typename T>
__global__ void __launch_bounds__(kCThreads) constrain_in_place(const CParams p) {
  extern __shared__ __align__(16) unsigned c_smem[];
  __shared__ int2 s_bias[kCBiases];
  __shared__ int s_listed, s_biases;
  __shared__ int s_request;
  int b = blockIdx.x, at_slice = blockIdx.y;
  if (at_slice >= p.ordered_from) {
    const int last = static_cast<int>(gridDim.y) - p.ordered_from, i = (at_slice - p.ordered_from) * p.B + b;
    at_slice = p.ordered_from + i % last;
    b = ordered_request(p, i / last, &s_request);
  }
  const int W = p.W, v0 = at_slice * W, n = min(W, p.V - v0), tid = threadIdx.x;
  const Slice slice = {c_smem, reinterpret_cast<uint16_t*>(c_smem + W), s_bias, &s_listed, &s_biases, b, v0, n, W};
  const int k0 = blockIdx.z * p.group_rows, rows = min(p.group_rows, p.P - k0);
  unsigned err = 0;
  const Request request(p, b);
  if (tid == 0) s_listed = s_biases = 0;
  for (int i = tid; i < W / 4; i += kCThreads) reinterpret_cast<uint4*>(c_smem)[i] = make_uint4(0, 0, 0, 0);
  Tokens tokens(p, request, b, err);
  __syncthreads();
  err |= count_slice(p, slice, request, tokens);
  list_slice(slice);
  const Penalties penalties(request, type_max(T()), err);
  T* x = static_cast<T*>(p.out) + (static_cast<int64_t>(b) * p.P + k0) * p.out_ld + v0;
  __syncthreads();  // the list
  auto touch = [&](int i) {
    Touched t(p, slice, i, k0);
#pragma unroll 4
    for (int k = 0; k < rows; ++k) {
      T* cell = x + k * p.out_ld + i;
      *cell = from_f32(t.value(penalties, to_f32(*cell)), T());
      t.past(p, slice, k0 + k);
    }
  };
  if (s_biases <= kCBiases) {
    for (int q = tid; q < s_listed; q += kCThreads) touch(slice.list[q]);
  } else {
    for (int part = 0; part < n; part += kCPart) {
      last_biases(p.c, b, v0 + part, min(kCPart, n - part), reinterpret_cast<int*>(s_bias));
      for (int q = tid; q < s_listed; q += kCThreads)
        if (slice.list[q] / kCPart == part / kCPart) touch(slice.list[q]);
    }
  }
  if (err && p.err) atomicOr(p.err, err);
}

}  // namespace asymspec_impl
