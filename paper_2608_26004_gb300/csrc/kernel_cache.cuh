// The paged key-value cache: block tables and slot maps (asymspec_cache_plan), and the
// writing of new keys and values (asymspec_cache_write).
#pragma once

#include "asymspec_serving.h"
#include "device_common.cuh"

namespace asymspec_impl {

struct PlanParams {
  const int32_t *lens, *accepted, *grow, *held, *free_count;
  int grow_all, B, block_size, num_blocks, table_width;
  int32_t *tables, *free_list;
  int64_t table_ld;
  int32_t *out_start, *out_len, *out_held, *out_free, *out_offsets, *out_positions;
  int64_t* out_slots;
  int64_t capacity;
  uint32_t* err;
};

constexpr int kPThreads = 1024;
constexpr int kPCluster = 8;

// Shared memory of the plan kernel: a request's tokens that stay, its blocks before (bit 31:
// not served) and the prefix sums of tokens, blocks taken and blocks given back.
constexpr size_t plan_smem_bytes(int B) {
  return static_cast<size_t>(B + 1) * (8 + 4 * 4);
}

// Largest i in [0, n) with first(i) <= x, for first(0) <= x, ascending.
template <typename A>
__device__ __forceinline__ int find_last(const A* first, int n, A x) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (first[mid] <= x) lo = mid;
    else hi = mid;
  }
  return lo;
}

// Inclusive prefix sums over the CTA of three numbers a thread.
__device__ __forceinline__ void scan3(int64_t& a, int& b, int& c, int64_t* wa, int* wb, int* wc) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int64_t a2 = __shfl_up_sync(~0u, a, d);
    const int b2 = __shfl_up_sync(~0u, b, d), c2 = __shfl_up_sync(~0u, c, d);
    if (lane >= d) a += a2, b += b2, c += c2;
  }
  if (lane == 31) wa[warp] = a, wb[warp] = b, wc[warp] = c;
  __syncthreads();
  for (int w = 0; w < warp; ++w) a += wa[w], b += wb[w], c += wc[w];
  __syncthreads();
}

// One CTA, or (CLUSTER) a cluster of them.  Every CTA goes over all requests by itself (a few
// numbers each: cheaper than an exchange), then they share the blocks given back, the
// blocks taken and the slots, each found by a search in the prefix sums, with a barrier
// between what one part writes and the next reads.  Bound by latency: 64 requests of 8 slots
// 5.1 us, 256 requests of 115,000 slots in all 17.3 us (8 CTAs; 120 with one).
template <bool CLUSTER>
__global__ void __launch_bounds__(kPThreads) cache_plan_kernel(const PlanParams p) {
  extern __shared__ int64_t p_smem[];
  __shared__ int64_t wa[32];
  __shared__ int wb[32], wc[32];
  __shared__ int s_taken;
  cg::cluster_group cluster = cg::this_cluster();
  const int rank = CLUSTER ? static_cast<int>(cluster.block_rank()) : 0;
  const int stride = (CLUSTER ? static_cast<int>(cluster.num_blocks()) : 1) * kPThreads;
  auto barrier = [&] {
    if constexpr (CLUSTER) cluster.sync();
    else __syncthreads();
  };
  const int B = p.B, bs = p.block_size, tid = threadIdx.x, at0 = rank * kPThreads + tid;
  int64_t* offs = p_smem;  // [B + 1]
  int* keep_of = reinterpret_cast<int*>(offs + B + 1);
  int* held_of = keep_of + B + 1;
  int* more_of = held_of + B + 1;  // blocks taken by the requests before
  int* less_of = more_of + B + 1;  // blocks given back by the requests before
  unsigned err = 0;
  const int free0 = *p.free_count, free_in = min(max(free0, 0), p.num_blocks);
  if (free_in != free0) err |= ASYMSPEC_DATA_BAD_LENGTH;
  if (tid == 0) s_taken = 0;
  int64_t off = 0;
  int more_sum = 0, less_sum = 0;
  const int64_t most = static_cast<int64_t>(p.table_width) * bs;
  for (int b0 = 0; b0 < B; b0 += kPThreads) {
    const int b = b0 + tid;
    int64_t g = 0;
    int more = 0, less = 0, keep = 0, held = 0;
    if (b < B) {
      const int l0 = p.lens[b], a0 = p.accepted ? p.accepted[b] : -1;
      const int g0 = p.grow ? p.grow[b] : p.grow_all, h0 = p.held[b];
      int64_t k = static_cast<int64_t>(max(l0, 0)) + max(a0, -1) + 1;
      g = max(g0, 0);
      held = min(max(h0, 0), p.table_width);
      bool bad = l0 < 0 || a0 < -1 || g0 < 0 || held != h0;
      bool served = true;
      if (k > most) k = most, bad = true;
      keep = static_cast<int>(k);
      int blocks = held;
      if (k + g > most) {  // too long for its table: what it has stays
        bad = true;
        served = false;
      } else {
        blocks = static_cast<int>((static_cast<unsigned>(k + g) + static_cast<unsigned>(bs) - 1u) /
                                  static_cast<unsigned>(bs));
      }
      if (bad) err |= ASYMSPEC_DATA_BAD_LENGTH;
      more = max(blocks - held, 0);
      less = max(held - blocks, 0);
      keep_of[b] = keep;
      held_of[b] = served ? held : held | INT_MIN;
    }
    const int64_t g1 = g;
    const int m1 = more, l1 = less;
    scan3(g, more, less, wa, wb, wc);
    if (b < B) {
      offs[b] = off + g - g1;
      more_of[b] = more_sum + more - m1;
      less_of[b] = less_sum + less - l1;
    }
    if (tid == kPThreads - 1) wa[0] = g, wb[0] = more, wc[0] = less;
    __syncthreads();
    off += wa[0];
    more_sum += wb[0];
    less_sum += wc[0];
    __syncthreads();
  }
  if (tid == 0) offs[B] = off, more_of[B] = more_sum, less_of[B] = less_sum;
  barrier();  // (the inputs are read: outputs may lie over them)
  const int64_t top = static_cast<int64_t>(free_in) + less_sum;  // (bad data: past num_blocks, and 2^31)
  // who is served; the state of the next call
  for (int b = tid; b < B; b += kPThreads) {
    const int m = more_of[b + 1] - more_of[b], l = less_of[b + 1] - less_of[b];
    const int held = held_of[b] & INT_MAX;
    bool served = held_of[b] >= 0;
    if (m > 0 && more_of[b + 1] > top) {
      served = false;
      err |= ASYMSPEC_DATA_NO_BLOCKS;
    } else if (m > 0) {
      atomicMax(&s_taken, more_of[b + 1]);
    }
    if (!served) held_of[b] = held | INT_MIN;
    if (rank != 0) continue;
    const int64_t g = offs[b + 1] - offs[b];
    p.out_start[b] = keep_of[b];
    p.out_len[b] = served ? keep_of[b] + static_cast<int>(g) : keep_of[b];
    p.out_held[b] = held - l + (served ? m : 0);
  }
  if (off > p.capacity) err |= ASYMSPEC_DATA_BAD_LENGTH;
  if (rank == 0)
    for (int b = tid; b <= B; b += kPThreads)
      p.out_offsets[b] = static_cast<int>(min(offs[b], static_cast<int64_t>(INT_MAX)));
  __syncthreads();
  // blocks given back go on the stack
  if (less_sum > 0) {
    for (int i = at0; i < less_sum; i += stride) {
      const int b = find_last(less_of, B, i);
      const int kept = (held_of[b] & INT_MAX) - (less_of[b + 1] - less_of[b]);
      const int64_t at = static_cast<int64_t>(free_in) + i;
      if (at < p.num_blocks) p.free_list[at] = p.tables[b * p.table_ld + kept + i - less_of[b]];
      else err |= ASYMSPEC_DATA_BAD_LENGTH;
    }
    barrier();
  }
  // and blocks are taken off it
  const int taken = s_taken;
  for (int i = at0; i < taken; i += stride) {
    const int b = find_last(more_of, B, i);
    const int64_t at = top - 1 - i;
    p.tables[b * p.table_ld + (held_of[b] & INT_MAX) + i - more_of[b]] =
        at < p.num_blocks ? __ldcg(p.free_list + at) : -1;
  }
  if (at0 == 0) *p.out_free = static_cast<int>(min(top - taken, static_cast<int64_t>(p.num_blocks)));
  barrier();
  // kPSlots slots a thread: one search, a division where a block begins
  constexpr int kPSlots = CLUSTER ? 4 : 1;
  const bool wide = (reinterpret_cast<uintptr_t>(p.out_slots) & 15u) == 0;
  const bool wide_pos = (reinterpret_cast<uintptr_t>(p.out_positions) & 15u) == 0;
  for (int64_t t0 = static_cast<int64_t>(at0) * kPSlots; t0 < p.capacity;
       t0 += static_cast<int64_t>(stride) * kPSlots) {
    int64_t slot[kPSlots];
    __align__(16) int pos[kPSlots];
    int b = t0 < off ? find_last(offs, B, t0) : 0, left = 0, next = 0;
    int64_t place = -1;
#pragma unroll
    for (int e = 0; e < kPSlots; ++e) {
      const int64_t t = t0 + e;
      slot[e] = -1;
      pos[e] = -1;
      if (t >= off || t >= p.capacity) continue;
      if (t >= offs[b + 1]) {
        do ++b;
        while (t >= offs[b + 1]);
        left = 0;
      }
      if (held_of[b] < 0) continue;
      if (left == 0) {
        next = keep_of[b] + static_cast<int>(t - offs[b]);
        const int page = __ldcg(p.tables + b * p.table_ld + next / bs), at = next % bs;
        const bool there = static_cast<unsigned>(page) < static_cast<unsigned>(p.num_blocks);
        if (!there) err |= ASYMSPEC_DATA_BAD_INDEX;
        place = there ? static_cast<int64_t>(page) * bs + at : -1;
        left = bs - at;
      }
      slot[e] = place;
      pos[e] = next;
      if (place >= 0) ++place;
      ++next;
      --left;
    }
    if (CLUSTER && wide && t0 + kPSlots <= p.capacity) {
#pragma unroll
      for (int e = 0; e + 1 < kPSlots; e += 2)
        *reinterpret_cast<longlong2*>(p.out_slots + t0 + e) = make_longlong2(slot[e], slot[e + 1]);
    } else {
#pragma unroll
      for (int e = 0; e < kPSlots; ++e)
        if (t0 + e < p.capacity) p.out_slots[t0 + e] = slot[e];
    }
    if (!p.out_positions) continue;
    if (CLUSTER && wide_pos && t0 + kPSlots <= p.capacity) {
      *reinterpret_cast<int4*>(p.out_positions + t0) = *reinterpret_cast<const int4*>(pos);
    } else {
#pragma unroll
      for (int e = 0; e < kPSlots; ++e)
        if (t0 + e < p.capacity) p.out_positions[t0 + e] = pos[e];
    }
  }
  if (err && p.err) atomicOr(p.err, err);
}

struct WriteParams {
  const void *k, *v;
  void *keys, *values;
  int64_t ks[2], vs[2], cks[3], cvs[3];
  const int64_t* slots;
  int T, num_blocks, block_size, kv_heads, head_dim;
  int log_lanes;  // 2^log_lanes lanes for a token
  uint32_t* err;
};

constexpr int kWThreads = 256;

// U: what is moved at once (16 bytes, or one element where something is not on the
// 16-byte boundaries); strides and head_dim in elements of U.  A copy, bound by its bytes: a
// warp, or part of one where a token has fewer vectors, takes a token, four of its
// vectors a lane on their way together, so that a slot is looked up and divided once.
// 16384 tokens of 8 heads of 128 bf16: 21.1 us = 6.4 TB/s (a thread per vector: 23.3).
template <typename U>
__global__ void __launch_bounds__(kWThreads) cache_write_kernel(const WriteParams p) {
  const int lanes = 1 << p.log_lanes, lane = threadIdx.x & (lanes - 1);
  const int per = p.kv_heads * p.head_dim;
  const unsigned slots = static_cast<unsigned>(p.num_blocks) * static_cast<unsigned>(p.block_size);
  const int64_t stride = static_cast<int64_t>(gridDim.x) * (kWThreads >> p.log_lanes);
  for (int64_t t = (static_cast<int64_t>(blockIdx.x) * kWThreads + threadIdx.x) >> p.log_lanes; t < p.T; t += stride) {
    const int64_t slot = p.slots[t];
    if (slot < 0) continue;
    if (slot >= slots) {
      if (lane == 0 && p.err) atomicOr(p.err, ASYMSPEC_DATA_BAD_INDEX);
      continue;
    }
    const unsigned block = static_cast<unsigned>(slot) / static_cast<unsigned>(p.block_size);
    const unsigned at = static_cast<unsigned>(slot) - block * static_cast<unsigned>(p.block_size);
    const U* k = static_cast<const U*>(p.k) + t * p.ks[0];
    const U* v = static_cast<const U*>(p.v) + t * p.vs[0];
    U* keys = static_cast<U*>(p.keys) + block * p.cks[0] + at * p.cks[1];
    U* values = static_cast<U*>(p.values) + block * p.cvs[0] + at * p.cvs[1];
    for (int e0 = lane; e0 < per; e0 += lanes * 4) {
      U x[4], y[4];
      int h[4], d[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int e = e0 + i * lanes;
        h[i] = e / p.head_dim;
        d[i] = e - h[i] * p.head_dim;
        if (e < per) {
          x[i] = k[h[i] * p.ks[1] + d[i]];
          y[i] = v[h[i] * p.vs[1] + d[i]];
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (e0 + i * lanes < per) {
          keys[h[i] * p.cks[2] + d[i]] = x[i];
          values[h[i] * p.cvs[2] + d[i]] = y[i];
        }
      }
    }
  }
}

}  // namespace asymspec_impl
