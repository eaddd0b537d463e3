// Attention of a few new tokens over a paged key-value cache (asymspec_cache_attend).
#pragma once

#include <cfloat>

#include "asymspec_serving.h"
#include "device_common.cuh"

namespace asymspec_impl {

struct AttendParams {
  const void *keys, *values, *q;
  void* out;
  float* lse;
  int64_t cks[3], cvs[3], qs[3], os[3];
  const int32_t *tables, *lens;
  int64_t table_ld;
  int B, Q, heads, kv_heads, D, num_blocks, block_size, table_width, window;
  int group;      // query heads of a kv head
  int rows;       // queries that share a kv head's keys: Q * group, row = query * group + head
  int row_tiles;  // tiles of 16 * WR of them
  float scale2;   // scale * log2(e)
  bool q_vec, out_vec;
  // Blocks of a multiple of 16 tokens (a step's keys lie in one block, in a row), and
  // strides within a block of fewer than 2^31 bytes:
  bool whole_steps;
  int block_bytes[2], token_bytes[2];  // of keys and values
  char* ws;
  uint32_t* err;
};

constexpr int kAGroups = 4;                 // groups of warps, each with keys of its own
constexpr int kAKeys = 16;                  // keys of a group's step
constexpr int kATile = kAGroups * kAKeys;   // keys of a CTA's step, the unit of the split
constexpr int kAMaxCtas = 456;              // CTAs that share the work (up to three on each of 152 SMs)
constexpr int kAJoinThreads = 128;

// The work is split by units: an item (a request, kv head and row tile) has one for each
// of its tiles, after kAItem for what it costs to begin and end one (64 requests of 64 to 8192
// tokens, kAItem = 1, 2, 3: 80, 75, 76 us).
constexpr int kAItem = 2;

// A CTA whose share begins after the first tile of an item says which.
struct AttendInfo {
  int64_t total;  // units of all items
  int64_t first;  // the item's first unit
  int b, hr, tiles, pad;
};

// Workspace: an AttendInfo per CTA; then, for two parts a CTA (one of an item that an
// earlier CTA began, one of an item that a later CTA goes on with), each row's maximum
// and sum, and each row's weighted values.
constexpr size_t kAInfoBytes = (kAMaxCtas * sizeof(AttendInfo) + 255) / 256 * 256;
__host__ __device__ constexpr size_t attend_ml_bytes(int rows) {
  return (static_cast<size_t>(2 * kAMaxCtas) * rows * 2 * sizeof(float) + 255) / 256 * 256;
}
constexpr size_t attend_ws_bytes(int rows, int DP) {
  return kAInfoBytes + attend_ml_bytes(rows) + static_cast<size_t>(2 * kAMaxCtas) * rows * DP * sizeof(float);
}

// Whether rows of keys, values and queries lie in shared memory 16 bytes further apart than they
// are long, so that the eight rows that ldmatrix reads meet no bank twice and all addresses are
// one and an immediate; else their 16-byte chunks are swizzled.  us, swizzled / with such rows:
// two warps a group (8 requests of 4096 to 32768 tokens, 32 rows a kv head of 128) 102.7 / 99.1,
// four (64 rows) 179 / 167; one (64 requests of one query) 74.7 / 79.3; heads of 256 167 / 183.
// fp32 has no room for longer rows.
template <typename T>
__host__ __device__ constexpr bool attend_long_rows(int DP, int WR) {
  return sizeof(T) == 2 && DP <= 128 && WR > 1;
}
template <typename T>
__host__ __device__ constexpr int attend_pitch(int DP, int WR) {
  return DP * static_cast<int>(sizeof(T)) + (attend_long_rows<T>(DP, WR) ? 16 : 0);
}

// Dynamic shared memory: the groups' rings, the queries (fp32: in two pieces), each warp's masks
// of keys that exist and its references and sums, and the numbers that find a CTA's share.
template <typename T>
constexpr size_t attend_smem_bytes(int DP, int WR, int ST) {
  return static_cast<size_t>(kAGroups) * ST * 2 * kAKeys * attend_pitch<T>(DP, WR) +
         static_cast<size_t>(16) * WR * attend_pitch<T>(DP, WR) * (sizeof(T) == 4 ? 2 : 1) + kAGroups * WR * ST * 4 +
         static_cast<size_t>(kAGroups) * 16 * WR * 8 + kAGroups * WR * 8 + 16;
}

__device__ __forceinline__ void put(float* p, float y) { *p = y; }
__device__ __forceinline__ void put(__nv_bfloat16* p, float y) { *p = __float2bfloat16_rn(y); }

// ln of a row's sum, from its reference and the sum of its weights: -infinity where it has no keys;
// where all of its scores are NaN its reference is -infinity too, and its sum the NaN.
__device__ __forceinline__ float lse_of(float m, float l) { return l == 0.f ? -INFINITY : fmaf(m, kLn2, logf(l)); }

__device__ __forceinline__ int attend_len(const AttendParams& p, int b) {
  return min(max(p.lens[b], 0), p.table_width * p.block_size);
}
// Where a request's keys begin: the first that any query sees, or up to 15 before it.
__device__ __forceinline__ int attend_first(const AttendParams& p, int len) {
  return p.window ? max(0, len - p.Q - p.window + 1) & ~(kAKeys - 1) : 0;
}
__device__ __forceinline__ int attend_tiles(const AttendParams& p, int len) {
  return max(1, (len - attend_first(p, len) + kATile - 1) / kATile);
}
__device__ __forceinline__ int64_t div64(int64_t a, int64_t b) {  // (of numbers >= 0)
  return (a | b) >> 32 ? a / b : static_cast<int64_t>(static_cast<unsigned>(a) / static_cast<unsigned>(b));
}
// CTA c's share: units c * each + min(c, more) on, of `each`, the first `more` CTAs one more.
struct AttendShares {
  int64_t each;
  int more;
  __device__ __forceinline__ AttendShares(int64_t total, int ctas)
      : each(div64(total, ctas)), more(static_cast<int>(total - each * ctas)) {}
  __device__ __forceinline__ int64_t start(int c) const { return c * each + min(c, more); }
  __device__ __forceinline__ int owner(int64_t unit) const {
    const int64_t big = (each + 1) * more;
    return static_cast<int>(unit < big ? div64(unit, each + 1) : more + div64(unit - big, each));
  }
};

// 16 bytes, or with bytes = 0 zeros (the address is then not read).
__device__ __forceinline__ void cp_async16_or_zero(unsigned smem, const void* gmem, int bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem), "l"(gmem), "r"(bytes) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ void ldmatrix4(unsigned (&r)[4], unsigned a) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a));
}
__device__ __forceinline__ void ldmatrix4_trans(unsigned (&r)[4], unsigned a) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a));
}
__device__ __forceinline__ void mma_bf16(float (&c)[4], const unsigned (&a)[4], unsigned b0, unsigned b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
      "{%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_tf32(float (&c)[4], const unsigned (&a)[4], unsigned b0, unsigned b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
      "{%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// x = hi + lo + (2^-21 |x| at most, of lo's sign, which is either), each with tf32's 11
// significant bits: hi rounded, its distance from x (exact) cut.  In integer arithmetic: the
// conversion instruction is slow (32 requests, a window of 2000: 43.7 us with it, 39.1 so).  An
// x that is a NaN or infinite makes lo a NaN.
__device__ __forceinline__ void split_tf32(float x, unsigned& hi, unsigned& lo) {
  hi = (__float_as_uint(x) + 0x1000u) & 0xFFFFE000u;
  lo = __float_as_uint(x - __uint_as_float(hi)) & 0xFFFFE000u;
}
// (x, y) = hi + lo + (2^-17 of each at most), packed bf16.
__device__ __forceinline__ void split_bf16(float x, float y, unsigned& hi, unsigned& lo) {
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(hi) : "f"(y), "f"(x));
  const float rx = x - __uint_as_float(hi << 16), ry = y - __uint_as_float(hi & 0xFFFF0000u);
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(lo) : "f"(ry), "f"(rx));
}

// Where 16-byte chunk `c` of row `r` lies in the row, if rows are not longer.  bf16: ldmatrix
// reads one chunk of eight rows.  fp32 keys: eight lanes read four chunks of two neighbouring
// rows; values: two chunks of four rows of one parity.
template <typename T, bool VALUES, bool LONG_ROWS>
__device__ __forceinline__ int swizzled(int r, int c) {
  if constexpr (LONG_ROWS) return c;
  return sizeof(T) == 2 || VALUES ? c ^ (r & 7) : c ^ (((r & 1) << 2) | ((r >> 1) & 3));
}

// Chunks 2 k and 2 k + 1 of a row from the address of its chunks 0 and 1.
template <bool LONG_ROWS>
__device__ __forceinline__ unsigned chunk_pair(unsigned at, int k) {
  return LONG_ROWS ? at + k * 32 : at ^ (k * 32);
}

__device__ __forceinline__ void group_barrier(int id, int threads) {
  asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory");
}

// The keys are split evenly over the CTAs, in tiles of 64, whatever the requests' lengths.
// A CTA has four groups of WR warps: a group takes 16 keys of each tile through a ring of
// its own (cp.async, its warps load a part each), and each of its warps 16 of the item's
// rows, with running references, sums and weighted values in registers.  When the CTA's share of
// an item ends, the groups' parts are joined in shared memory.
// Bound by the bytes of keys and values at 16 rows: bf16, 64 requests of 64 to 8192 tokens, 32
// heads on 8 of 128: 74 us = 5.9 TB/s; by issue and latency at 32 (16 requests of 4096 to
// 131072 tokens, 8 queries each: 425 us = 6.0 TB/s) and by the matrix instructions at 64 (8
// requests to 32768: 167 us, 99 at 32 rows).  fp32, 32 requests, 5 queries, a window of 2000, 8
// heads of 64: 37 us = 4.2 TB/s, waiting for its products.  kH: halves of a warp's 16 rows in use.
template <typename T, int DP, int WR, int ST, int PER_SM, int kH>
__global__ void __launch_bounds__(kAGroups * WR * 32, PER_SM) attend_split(const AttendParams p) {
  constexpr bool BF = sizeof(T) == 2;
  constexpr int kThreadsN = kAGroups * WR * 32, kWarpsN = kAGroups * WR;
  constexpr int kRowBytes = DP * sizeof(T), kChunks = kRowBytes / 16, PE = 16 / sizeof(T);
  constexpr bool kLong = attend_long_rows<T>(DP, WR);
  constexpr int kPitch = attend_pitch<T>(DP, WR);
  constexpr int kHalf = kAKeys * kPitch;  // bytes of a step's keys (and of its values)
  constexpr int kRows = 16 * WR;
  constexpr int NT = DP / 8;
  constexpr int kLoads = kChunks / 2 / WR;   // vectors that a lane loads of a step's keys
  constexpr size_t kMlBytes = attend_ml_bytes(kRows);
  constexpr float kSlack = 8.f;
  constexpr bool kQRegs = BF && DP <= 128 && WR == 1;
  static_assert(kLoads >= 1 && (BF ? 1 : 2) * ST >= WR, "a warp loads, and the parts fit in the rings");
  extern __shared__ __align__(1024) unsigned char a_smem[];
  unsigned char* at_q = a_smem + static_cast<size_t>(kAGroups) * ST * 2 * kHalf;
  T* qs = reinterpret_cast<T*>(at_q);  // fp32: the high pieces, then the low ones
  unsigned* masks0 = reinterpret_cast<unsigned*>(at_q + static_cast<size_t>(kRows) * kPitch * (BF ? 1 : 2));
  float* s_ml = reinterpret_cast<float*>(masks0 + kWarpsN * ST);
  int64_t* s_scan = reinterpret_cast<int64_t*>(s_ml + kWarpsN * 16 * 2);
  int64_t* s_find = s_scan + kWarpsN;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t4 = lane & 3;
  const int group = warp / WR, wr = warp % WR;  // whose keys; which rows
  unsigned* masks = masks0 + warp * ST;
  unsigned char* ring = a_smem + group * ST * 2 * kHalf;
  const unsigned ring_at = smem_u32(ring), q_at = smem_u32(qs) + wr * 16 * kPitch;
  const int c = blockIdx.x, ctas = gridDim.x;
  const int HR = p.kv_heads * p.row_tiles;
  unsigned err = 0;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

  // this CTA's share of the units, and where it begins
  const int per = (p.B + kThreadsN - 1) / kThreadsN;
  int64_t mine = 0;
  for (int b = tid * per; b < min((tid + 1) * per, p.B); ++b) {
    const int len = attend_len(p, b);
    if (len != p.lens[b]) err |= ASYMSPEC_DATA_BAD_LENGTH;
    mine += attend_tiles(p, len) + kAItem;
  }
  int64_t upto = mine;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int64_t o = __shfl_up_sync(~0u, upto, d);
    if (lane >= d) upto += o;
  }
  if (lane == 31) s_scan[warp] = upto;
  __syncthreads();
  int64_t total = 0;
  for (int w = 0; w < kWarpsN; ++w) {
    if (w < warp) upto += s_scan[w];
    total += s_scan[w];
  }
  total *= HR;
  const AttendShares shares(total, ctas);
  int64_t u = shares.start(c);
  const int64_t u_end = shares.start(c + 1);
  if (u < u_end && (upto - mine) * HR <= u && u < upto * HR) {
    int64_t v = u - (upto - mine) * HR;
    int b = tid * per;
    for (;; ++b) {
      const int64_t n = static_cast<int64_t>(attend_tiles(p, attend_len(p, b)) + kAItem) * HR;
      if (v < n) break;
      v -= n;
    }
    s_find[0] = b;
    s_find[1] = v;
  }
  __syncthreads();
  AttendInfo* info = reinterpret_cast<AttendInfo*>(p.ws) + c;
  if (u >= u_end) {
    if (tid == 0) info->tiles = 0;
    if (err && p.err) atomicOr(p.err, err);
    return;
  }
  int b = static_cast<int>(s_find[0]);
  int len = attend_len(p, b), n_tiles = attend_tiles(p, len);
  int hr = static_cast<int>(div64(s_find[1], n_tiles + kAItem));
  int at_unit = static_cast<int>(s_find[1] - static_cast<int64_t>(hr) * (n_tiles + kAItem));
  if (tid == 0) {
    info->total = total;
    info->first = u - at_unit;
    info->b = b;
    info->hr = hr;
    info->tiles = at_unit > kAItem ? n_tiles : 0;
  }

  // this lane's vectors of a step: i = 0 .. kLoads - 1
  const int lane_id = wr * 32 + lane;
  auto row_of = [&](int i) { return (i * 32 * WR + lane_id) / kChunks; };
  auto chunk_of = [&](int i) { return (i * 32 * WR + lane_id) % kChunks; };
  // where a group loads whole rows at once, they are kLaneRows apart: the same chunk
  constexpr bool kSameChunk = kChunks <= 32 * WR;
  constexpr int kLaneRows = kSameChunk ? 32 * WR / kChunks : 1;
  const int row0 = row_of(0), chunk0 = chunk_of(0);
  const unsigned to_k = row0 * kPitch + swizzled<T, false, kLong>(row0, chunk0) * 16;
  const unsigned to_v = kHalf + row0 * kPitch + swizzled<T, true, kLong>(row0, chunk0) * 16;
  const int from_k = row0 * p.token_bytes[0] + chunk0 * 16, from_v = row0 * p.token_bytes[1] + chunk0 * 16;
  const int chunk_bytes = chunk0 * PE < p.D ? 16 : 0;
  const int step_blocks = kATile / p.block_size, step_rest = kATile % p.block_size;

  float O[NT][4], m[kH], l[kH];
  unsigned qf[kQRegs ? DP / 16 : 1][4];
  for (; u < u_end; at_unit = 0) {
    if (hr == HR) {
      hr = 0;
      ++b;
      len = attend_len(p, b);
      n_tiles = attend_tiles(p, len);
    }
    const int end_unit = static_cast<int>(min(static_cast<int64_t>(n_tiles + kAItem), at_unit + (u_end - u)));
    const int t0 = max(0, at_unit - kAItem), t1 = end_unit - kAItem;
    u += end_unit - at_unit;
    if (t1 <= t0) continue;  // (the item's first tile is the next CTA's)
    const int kh = hr / p.row_tiles, R0 = (hr % p.row_tiles) * kRows;
    const int lo = attend_first(p, len);
    const int rows = min(kRows, p.rows - R0);  // of the item
    const T* keys = static_cast<const T*>(p.keys) + kh * p.cks[2];
    const T* values = static_cast<const T*>(p.values) + kh * p.cvs[2];
    const int32_t* table = p.tables + b * p.table_ld;
    const int k_group = lo + group * kAKeys;  // the group's first key of tile 0

    // the next step to load: this lane's key of it (lane % 16), its block and place there
    int next_key = k_group + t0 * kATile + (lane & 15);
    int next_block = next_key / p.block_size, next_at = next_key % p.block_size;
    const int end_key = min(len, lo + t1 * kATile);
    auto page_of = [&] { return next_key < end_key ? __ldg(table + next_block) : INT_MIN; };
    auto advance = [&] {
      next_key += kATile;
      next_block += step_blocks;
      next_at += step_rest;
      if (next_at >= p.block_size) next_at -= p.block_size, ++next_block;
    };
    auto issue = [&](int stage, int page, int key, int at) {
      const unsigned sk = ring_at + stage * 2 * kHalf, sv = sk + kHalf;
      const bool there = static_cast<unsigned>(page) < static_cast<unsigned>(p.num_blocks);
      const unsigned live = __ballot_sync(~0u, there) & 0xFFFFu;
      if (lane == 0) masks[stage] = live;
      if (kSameChunk && p.whole_steps && live == 0xFFFFu) {
        const int first = at - (lane & 15);
        const char* fk = reinterpret_cast<const char*>(keys) + from_k +
                         (static_cast<int64_t>(page) * p.block_bytes[0] + static_cast<int64_t>(first) * p.token_bytes[0]);
        const char* fv = reinterpret_cast<const char*>(values) + from_v +
                         (static_cast<int64_t>(page) * p.block_bytes[1] + static_cast<int64_t>(first) * p.token_bytes[1]);
        const unsigned dk = sk + to_k, dv = sk + to_v;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
          constexpr int kStep = kLaneRows * kPitch;
          cp_async16_or_zero((dk ^ (swizzled<T, false, kLong>(i * kLaneRows, 0) * 16)) + i * kStep, fk, chunk_bytes);
          cp_async16_or_zero((dv ^ (swizzled<T, true, kLong>(i * kLaneRows, 0) * 16)) + i * kStep, fv, chunk_bytes);
          fk += kLaneRows * p.token_bytes[0];
          fv += kLaneRows * p.token_bytes[1];
        }
      } else if (live != 0 || __any_sync(~0u, key < end_key)) {
        // (up to 15 keys are before the window of every query: their block may be gone)
        if (!there && key < end_key && (p.window == 0 || key > len - p.Q - p.window)) err |= ASYMSPEC_DATA_BAD_INDEX;
        const int64_t ok = there ? page * p.cks[0] + at * p.cks[1] : 0;
        const int64_t ov = there ? page * p.cvs[0] + at * p.cvs[1] : 0;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
          const int r = row_of(i), ch = chunk_of(i);
          const int64_t rk = __shfl_sync(~0u, ok, r), rv = __shfl_sync(~0u, ov, r);
          const bool on = ((live >> r) & 1u) && ch * PE < p.D;
          const int el = on ? ch * PE : 0;
          cp_async16_or_zero(sk + r * kPitch + swizzled<T, false, kLong>(r, ch) * 16, keys + rk + el, on ? 16 : 0);
          cp_async16_or_zero(sv + r * kPitch + swizzled<T, true, kLong>(r, ch) * 16, values + rv + el, on ? 16 : 0);
        }
      }
      cp_async_commit();
    };
    int next_page = page_of();
    if constexpr (ST > 1) {
      int pages[ST - 1], keys_of[ST - 1], ats[ST - 1];
#pragma unroll
      for (int s = 0; s < ST - 1; ++s) {
        pages[s] = next_page, keys_of[s] = next_key, ats[s] = next_at;
        advance();
        next_page = page_of();
      }
#pragma unroll
      for (int s = 0; s < ST - 1; ++s) issue(s, pages[s], keys_of[s], ats[s]);
    }

    // the item's queries
    for (int e = tid; e < kRows * kChunks; e += kThreadsN) {
      const int r = e / kChunks, ch = e % kChunks;
      const int i = (R0 + r) / p.group, h = kh * p.group + (R0 + r) % p.group;
      const T* src = static_cast<const T*>(p.q) + b * p.qs[0] + i * p.qs[1] + h * p.qs[2] + ch * PE;
      uint4 v = make_uint4(0, 0, 0, 0);
      if (r < rows && ch * PE < p.D) {
        if (p.q_vec) {
          v = *reinterpret_cast<const uint4*>(src);
        } else {
          __align__(16) T x[PE];
#pragma unroll
          for (int k = 0; k < PE; ++k) x[k] = src[k];
          v = *reinterpret_cast<const uint4*>(x);
        }
      }
      const int at = r * (kPitch / static_cast<int>(sizeof(T))) + swizzled<T, false, kLong>(r, ch) * PE;
      if constexpr (BF) {
        *reinterpret_cast<uint4*>(qs + at) = v;
      } else {
        uint4 hi, lw;
        split_tf32(__uint_as_float(v.x), hi.x, lw.x);
        split_tf32(__uint_as_float(v.y), hi.y, lw.y);
        split_tf32(__uint_as_float(v.z), hi.z, lw.z);
        split_tf32(__uint_as_float(v.w), hi.w, lw.w);
        *reinterpret_cast<uint4*>(qs + at) = hi;
        *reinterpret_cast<uint4*>(qs + kRows * DP + at) = lw;
      }
    }
    // of this thread's rows: the last key seen; of the warp's the least, and the windows'
    // largest first
    const int R = R0 + wr * 16, warp_rows = rows - wr * 16;  // (may be none)
    int last[kH];
#pragma unroll
    for (int h = 0; h < kH; ++h) {
      last[h] = h * 8 + g < warp_rows ? len - p.Q + (R + h * 8 + g) / p.group : -1;
      m[h] = -INFINITY;
      l[h] = 0.f;
    }
    const int least = len - p.Q + R / p.group;
    const int from = p.window ? len - p.Q + (R + min(warp_rows, 16) - 1) / p.group - p.window + 1 : 0;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 4; ++e) O[n][e] = 0.f;
    __syncthreads();
    if constexpr (kQRegs) {
      const unsigned at = q_at + (lane & 15) * kPitch + swizzled<T, false, kLong>(lane, lane >> 4) * 16;
#pragma unroll
      for (int k = 0; k < DP / 16; ++k) ldmatrix4(qf[k], chunk_pair<kLong>(at, k));
    }

    int stage = 0;
    for (int t = t0; t < t1; ++t) {
      cp_async_wait<ST - 1 - (ST > 1)>();
      // the group's warps have loaded the step, and are done with the one before
      if constexpr (WR > 1) group_barrier(1 + group, WR * 32);
      else __syncwarp();
      if constexpr (ST > 1) {
        issue(stage == 0 ? ST - 1 : stage - 1, next_page, next_key, next_at);
        advance();
        next_page = page_of();
      } else {
        issue(0, next_page, next_key, next_at);
        advance();
        next_page = page_of();
        cp_async_wait<0>();
        if constexpr (WR > 1) group_barrier(1 + group, WR * 32);
        else __syncwarp();
      }
      const unsigned char* ks = ring + stage * 2 * kHalf;
      const unsigned char* vs = ks + kHalf;
      const unsigned ks_at = ring_at + stage * 2 * kHalf, vs_at = ks_at + kHalf;
      const unsigned live = masks[stage];
      const int k0 = k_group + t * kATile;
      if (live != 0 && warp_rows > 0) {
        // scores of keys 0-7 and 8-15
        float S[2][4];
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int e = 0; e < 4; ++e) S[n][e] = 0.f;
        if constexpr (BF) {
          const unsigned at = ks_at + (((lane >> 4) << 3) + (lane & 7)) * kPitch +
                              swizzled<T, false, kLong>(lane, (lane >> 3) & 1) * 16;
          const unsigned q_lane = q_at + (lane & 15) * kPitch + swizzled<T, false, kLong>(lane, lane >> 4) * 16;
#pragma unroll
          for (int k = 0; k < DP / 16; ++k) {
            unsigned kf[4];
            ldmatrix4(kf, chunk_pair<kLong>(at, k));
            if constexpr (kQRegs) {
              mma_bf16(S[0], qf[k], kf[0], kf[1]);
              mma_bf16(S[1], qf[k], kf[2], kf[3]);
            } else {
              unsigned qv[4];
              ldmatrix4(qv, chunk_pair<kLong>(q_lane, k));
              mma_bf16(S[0], qv, kf[0], kf[1]);
              mma_bf16(S[1], qv, kf[2], kf[3]);
            }
          }
        } else {
          // The sum over a head's elements in an order of its own: of each 16, lane t4 of a
          // quad takes elements 4 t4 .. 4 t4 + 3, two for each of two products.  The matrix
          // unit's running sums are cut, not rounded: the pieces' products have sums of their
          // own, the large ones two, added up in fp32 at the end.
          const float* kf = reinterpret_cast<const float*>(ks);
          const float* qw = reinterpret_cast<const float*>(qs) + wr * 16 * DP;
          const uint4 none = make_uint4(0, 0, 0, 0);
          float large[2][4], small[2][4];
#pragma unroll
          for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) large[n][e] = small[n][e] = 0.f;
#pragma unroll
          for (int k = 0; k < DP / 16; ++k) {
            const int at = g * DP + swizzled<T, false, kLong>(g, 4 * k + t4) * 4;  // (row g + 8: the same chunk)
            const uint4 h0 = *reinterpret_cast<const uint4*>(qw + at);
            const uint4 h1 = kH == 1 ? none : *reinterpret_cast<const uint4*>(qw + at + 8 * DP);
            const uint4 l0 = *reinterpret_cast<const uint4*>(qw + kRows * DP + at);
            const uint4 l1 = kH == 1 ? none : *reinterpret_cast<const uint4*>(qw + kRows * DP + at + 8 * DP);
            const unsigned qh[2][4] = {{h0.x, h1.x, h0.y, h1.y}, {h0.z, h1.z, h0.w, h1.w}};
            const unsigned ql[2][4] = {{l0.x, l1.x, l0.y, l1.y}, {l0.z, l1.z, l0.w, l1.w}};
#pragma unroll
            for (int n = 0; n < 2; ++n) {
              const float4 x = *reinterpret_cast<const float4*>(kf + at + n * 8 * DP);
              unsigned kh4[4], kl4[4];
              split_tf32(x.x, kh4[0], kl4[0]);
              split_tf32(x.y, kh4[1], kl4[1]);
              split_tf32(x.z, kh4[2], kl4[2]);
              split_tf32(x.w, kh4[3], kl4[3]);
              mma_tf32(S[n], qh[0], kh4[0], kh4[1]);
              mma_tf32(large[n], qh[1], kh4[2], kh4[3]);
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                mma_tf32(small[n], ql[e], kh4[2 * e], kh4[2 * e + 1]);
                mma_tf32(small[n], qh[e], kl4[2 * e], kl4[2 * e + 1]);
              }
            }
          }
#pragma unroll
          for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int e = 0; e < 2 * kH; ++e) S[n][e] += large[n][e] + small[n][e];
        }
        const bool whole = live == 0xFFFFu && k0 + kAKeys - 1 <= least && k0 >= from;
#pragma unroll
        for (int h = 0; h < kH; ++h) {
          float top = -INFINITY;
#pragma unroll
          for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              float& s = S[n][2 * h + e];
              s *= p.scale2;
              if (!whole) {
                const int kk = n * 8 + 2 * t4 + e, j = k0 + kk;
                const bool seen = ((live >> kk) & 1u) && j <= last[h] && (p.window == 0 || j > last[h] - p.window);
                s = seen ? s : -INFINITY;
              }
              top = fmaxf(top, s);
            }
          // (m is a reference that scores exceed by 2^kSlack at most: the maximum itself, kept,
          // would rescale the values at most steps, for one of the rows or another)
          if (__any_sync(~0u, top > m[h] + kSlack)) {
            float v = fmaxf(m[h], top);
            v = fmaxf(v, __shfl_xor_sync(~0u, v, 1));
            v = fmaxf(v, __shfl_xor_sync(~0u, v, 2));
            const float f = v == m[h] ? 1.f : ex2(m[h] - v);
            m[h] = v;
            l[h] *= f;
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              O[n][2 * h] *= f;
              O[n][2 * h + 1] *= f;
            }
          }
          const float ref = m[h] == -INFINITY ? 0.f : m[h];
#pragma unroll
          for (int n = 0; n < 2; ++n) {
            S[n][2 * h] = ex2(S[n][2 * h] - ref);
            S[n][2 * h + 1] = ex2(S[n][2 * h + 1] - ref);
            l[h] += S[n][2 * h] + S[n][2 * h + 1];
          }
        }
        if constexpr (BF) {
          // weights in two bf16 pieces (2^-17): in one (2^-9) they would cost as much as the
          // output's own rounding
          unsigned ph[4], pl[4];
#pragma unroll
          for (int n = 0; n < 2; ++n) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
              if (h < kH) split_bf16(S[n][2 * h], S[n][2 * h + 1], ph[2 * n + h], pl[2 * n + h]);
              else ph[2 * n + h] = pl[2 * n + h] = 0;
          }
          const unsigned at = vs_at + (lane & 15) * kPitch + swizzled<T, false, kLong>(lane, lane >> 4) * 16;
#pragma unroll
          for (int n = 0; n < NT / 2; ++n) {
            unsigned vf[4];
            ldmatrix4_trans(vf, chunk_pair<kLong>(at, n));
            mma_bf16(O[2 * n], pl, vf[0], vf[1]);
            mma_bf16(O[2 * n + 1], pl, vf[2], vf[3]);
            mma_bf16(O[2 * n], ph, vf[0], vf[1]);
            mma_bf16(O[2 * n + 1], ph, vf[2], vf[3]);
          }
        } else {
          // Keys 2 t4 and 2 t4 + 1 of each eight are the products' elements t4 and t4 + 4; of each
          // 32 elements of a head, lane group g takes 4 g .. 4 g + 3, one for each of four
          // products.  A step's products are summed by themselves and added to the running
          // values in fp32, which rounds where the matrix unit would cut.
          const float* vf = reinterpret_cast<const float*>(vs);
          unsigned ph[2][4], pl[2][4];
#pragma unroll
          for (int n8 = 0; n8 < 2; ++n8) {
#pragma unroll
            for (int e = 0; e < 4; ++e) ph[n8][e] = pl[n8][e] = 0;
#pragma unroll
            for (int h = 0; h < kH; ++h) {
              split_tf32(S[n8][2 * h], ph[n8][h], pl[n8][h]);
              split_tf32(S[n8][2 * h + 1], ph[n8][2 + h], pl[n8][2 + h]);
            }
          }
#pragma unroll
          for (int i = 0; i < DP / 32; ++i) {
            float sum[4][4];
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
              for (int j = 0; j < 4; ++j) sum[e][j] = 0.f;
#pragma unroll
            for (int n8 = 0; n8 < 2; ++n8) {
              const int r0 = n8 * 8 + 2 * t4, r1 = r0 + 1;
              const float4 x = *reinterpret_cast<const float4*>(vf + r0 * DP + swizzled<T, true, kLong>(r0, 8 * i + g) * 4);
              const float4 y = *reinterpret_cast<const float4*>(vf + r1 * DP + swizzled<T, true, kLong>(r1, 8 * i + g) * 4);
              const float xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                unsigned h0, l0, h1, l1;
                split_tf32(xs[e], h0, l0);
                split_tf32(ys[e], h1, l1);
                mma_tf32(sum[e], pl[n8], h0, h1);
                mma_tf32(sum[e], ph[n8], l0, l1);
                mma_tf32(sum[e], ph[n8], h0, h1);
              }
            }
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
              for (int j = 0; j < 2 * kH; ++j) O[4 * i + e][j] += sum[e][j];
          }
        }
      }
      stage = stage + 1 == ST ? 0 : stage + 1;
    }

    cp_async_wait<0>();
    // Infinities and NaN: a weight of zero times one that its row does not see, or one in
    // two pieces, is a NaN that the formula does not have.  A warp that ends with any works its
    // keys again, one product after another, and leaves out what a row does not see.
    float odd = 0.f;
#pragma unroll
    for (int h = 0; h < kH; ++h)
      if (h * 8 + g < warp_rows) {
        odd = fmaf(0.f, l[h], odd);
#pragma unroll
        for (int n = 0; n < NT; ++n) odd = fmaf(0.f, O[n][2 * h], fmaf(0.f, O[n][2 * h + 1], odd));
      }
    if (__any_sync(~0u, odd != 0.f)) {
#pragma unroll
      for (int h = 0; h < kH; ++h) {
        m[h] = -INFINITY;
        l[h] = 0.f;
#pragma unroll
        for (int n = 0; n < NT; ++n) O[n][2 * h] = O[n][2 * h + 1] = 0.f;
      }
      for (int k = 0; k < (t1 - t0) * kAKeys; ++k) {
        const int j = k_group + (t0 + k / kAKeys) * kATile + k % kAKeys;
        if (j >= len) break;
        const int page = table[j / p.block_size], at = j % p.block_size;
        if (static_cast<unsigned>(page) >= static_cast<unsigned>(p.num_blocks)) continue;
        const T* kr = keys + page * p.cks[0] + at * p.cks[1];
        const T* vr = values + page * p.cvs[0] + at * p.cvs[1];
#pragma unroll 1
        for (int h = 0; h < kH; ++h) {
          const int r = R + min(h * 8 + g, warp_rows - 1);
          const T* qr = static_cast<const T*>(p.q) + b * p.qs[0] + r / p.group * p.qs[1] +
                        (kh * p.group + r % p.group) * p.qs[2];
          float s = 0.f;
          for (int d = t4; d < p.D; d += 4) s = fmaf(to_f32(qr[d]), to_f32(kr[d]), s);
          s += __shfl_xor_sync(~0u, s, 1);
          s += __shfl_xor_sync(~0u, s, 2);
          s *= p.scale2;
          const int end = h ? last[kH - 1] : last[0];
          if (j > end || (p.window != 0 && j <= end - p.window)) continue;
          const float old = h ? m[kH - 1] : m[0], v = fmaxf(old, s), ref = v == -INFINITY ? 0.f : v;
          const float f = v == old ? 1.f : ex2(old - v), w = ex2(s - ref);
          if (h) m[kH - 1] = v, l[kH - 1] = l[kH - 1] * f + (t4 == 0 ? w : 0.f);
          else m[0] = v, l[0] = l[0] * f + (t4 == 0 ? w : 0.f);
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const int d = BF ? n * 8 + 2 * t4 + e : (n >> 2) * 32 + 8 * t4 + 4 * e + (n & 3);
              const float x = d < p.D ? to_f32(vr[d]) : 0.f;
              if (h) O[n][2 + e] = fmaf(w, x, O[n][2 + e] * f);
              else O[n][e] = fmaf(w, x, O[n][e] * f);
            }
        }
      }
    }

    // the groups' parts of the item: each warp leaves its values in its group's ring
    if constexpr (WR > 1) group_barrier(1 + group, WR * 32);
    else __syncwarp();
    float* mine_o = reinterpret_cast<float*>(ring) + wr * 16 * DP;
#pragma unroll
    for (int h = 0; h < kH; ++h) {
      const int r = h * 8 + g;
      float s = l[h];
      s += __shfl_xor_sync(~0u, s, 1);
      s += __shfl_xor_sync(~0u, s, 2);
      if (t4 == 0) {
        s_ml[(group * kRows + wr * 16 + r) * 2] = m[h];
        s_ml[(group * kRows + wr * 16 + r) * 2 + 1] = s;
      }
      float* row = mine_o + r * DP;
      if constexpr (BF) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
          *reinterpret_cast<float2*>(row + ((n ^ (r & 7)) * 8 + 2 * t4)) = make_float2(O[n][2 * h], O[n][2 * h + 1]);
      } else {
#pragma unroll
        for (int i = 0; i < DP / 32; ++i)
#pragma unroll
          for (int e = 0; e < 2; ++e)
            *reinterpret_cast<float4*>(row + (((4 * i + t4) ^ (r & 7)) * 8 + 4 * e)) = make_float4(
                O[4 * i][2 * h + e], O[4 * i + 1][2 * h + e], O[4 * i + 2][2 * h + e], O[4 * i + 3][2 * h + e]);
      }
    }
    __syncthreads();
    const bool all = t0 == 0 && t1 == n_tiles;
    const int part = t0 > 0 ? 2 * c : 2 * c + 1;
    float* ws_ml = reinterpret_cast<float*>(p.ws + kAInfoBytes) + static_cast<size_t>(part) * kRows * 2;
    float* ws_o = reinterpret_cast<float*>(p.ws + kAInfoBytes + kMlBytes) + static_cast<size_t>(part) * kRows * DP;
    for (int e = tid; e < rows * (DP / 4); e += kThreadsN) {
      const int r = e / (DP / 4), d = (e % (DP / 4)) * 4;
      float M = -INFINITY, L = 0.f, x[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < kAGroups; ++w) M = fmaxf(M, s_ml[(w * kRows + r) * 2]);
#pragma unroll
      for (int w = 0; w < kAGroups; ++w) {
        const float mw = s_ml[(w * kRows + r) * 2], lw = s_ml[(w * kRows + r) * 2 + 1];
        const float f = mw == M ? 1.f : ex2(mw - M);
        const float4 o = *reinterpret_cast<const float4*>(
            reinterpret_cast<const float*>(a_smem + w * ST * 2 * kHalf) + r * DP + (((d >> 3) ^ (r & 7)) * 8 + (d & 7)));
        L = fmaf(f, lw, L);
        x[0] = fmaf(f, o.x, x[0]);
        x[1] = fmaf(f, o.y, x[1]);
        x[2] = fmaf(f, o.z, x[2]);
        x[3] = fmaf(f, o.w, x[3]);
      }
      if (all) {
        const float inv = L == 0.f ? 0.f : 1.f / L;
        const int i = (R0 + r) / p.group, h = kh * p.group + (R0 + r) % p.group;
        T* out = static_cast<T*>(p.out) + b * p.os[0] + i * p.os[1] + h * p.os[2] + d;
        if (d < p.D) {  // (D is a multiple of 4)
          __align__(16) T y[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) put(y + k, x[k] * inv);
          if (p.out_vec) {
            if constexpr (BF) *reinterpret_cast<uint2*>(out) = *reinterpret_cast<const uint2*>(y);
            else *reinterpret_cast<float4*>(out) = *reinterpret_cast<const float4*>(y);
          } else {
#pragma unroll
            for (int k = 0; k < 4; ++k) out[k] = y[k];
          }
        }
        if (d == 0 && p.lse)
          p.lse[(static_cast<int64_t>(b) * p.Q + i) * p.heads + h] = lse_of(M, L);
      } else {
        *reinterpret_cast<float4*>(ws_o + r * DP + d) = make_float4(x[0], x[1], x[2], x[3]);
        if (d == 0) *reinterpret_cast<float2*>(ws_ml + r * 2) = make_float2(M, L);
      }
    }
    __syncthreads();
    ++hr;
  }
  if (err && p.err) atomicOr(p.err, err);
}

// The items whose keys lie in several CTAs' shares: one CTA per row of the first CTA that
// went on with an item.  The parts join in the order of the CTAs.
template <typename T, int DP, int kRows>
__global__ void __launch_bounds__(kAJoinThreads) attend_join(const AttendParams p, int ctas) {
  constexpr int kCols = DP / 4, kWays = kAJoinThreads / kCols, kAWarps = kAJoinThreads / 32;
  constexpr size_t kMlBytes = attend_ml_bytes(kRows);
  __shared__ float s_w[kAMaxCtas], s_l[kAMaxCtas], s_red[kAWarps];
  __shared__ __align__(16) float s_x[kAJoinThreads * 4];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int c = blockIdx.x + 1, r = blockIdx.y, tid = threadIdx.x;
  const AttendInfo in = reinterpret_cast<const AttendInfo*>(p.ws)[c];
  if (in.tiles == 0) return;
  const int R0 = (in.hr % p.row_tiles) * kRows, kh = in.hr / p.row_tiles;
  if (R0 + r >= p.rows) return;
  const AttendShares shares(in.total, ctas);
  const int c0 = shares.owner(in.first + kAItem), c1 = shares.owner(in.first + kAItem + in.tiles - 1);
  if (c0 + 1 != c) return;
  const int parts = c1 - c0 + 1;
  const float* ml = reinterpret_cast<const float*>(p.ws + kAInfoBytes);
  const float* os = reinterpret_cast<const float*>(p.ws + kAInfoBytes + kMlBytes);
  auto part_of = [&](int k) { return k == 0 ? 2 * c0 + 1 : 2 * (c0 + k); };
  float M = -INFINITY;
  for (int k = tid; k < parts; k += kAJoinThreads) {
    const float2 x = *reinterpret_cast<const float2*>(ml + (static_cast<size_t>(part_of(k)) * kRows + r) * 2);
    s_w[k] = x.x;
    s_l[k] = x.y;
    M = fmaxf(M, x.x);
  }
#pragma unroll
  for (int d = 16; d; d >>= 1) M = fmaxf(M, __shfl_xor_sync(~0u, M, d));
  if ((tid & 31) == 0) s_red[tid >> 5] = M;
  __syncthreads();
  M = s_red[0];
#pragma unroll
  for (int w = 1; w < kAWarps; ++w) M = fmaxf(M, s_red[w]);
  const int col = tid % kCols, way = tid / kCols;
  float x[4] = {0.f, 0.f, 0.f, 0.f}, L = 0.f;
#pragma unroll 8
  for (int k = way; k < parts; k += kWays) {
    const float f = s_w[k] == M ? 1.f : ex2(s_w[k] - M);
    const float4 o = *reinterpret_cast<const float4*>(os + (static_cast<size_t>(part_of(k)) * kRows + r) * DP + col * 4);
    L = fmaf(f, s_l[k], L);
    x[0] = fmaf(f, o.x, x[0]);
    x[1] = fmaf(f, o.y, x[1]);
    x[2] = fmaf(f, o.z, x[2]);
    x[3] = fmaf(f, o.w, x[3]);
  }
  __syncthreads();
  *reinterpret_cast<float4*>(s_x + tid * 4) = make_float4(x[0], x[1], x[2], x[3]);
  if (col == 0) s_w[way] = L;
  __syncthreads();
  if (way != 0) return;
  L = s_w[0];
  for (int w = 1; w < kWays; ++w) {
    L += s_w[w];
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] += s_x[(w * kCols + col) * 4 + e];
  }
  const float inv = L == 0.f ? 0.f : 1.f / L;
  const int i = (R0 + r) / p.group, h = kh * p.group + (R0 + r) % p.group, d = col * 4;
  T* out = static_cast<T*>(p.out) + in.b * p.os[0] + i * p.os[1] + h * p.os[2] + d;
  if (d < p.D) {
#pragma unroll
    for (int k = 0; k < 4; ++k) put(out + k, x[k] * inv);
  }
  if (d == 0 && p.lse)
    p.lse[(static_cast<int64_t>(in.b) * p.Q + i) * p.heads + h] = lse_of(M, L);
}

}  // namespace asymspec_impl
