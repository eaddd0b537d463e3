// Attention of a few new tokens over a paged cache in 4 bits (asymspec_cache4_attend).
#pragma once

#include "kernel_attend.cuh"
#include "kernel_cache4.cuh"

namespace asymspec_impl {

struct Attend4Params {
  AttendParams a;  // (its keys, values and their strides are not read)
  const char* codes[2];
  const char* scales[2];
  int64_t head_codes[2], head_scales[2];          // strides in bytes: of heads,
  unsigned codes_of[2][2], scales_of[2][2];  // and of blocks and tokens
  float value_scale;
  unsigned divide;  // key / block_size is the high half of 2 key * divide, shifted
  int shift;
  unsigned divide_rows;  // the same for row / group
  int shift_rows;
  bool wide_scales;  // a token's scales of a head are DP / 16 bytes on such boundaries
  bool wide_codes;   // its codes DP / 2 bytes on 32-byte boundaries
};

// 8x8 elements of 16 bits, a row to four lanes, into its columns.
__device__ __forceinline__ unsigned transposed(unsigned x) {
  unsigned y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ unsigned pack_f16(float x, float y) {
  unsigned r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(y), "f"(x));
  return r;
}
__device__ __forceinline__ void mma_f16(float (&c)[4], unsigned a0, unsigned a1, unsigned a2, unsigned a3, unsigned b0,
                                        unsigned b1) {
  asm(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
      "{%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// The bits of x where those of m are set, of y elsewhere (as one instruction, which the compiler did not find).
__device__ __forceinline__ unsigned select_bits(unsigned m, unsigned x, unsigned y) {
  unsigned r;
  asm("lop3.b32 %0, %1, %2, %3, 0xCA;" : "=r"(r) : "r"(m), "r"(x), "r"(y));
  return r;
}
// p + n * size.
__device__ __forceinline__ const char* stepped(const char* p, int n, unsigned size) {
  return p + static_cast<uint64_t>(static_cast<unsigned>(n)) * size;
}
__device__ __forceinline__ void cp_async16(unsigned smem, const void* gmem) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem), "l"(gmem) : "memory");
}
// N = 4, 8 or 16 bytes, or with bytes = 0 zeros (the address is then not read).
template <int N>
__device__ __forceinline__ void cp_async_or_zero(unsigned smem, const void* gmem, int bytes) {
  if constexpr (N == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem), "l"(gmem), "r"(bytes) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(smem), "l"(gmem), "n"(N), "r"(bytes) : "memory");
}

// Dynamic shared memory.  A group's step is kASubs times 16 keys: their codes, their values' codes in rows
// 16 bytes longer than they are (lanes read the rows 2 t of their own then without meeting a bank twice), and
// both's scales, in rows 4 bytes longer where they begin off the boundaries.  Where an item ends, the
// group's ring takes its rows' values.
constexpr int kASubs = 2;
__host__ __device__ constexpr int attend4_sub_bytes(int DP) { return kAKeys * (DP / 2 + DP / 2 + 16 + DP / 8 + 8); }
__host__ __device__ constexpr int attend4_group_bytes(int DP, int rows, int ST) {
  const int ring = ST * kASubs * attend4_sub_bytes(DP);
  return ring > rows * DP * 4 ? ring : rows * DP * 4;
}
__host__ __device__ constexpr int attend4_query_pitch(int DP) { return DP * 2 + 16; }
constexpr size_t attend4_smem_bytes(int DP, int rows, int ST, int pieces) {
  return static_cast<size_t>(kAGroups) * attend4_group_bytes(DP, rows, ST) +
         static_cast<size_t>(rows) * (attend4_query_pitch(DP) * pieces + 4) + kAGroups * ST * 16 + 16 +
         static_cast<size_t>(kAGroups) * rows * 8 + kAGroups * 8 * 8 + 32;
}

// Of 32-bit word N at `p`.
template <int N>
__device__ __forceinline__ void load_words(const unsigned char* p, unsigned (&w)[N]) {
  if constexpr (N % 4 == 0) {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      const uint4 v = *reinterpret_cast<const uint4*>(p + 4 * i);
      w[i] = v.x, w[i + 1] = v.y, w[i + 2] = v.z, w[i + 3] = v.w;
    }
  } else if constexpr (N == 2) {
    const uint2 v = *reinterpret_cast<const uint2*>(p);
    w[0] = v.x, w[1] = v.y;
  } else {
    w[0] = *reinterpret_cast<const unsigned*>(p);
  }
}

// The keys are split evenly over the CTAs and over a CTA's four groups of warps, as
// attend_split's are; this kernel serves fp32 queries (bf16 ones: attend4_tensor).  A step's products are formed
// the other way round: keys, then a head's elements, are the rows of the matrix instructions and up to 8
// queries their columns, so that one kv head's few queries fill them, and the codes become their operands
// in the registers that the lanes load them into: two codes of a byte are two neighbouring elements of a key;
// for the values the bytes of two keys are interleaved first.  e2m1 times e4m3 has 6 significant bits and lies
// between 2^-10 and 2688: fp16 holds it, keys and values are exact; queries, each row times a power of two, are
// two fp16 pieces (2^-22 of an element down to 2^-27 of its row's largest), and so are the weights.  The pools' numbers are left to the scores' factors and
// the end.  The conversion of two codes and its product with their scale take a warp 0.78 cycles of an SM; codes
// that were whole numbers, taken out by masks, took 1.34.
// Bound by latency at few CTAs: 32 requests of 5 queries, a window of 2000, 8 heads of 64 25 us (bf16 keys and
// values, attend_split: 39 in fp32), 3.4 of them the bytes; 64 requests of 64 to 8192 tokens, 32 heads on 8 of 128 70.
// NT: tiles of 8 rows of a warp.
template <int DP, int NT, int WR, int ST, int PER_SM>
__global__ void __launch_bounds__(kAGroups * WR * 32, PER_SM) attend4_split(const __grid_constant__ Attend4Params P) {
  constexpr int kPieces = 2;
  constexpr int kThreadsN = kAGroups * WR * 32, kWarpsN = kAGroups * WR;
  constexpr int kWarpRows = 8 * NT, kRows = kWarpRows * WR;
  constexpr int kKeyRow = DP / 2, kValueRow = DP / 2 + 16, kScaleRow = DP / 16;
  constexpr int kValues = kAKeys * kKeyRow, kScales = kValues + kAKeys * kValueRow;
  constexpr int kSub = attend4_sub_bytes(DP), kStep = kASubs * kSub, kGroup = attend4_group_bytes(DP, kRows, ST);
  constexpr int kQPitch = attend4_query_pitch(DP);
  constexpr int KW = DP / 32;  // words of a lane's part of a key
  constexpr int VW = DP / 64;  // words of a lane's part of a value
  constexpr int MT = DP / 16;  // tiles of 16 elements of a head
  constexpr int kChunks = DP / 32;                 // 16-byte chunks of a key
  constexpr int kLaneRows = 32 * WR / kChunks;     // keys that the group's lanes load at once
  constexpr int kLoads = kASubs * kAKeys > kLaneRows ? kASubs * kAKeys / kLaneRows : 1;
  constexpr int U = NT == 1 ? kASubs : 1;          // sixteens of keys that are worked at together
  constexpr size_t kInfoBytes = attend_info_bytes(PER_SM * kASms), kMlBytes = attend_ml_bytes(kRows, PER_SM * kASms);
  constexpr float kBelow = 12.f, kSlack = 15.f - kBelow;
  constexpr bool kQRegs = kPieces * NT * KW * 4 <= 32;
  static_assert(ST >= 2 && kStep % 16 == 0 && kGroup % 16 == 0, "the ring");
  extern __shared__ __align__(1024) unsigned char a_smem[];
  const AttendParams& p = P.a;
  unsigned char* at_q = a_smem + kAGroups * kGroup;
  float* s_factor = reinterpret_cast<float*>(at_q + kRows * kQPitch * kPieces);
  float* s_ml = s_factor + kRows;
  uint4* masks0 = reinterpret_cast<uint4*>((reinterpret_cast<uintptr_t>(s_ml + kAGroups * kRows * 2) + 15) & ~uintptr_t(15));
  int64_t* s_scan = reinterpret_cast<int64_t*>(masks0 + kAGroups * ST);
  int64_t* s_find = s_scan + kWarpsN;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t4 = lane & 3;
  const int group = warp / WR, wr = warp % WR;  // whose keys; which rows
  // of a step's sixteens of keys: keys that exist; scales that begin off the 4-byte boundaries
  unsigned* masks = reinterpret_cast<unsigned*>(masks0 + group * ST);
  unsigned char* ring = a_smem + group * kGroup;
  const unsigned ring_at = smem_u32(ring);
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
    // (the first CTA that goes on with an item: the one before has its first tile)
    info->tiles = at_unit > kAItem && shares.start(c - 1) <= u - at_unit + kAItem ? n_tiles : 0;
  }

  // what this lane loads of a step: chunk `chunk` of keys load_row + i * kLaneRows and of their values;
  // and of each sixteen the scales of key lane % 16, or of its value
  const int lane_id = wr * 32 + lane;
  const int chunk = lane_id % kChunks, load_row = lane_id / kChunks;
  const bool chunk_on = chunk * 32 < p.D && load_row < kASubs * kAKeys;
  const int what = lane >> 4;
  const unsigned scales_block = P.scales_of[what][0], scales_token = P.scales_of[what][1];
  const int scale_row = P.wide_scales ? kScaleRow : kScaleRow + 4;

  float O[NT][MT][4], m[NT][2], l[NT][2], factor[NT][2];
  unsigned qf[kQRegs ? kPieces : 1][kQRegs ? NT : 1][kQRegs ? KW : 1][4];
  int last[NT][2];
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
    const char* key_codes = P.codes[0] + kh * P.head_codes[0] + chunk * 16;
    const char* value_codes = P.codes[1] + kh * P.head_codes[1] + chunk * 16;
    const char* scales = P.scales[what] + kh * P.head_scales[what];
    const int32_t* table = p.tables + b * p.table_ld;
    const int k_group = lo + group * kAKeys;  // the group's first key of tile 0

    // the next step to load: its first key, and the blocks of the keys that this lane loads of it
    int next_key = k_group + t0 * kATile;
    const int end_key = min(len, lo + t1 * kATile);
    struct Place {
      int page, at;
    };
    auto place = [&](int key) {
      const int block = static_cast<int>(__umulhi(2u * static_cast<unsigned>(key), P.divide) >> P.shift);
      return Place{key < end_key ? __ldg(table + block) : INT_MIN, key - block * p.block_size};
    };
    Place places[kLoads], scale_places[kASubs];
    auto find = [&] {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int r = load_row + i * kLaneRows;
        places[i] = place(next_key + r % kAKeys + r / kAKeys * kATile);
      }
#pragma unroll
      for (int s = 0; s < kASubs; ++s)
        if (WR == 1 || wr == s) scale_places[s] = place(next_key + (lane & 15) + s * kATile);
      next_key += kASubs * kATile;
    };
    auto there = [&](int page) { return static_cast<unsigned>(page) < static_cast<unsigned>(p.num_blocks); };
    auto issue = [&](int stage) {
      const unsigned at = ring_at + stage * kStep;
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int r = load_row + i * kLaneRows;
        const Place x = places[i];
        if (there(x.page) && chunk_on) {
          const unsigned to = at + r / kAKeys * kSub + chunk * 16;
          cp_async16(to + r % kAKeys * kKeyRow,
                     stepped(stepped(key_codes, x.page, P.codes_of[0][0]), x.at, P.codes_of[0][1]));
          cp_async16(to + kValues + r % kAKeys * kValueRow,
                     stepped(stepped(value_codes, x.page, P.codes_of[1][0]), x.at, P.codes_of[1][1]));
        }
      }
#pragma unroll
      for (int s = 0; s < kASubs; ++s) {
        if (WR > 1 && wr != s) continue;
        const Place x = scale_places[s];
        const bool on = there(x.page);
        const unsigned live = __ballot_sync(~0u, on) & 0xFFFFu;
        // (up to 15 keys are before the window of every query: their block may be gone)
        if (!on) {
          const int key = next_key - kASubs * kATile + (lane & 15) + s * kATile;
          if (key < end_key && (p.window == 0 || key > len - p.Q - p.window)) err |= ASYMSPEC_DATA_BAD_INDEX;
        }
        // zeros for a key that does not exist: its codes are what the memory held, finite in any case
        const char* from = scales;
        if (on) from = stepped(stepped(from, x.page, scales_block), x.at, scales_token);
        const unsigned to = at + s * kSub + kScales + lane * scale_row;  // (row lane: values' after the keys')
        if (P.wide_scales) {
          cp_async_or_zero<kScaleRow>(to, from, on ? kScaleRow : 0);
        } else {
          const int off = static_cast<int>(reinterpret_cast<uintptr_t>(from) & 2);
          from -= off;
#pragma unroll
          for (int i = 0; i <= VW; ++i)  // (words that hold some of them)
            if (4 * i < off + p.D / 16) cp_async_or_zero<4>(to + 4 * i, from + 4 * i, on ? 4 : 0);
          const unsigned odd = __ballot_sync(~0u, off != 0);
          if (lane == 0) masks[4 * stage + 2 + s] = odd;
        }
        if (lane == 0) masks[4 * stage + s] = live;
      }
      cp_async_commit();
    };
    find();
#pragma unroll
    for (int s = 0; s < ST - 1; ++s) {
      issue(s);
      find();
    }

    // the item's queries, each row times the power of two that takes its largest element to 2^13; what is left of an
    // element is taken times 2^11, or fp16's smallest step would show in those below 2^-16 of the largest
    for (int r = warp; r < kRows; r += kWarpsN) {
      const int i = (R0 + r) / p.group, h = kh * p.group + (R0 + r) % p.group;
      const float* src = static_cast<const float*>(p.q) + b * p.qs[0] + i * p.qs[1] + h * p.qs[2];
      float x[DP / 32];
      unsigned most = 0;
#pragma unroll
      for (int k = 0; k < DP / 32; ++k) {
        const int d = lane + 32 * k;
        x[k] = r < rows && d < p.D ? src[d] : 0.f;
        most = max(most, __float_as_uint(x[k]) & 0x7FFFFFFFu);
      }
      const unsigned e = min(max(__reduce_max_sync(~0u, most) >> 23, 14u), 254u);
      const float up = __uint_as_float((267u - e) << 23);  // 2^(13 - (e - 127))
      __half* to = reinterpret_cast<__half*>(at_q + r * kQPitch);
#pragma unroll
      for (int k = 0; k < DP / 32; ++k) {
        const float y = x[k] * up;
        const __half hi = __float2half_rn(y);
        to[lane + 32 * k] = hi;
        to[kRows * kQPitch / 2 + lane + 32 * k] = __float2half_rn((y - __half2float(hi)) * 0x1p11f);
      }
      if (lane == 0) s_factor[r] = p.scale2 * __uint_as_float((e - 13u) << 23);
    }
    // of this thread's rows: the last key seen; of the warp's the least, and the windows'
    // largest first
    const int R = R0 + wr * kWarpRows, warp_rows = rows - wr * kWarpRows;  // (may be none)
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int r = n * 8 + 2 * t4 + e;
        last[n][e] = r < warp_rows ? len - p.Q + (R + r) / p.group : -1;
        m[n][e] = -INFINITY;
        l[n][e] = 0.f;
      }
    const int least = len - p.Q + R / p.group;
    const int from = p.window ? len - p.Q + (R + min(warp_rows, kWarpRows) - 1) / p.group - p.window + 1 : 0;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) O[n][i][e] = 0.f;
    __syncthreads();
    const unsigned char* q_lane = at_q + (wr * kWarpRows + g) * kQPitch + t4 * (DP / 2);
    auto query = [&](int piece, int n, int w, unsigned (&x)[4]) {
      load_words<4>(q_lane + (piece * kRows + n * 8) * kQPitch + w * 16, x);
    };
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      factor[n][0] = s_factor[wr * kWarpRows + n * 8 + 2 * t4];
      factor[n][1] = s_factor[wr * kWarpRows + n * 8 + 2 * t4 + 1];
      if constexpr (kQRegs) {
#pragma unroll
        for (int k = 0; k < kPieces; ++k)
#pragma unroll
          for (int w = 0; w < KW; ++w) query(k, n, w, qf[k][n][w]);
      }
    }

    int stage = 0;
    for (int t = t0; t < t1; t += kASubs) {
      cp_async_wait<ST - 2>();
      // the group's warps have loaded the step, and are done with the one before
      if constexpr (WR > 1) group_barrier(1 + group, WR * 32);
      else __syncwarp();
      issue(stage == 0 ? ST - 1 : stage - 1);
      find();
#pragma unroll 1
      for (int s0 = 0; s0 < kASubs; s0 += U) {
        const unsigned char* st = ring + stage * kStep + s0 * kSub;
        unsigned live[U], any = 0;
#pragma unroll
        for (int u2 = 0; u2 < U; ++u2) any |= live[u2] = masks[4 * stage + s0 + u2];
        const int k0 = k_group + (t + s0) * kATile;  // (and kATile further for the second)
        if (any == 0 || warp_rows <= 0) continue;
        // scores of keys g and g + 8 (rows of the products) and of queries 2 t4 and 2 t4 + 1: a
        // lane's part of a key are DP / 4 elements in a row
        float S[U][NT][4];
        {
          unsigned ka[U][KW], kb[U][KW], sa[U][VW], sb[U][VW];
#pragma unroll
          for (int y = 0; y < U; ++y) {
            const unsigned char* sub = st + y * kSub;
            load_words<KW>(sub + g * kKeyRow + t4 * (DP / 8), ka[y]);
            load_words<KW>(sub + (g + 8) * kKeyRow + t4 * (DP / 8), kb[y]);
            const unsigned char* sk = sub + kScales + g * scale_row + t4 * VW;
            const unsigned char* sl = sk + 8 * scale_row;
            if (!P.wide_scales) {
              const unsigned odd = masks[4 * stage + 2 + s0 + y];
              sk += (odd >> g & 1u) * 2;
              sl += (odd >> (g + 8) & 1u) * 2;
            }
            if constexpr (VW == 1) {
              const unsigned v = t4 * 16 < p.D ? sk[0] : 0u, w = t4 * 16 < p.D ? sl[0] : 0u;
              sa[y][0] = e4m3_to_f16(v | v << 8);
              sb[y][0] = e4m3_to_f16(w | w << 8);
            } else {
#pragma unroll
              for (int i = 0; i < VW; i += 2) {
                // (a lane's part of a key, or its half, is of the head or past it)
                const bool on = P.wide_scales || t4 * (DP / 4) + i * 16 < p.D;
                const unsigned v = e4m3_to_f16(on ? *reinterpret_cast<const uint16_t*>(sk + i) : 0u);
                const unsigned w = e4m3_to_f16(on ? *reinterpret_cast<const uint16_t*>(sl + i) : 0u);
                sa[y][i] = __byte_perm(v, v, 0x1010), sa[y][i + 1] = __byte_perm(v, v, 0x3232);
                sb[y][i] = __byte_perm(w, w, 0x1010), sb[y][i + 1] = __byte_perm(w, w, 0x3232);
              }
            }
          }
          float more[U][NT][4], small[U][NT][4];
#pragma unroll
          for (int y = 0; y < U; ++y)
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                S[y][n][e] = more[y][n][e] = small[y][n][e] = 0.f;
              }
#pragma unroll
          for (int w = 0; w < KW; ++w)
#pragma unroll
            for (int y = 0; y < U; ++y) {
              unsigned fa[4], fb[4];
              e2m1_to_f16(ka[y][w], fa);
              e2m1_to_f16(kb[y][w], fb);
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                fa[i] = mul_f16x2(fa[i], sa[y][w / 2]);
                fb[i] = mul_f16x2(fb[i], sb[y][w / 2]);
              }
#pragma unroll
              for (int n = 0; n < NT; ++n) {
                unsigned x[4];
                if constexpr (kQRegs) {
#pragma unroll
                  for (int i = 0; i < 4; ++i) x[i] = qf[0][n][w][i];
                } else {
                  query(0, n, w, x);
                }
                mma_f16(S[y][n], fa[0], fb[0], fa[1], fb[1], x[0], x[1]);
                // (the matrix unit's running sums are cut, not rounded: short ones, added up in fp32)
                mma_f16(more[y][n], fa[2], fb[2], fa[3], fb[3], x[2], x[3]);
                if constexpr (kQRegs) {
#pragma unroll
                  for (int i = 0; i < 4; ++i) x[i] = qf[kPieces - 1][n][w][i];
                } else {
                  query(1, n, w, x);
                }
                mma_f16(small[y][n], fa[0], fb[0], fa[1], fb[1], x[0], x[1]);
                mma_f16(small[y][n], fa[2], fb[2], fa[3], fb[3], x[2], x[3]);
              }
            }
#pragma unroll
          for (int y = 0; y < U; ++y)
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
              for (int e = 0; e < 4; ++e) S[y][n][e] += fmaf(small[y][n][e], 0x1p-11f, more[y][n][e]);
        }
        bool whole = k0 + (U - 1) * kATile + kAKeys - 1 <= least && k0 >= from;
#pragma unroll
        for (int y = 0; y < U; ++y) whole = whole && live[y] == 0xFFFFu;
        // Weights are 2^(s - m), m kBelow below the largest score at the time; only a score kSlack above
        // that raises it (the maximum itself, kept, would rescale the values at most steps, for one
        // of the rows or another).  So weights stay below 2^15, and fp16, whose step is 2^-24 at the
        // smallest, holds one of 2^-36 of a row's largest.
        bool above = false;
        float top[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            top[n][e] = -INFINITY;
#pragma unroll
            for (int y = 0; y < U; ++y)
#pragma unroll
              for (int k = 0; k < 2; ++k) {
                float& s = S[y][n][2 * k + e];
                s *= factor[n][e];
                if (!whole) {
                  const int j = k0 + y * kATile + g + 8 * k;
                  const bool seen = ((live[y] >> (g + 8 * k)) & 1u) && j <= last[n][e] && (p.window == 0 || j > last[n][e] - p.window);
                  s = seen ? s : -INFINITY;
                }
                top[n][e] = fmaxf(top[n][e], s);
              }
            above = above || top[n][e] > m[n][e] + (kBelow + kSlack);
          }
        if (__any_sync(~0u, above)) {
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              float v = top[n][e];
              v = fmaxf(v, __shfl_xor_sync(~0u, v, 4));
              v = fmaxf(v, __shfl_xor_sync(~0u, v, 8));
              v = fmaxf(v, __shfl_xor_sync(~0u, v, 16));
              v = fmaxf(m[n][e], v - kBelow);
              const float f = v == m[n][e] ? 1.f : ex2(m[n][e] - v);
              m[n][e] = v;
              l[n][e] *= f;
#pragma unroll
              for (int i = 0; i < MT; ++i) {
                O[n][i][e] *= f;
                O[n][i][2 + e] *= f;
              }
            }
        }
        // weights, turned so that queries are the columns of the second products
        unsigned wt[U][kPieces][NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float ref = m[n][e] == -INFINITY ? 0.f : m[n][e];
#pragma unroll
            for (int y = 0; y < U; ++y) {
              S[y][n][e] = ex2(S[y][n][e] - ref);
              S[y][n][2 + e] = ex2(S[y][n][2 + e] - ref);
              l[n][e] += S[y][n][e] + S[y][n][2 + e];
            }
          }
#pragma unroll
          for (int y = 0; y < U; ++y)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              const unsigned hi = pack_f16(S[y][n][2 * k], S[y][n][2 * k + 1]);
              wt[y][0][n][k] = transposed(hi);
              const float2 x = f16x2_to_f32(hi);
              wt[y][kPieces - 1][n][k] = transposed(pack_f16(S[y][n][2 * k] - x.x, S[y][n][2 * k + 1] - x.y));
            }
        }
        // values: of keys 2 t4, 2 t4 + 1 and those + 8, the lane's DP / 8 elements in a row from g * DP / 8
        // on; even ones are rows g of the products, odd ones rows g + 8
        const int group_at = VW == 1 ? g / 2 : g * (VW / 2);  // the lane's first group of 16 elements
        const bool head = P.wide_scales || group_at * 16 < p.D;
#pragma unroll
        for (int y = 0; y < U; ++y) {
          const unsigned char* sv = st + y * kSub + kValues + 2 * t4 * kValueRow + g * (DP / 16);
          const unsigned char* ss = st + y * kSub + kScales + (kAKeys + 2 * t4) * scale_row + group_at;
          const unsigned odd = P.wide_scales ? 0u : masks[4 * stage + 2 + s0 + y] >> (16 + 2 * t4);
          unsigned x[4][VW], s2[2][VW == 4 ? 2 : 1];
#pragma unroll
          for (int k = 0; k < 4; ++k) load_words<VW>(sv + ((k & 1) + (k >> 1) * 8) * kValueRow, x[k]);
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const unsigned char* s0p = ss + k * 8 * scale_row;
            const unsigned char* s1p = s0p + scale_row;
            if (!P.wide_scales) {
              s0p += (odd >> (k * 8) & 1u) * 2;
              s1p += (odd >> (k * 8 + 1) & 1u) * 2;
            }
            if constexpr (VW == 4) {
              const unsigned v = head ? *reinterpret_cast<const uint16_t*>(s0p) : 0u;
              const unsigned z = head ? *reinterpret_cast<const uint16_t*>(s1p) : 0u;
              s2[k][0] = e4m3_to_f16(__byte_perm(v, z, 0x0040));
              s2[k][1] = e4m3_to_f16(__byte_perm(v, z, 0x0051));
            } else {
              s2[k][0] = e4m3_to_f16(head ? *s0p | *s1p << 8 : 0);
            }
          }
#pragma unroll
          for (int w = 0; w < VW; ++w) {
            unsigned f[2][2][4];  // key pair, parity of the element
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              const unsigned v = x[2 * k][w], z = x[2 * k + 1][w];
              e2m1_to_f16(select_bits(0x0F0F0F0Fu, v, z << 4), f[k][0]);
              e2m1_to_f16(select_bits(0x0F0F0F0Fu, v >> 4, z), f[k][1]);
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                f[k][0][i] = mul_f16x2(f[k][0][i], s2[k][VW == 4 ? w / 2 : 0]);
                f[k][1][i] = mul_f16x2(f[k][1][i], s2[k][VW == 4 ? w / 2 : 0]);
              }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
              for (int n = 0; n < NT; ++n) {
                float sum[4] = {0.f, 0.f, 0.f, 0.f};
                mma_f16(sum, f[0][0][i], f[0][1][i], f[1][0][i], f[1][1][i], wt[y][kPieces - 1][n][0],
                        wt[y][kPieces - 1][n][1]);
                mma_f16(sum, f[0][0][i], f[0][1][i], f[1][0][i], f[1][1][i], wt[y][0][n][0], wt[y][0][n][1]);
#pragma unroll
                for (int e = 0; e < 4; ++e) O[n][4 * w + i][e] += sum[e];
              }
          }
        }
      }
      stage = stage + 1 == ST ? 0 : stage + 1;
    }
    cp_async_wait<0>();

    // A NaN (a scale, or a query): a weight of zero times one that its row does not see is a NaN that the
    // formula does not have.  A warp that ends with any works its keys again, one after another, and
    // leaves out what a row does not see.
    float odd = 0.f;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 2; ++e)
        if (n * 8 + 2 * t4 + e < warp_rows) {
          odd = fmaf(0.f, l[n][e], odd);
#pragma unroll
          for (int i = 0; i < MT; ++i) odd = fmaf(0.f, O[n][i][e], fmaf(0.f, O[n][i][2 + e], odd));
        }
    if (__any_sync(~0u, odd != 0.f)) {
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          m[n][e] = -INFINITY;
          l[n][e] = 0.f;
#pragma unroll
          for (int i = 0; i < MT; ++i) O[n][i][e] = O[n][i][2 + e] = 0.f;
        }
      for (int k = 0; k < (t1 - t0) * kAKeys; ++k) {
        const int j = k_group + (t0 + k / kAKeys) * kATile + k % kAKeys;
        if (j >= len) break;
        const int page = table[j / p.block_size], at = j % p.block_size;
        if (!there(page)) continue;
        const unsigned char* code[2];
        const unsigned char* scale[2];
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          code[w] = reinterpret_cast<const unsigned char*>(P.codes[w]) + kh * P.head_codes[w] +
                    static_cast<uint64_t>(page) * P.codes_of[w][0] + static_cast<uint64_t>(at) * P.codes_of[w][1];
          scale[w] = reinterpret_cast<const unsigned char*>(P.scales[w]) + kh * P.head_scales[w] +
                     static_cast<uint64_t>(page) * P.scales_of[w][0] + static_cast<uint64_t>(at) * P.scales_of[w][1];
        }
        auto pair = [&](int w, int d) {  // elements d and d + 1, d even
          unsigned f[4];
          e2m1_to_f16(code[w][d / 2], f);
          const unsigned s = scale[w][d / 16];
          return f16x2_to_f32(mul_f16x2(f[0], e4m3_to_f16(s | s << 8)));
        };
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int r = R + min(n * 8 + 2 * t4 + e, warp_rows - 1);
            const float* qr = static_cast<const float*>(p.q) + b * p.qs[0] + r / p.group * p.qs[1] +
                              (kh * p.group + r % p.group) * p.qs[2];
            float s = 0.f;
#pragma unroll 1
            for (int d = 2 * g; d < p.D; d += 16) {
              const float2 x = pair(0, d);
              s = fmaf(qr[d], x.x, s);
              s = fmaf(qr[d + 1], x.y, s);
            }
            s += __shfl_xor_sync(~0u, s, 4);
            s += __shfl_xor_sync(~0u, s, 8);
            s += __shfl_xor_sync(~0u, s, 16);
            s *= p.scale2;
            // (a row that does not see the key takes nothing of it)
            if (j > last[n][e] || (p.window != 0 && j <= last[n][e] - p.window)) continue;
            const float old = m[n][e], v = fmaxf(old, s), ref = v == -INFINITY ? 0.f : v;
            const float f = v == old ? 1.f : ex2(old - v), w = ex2(s - ref);
            m[n][e] = v;
            l[n][e] = l[n][e] * f + (g == 0 ? w : 0.f);
#pragma unroll
            for (int i = 0; i < MT; ++i) {
              const int d = g * (DP / 8) + 2 * i;
              const float2 x = d < p.D ? pair(1, d) : make_float2(0.f, 0.f);
              O[n][i][e] = fmaf(w, x.x, O[n][i][e] * f);
              O[n][i][2 + e] = fmaf(w, x.y, O[n][i][2 + e] * f);
            }
          }
      }
    }

    // the groups' parts of the item: each warp leaves its values in its group's ring
    if constexpr (WR > 1) group_barrier(1 + group, WR * 32);
    else __syncwarp();
    auto chunk_at = [](int ch) { return ch ^ ((ch >> 3) & 7); };  // (of 16 bytes, so that lanes g meet few banks twice)
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int r = wr * kWarpRows + n * 8 + 2 * t4 + e;
        float s = l[n][e];
        s += __shfl_xor_sync(~0u, s, 4);
        s += __shfl_xor_sync(~0u, s, 8);
        s += __shfl_xor_sync(~0u, s, 16);
        if (g == 0) {
          s_ml[(group * kRows + r) * 2] = m[n][e];
          s_ml[(group * kRows + r) * 2 + 1] = s;
        }
        float* row = reinterpret_cast<float*>(ring) + r * DP;
#pragma unroll
        for (int i = 0; i < MT; ++i) {
          const int d = g * (DP / 8) + 2 * i;
          *reinterpret_cast<float2*>(row + chunk_at(d / 4) * 4 + (d & 2)) = make_float2(O[n][i][e], O[n][i][2 + e]);
        }
      }
    __syncthreads();
    const bool all = t0 == 0 && t1 == n_tiles;
    const int part = t0 > 0 ? 2 * c : 2 * c + 1;
    float* ws_ml = reinterpret_cast<float*>(p.ws + kInfoBytes) + static_cast<size_t>(part) * kRows * 2;
    float* ws_o = reinterpret_cast<float*>(p.ws + kInfoBytes + kMlBytes) + static_cast<size_t>(part) * kRows * DP;
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
            reinterpret_cast<const float*>(a_smem + w * kGroup) + r * DP + chunk_at(d / 4) * 4);
        L = fmaf(f, lw, L);
        x[0] = fmaf(f, o.x, x[0]);
        x[1] = fmaf(f, o.y, x[1]);
        x[2] = fmaf(f, o.z, x[2]);
        x[3] = fmaf(f, o.w, x[3]);
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) x[k] *= P.value_scale;
      if (all) {
        const float inv = L == 0.f ? 0.f : 1.f / L;
        const int i = (R0 + r) / p.group, h = kh * p.group + (R0 + r) % p.group;
        float* out = static_cast<float*>(p.out) + b * p.os[0] + i * p.os[1] + h * p.os[2] + d;
        if (d < p.D) {  // (D is a multiple of 4)
          if (p.out_vec) {
            *reinterpret_cast<float4*>(out) = make_float4(x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv);
          } else {
#pragma unroll
            for (int k = 0; k < 4; ++k) out[k] = x[k] * inv;
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

// The items whose keys lie in several CTAs' shares; the parts join in the order of the CTAs.  Up to 16 rows
// (grid.y > 1 of them, or one) a CTA takes a row of the first CTA that went on with an item, if its CTA was one.  With
// more rows most of so many CTAs would end at once (8 kv heads of 32 rows, 608 CTAs: 19,000 of them, 8 us):
// each then looks for those CTAs among all, a few hundred numbers, and takes its turn of their rows.
// CTAS: of the split at most.
template <typename T, int DP, int kRows, int CTAS>
__global__ void __launch_bounds__(kAJoinThreads) attend4_join(const __grid_constant__ AttendParams p, int ctas) {
  constexpr int kCols = DP / 4, kWays = kAJoinThreads / kCols, kAWarps = kAJoinThreads / 32;
  constexpr size_t kInfoBytes = attend_info_bytes(CTAS), kMlBytes = attend_ml_bytes(kRows, CTAS);
  __shared__ float s_w[CTAS], s_l[CTAS], s_red[kAWarps];
  __shared__ __align__(16) float s_x[kAJoinThreads * 4];
  __shared__ uint16_t s_list[CTAS];
  __shared__ int s_count[kAWarps];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const AttendInfo* info = reinterpret_cast<const AttendInfo*>(p.ws);
  const float* ml = reinterpret_cast<const float*>(p.ws + kInfoBytes);
  const float* os = reinterpret_cast<const float*>(p.ws + kInfoBytes + kMlBytes);
  int count = 0;
  const bool direct = gridDim.y > 1 || p.rows == 1;
  if (direct && info[blockIdx.x + 1].tiles == 0) return;
  for (int c0 = 0; c0 < (direct ? 0 : ctas); c0 += kAJoinThreads) {
    const int c = c0 + tid;
    const bool on = c < ctas && info[c].tiles != 0;
    const unsigned which = __ballot_sync(~0u, on);
    if (lane == 0) s_count[warp] = __popc(which);
    __syncthreads();
    int at = count;
#pragma unroll
    for (int w = 0; w < kAWarps; ++w) {
      if (w < warp) at += s_count[w];
      count += s_count[w];
    }
    if (on) s_list[at + __popc(which & ((1u << lane) - 1u))] = static_cast<uint16_t>(c);
    __syncthreads();
  }
  const int rows_most = min(p.rows, kRows);
  for (int w = direct ? 0 : blockIdx.x; w < (direct ? 1 : count * rows_most); w += gridDim.x) {
    const int c = direct ? blockIdx.x + 1 : s_list[w / rows_most], r = direct ? blockIdx.y : w % rows_most;
    const AttendInfo in = info[c];
    const int R0 = (in.hr % p.row_tiles) * kRows, kh = in.hr / p.row_tiles;
    if (R0 + r >= p.rows) continue;
    const AttendShares shares(in.total, ctas);
    const int c0 = c - 1, c1 = shares.owner(in.first + kAItem + in.tiles - 1);
    const int parts = c1 - c0 + 1;
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
    if (lane == 0) s_red[warp] = M;
    __syncthreads();
    M = s_red[0];
#pragma unroll
    for (int k = 1; k < kAWarps; ++k) M = fmaxf(M, s_red[k]);
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
    if (way == 0) {
      L = s_w[0];
      for (int k = 1; k < kWays; ++k) {
        L += s_w[k];
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] += s_x[(k * kCols + col) * 4 + e];
      }
      const float inv = L == 0.f ? 0.f : 1.f / L;
      const int i = (R0 + r) / p.group, h = kh * p.group + (R0 + r) % p.group, d = col * 4;
      T* out = static_cast<T*>(p.out) + in.b * p.os[0] + i * p.os[1] + h * p.os[2] + d;
      if (d < p.D) {
        __align__(16) T y[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) put(y + k, x[k] * inv);
        if (p.out_vec) {
          if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2*>(out) = *reinterpret_cast<const uint2*>(y);
          else *reinterpret_cast<float4*>(out) = *reinterpret_cast<const float4*>(y);
        } else {
#pragma unroll
          for (int k = 0; k < 4; ++k) out[k] = y[k];
        }
      }
      if (d == 0 && p.lse) p.lse[(static_cast<int64_t>(in.b) * p.Q + i) * p.heads + h] = lse_of(M, L);
    }
    __syncthreads();  // (before the next row's numbers)
  }
}

}  // namespace asymspec_impl
