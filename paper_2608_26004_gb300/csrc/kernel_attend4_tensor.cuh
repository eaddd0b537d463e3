// Attention of a few new tokens over a paged cache in 4 bits on the tensor cores' own memory
// (asymspec_cache4_attend, bf16 queries).
#pragma once

#include "kernel_attend4.cuh"

namespace asymspec_impl {

constexpr int kTThreads = 128;
constexpr int kTKeys = 128;  // keys of a step, one a thread: the unit of the split
constexpr unsigned long long kTWaitNs = 200000000ull;
// Steps whose products are summed in tensor memory (a power of two).  The tensor core cuts its running sums and does not
// round them, by 2^-23 at most each 16 keys and always one way: a million keys in one CTA came out 0.2 % short.  So every
// 8192 keys, 2^-14, the sums go to the workspace, where they are added up with rounding.
constexpr int kTSteps = 64;
#ifdef ASYMSPEC_TEST_LATE_PRODUCTS  // (a test's build: every wait, once it has ended, counts as one that gave up)
constexpr bool kTestLate = true;
#else
constexpr bool kTestLate = false;
#endif

__device__ __forceinline__ int tensor_tiles(const AttendParams& p, int len) {
  return max(1, (len - attend_first(p, len) + kTKeys - 1) / kTKeys);
}

// ----------------------------------------------------------- tcgen05

// (Waits until there is room, which CTAs that end make: none waits for another that has begun.)
template <int COLS>
__device__ __forceinline__ void tmem_alloc(unsigned smem) {
  asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem), "n"(COLS) : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
}
template <int COLS>
__device__ __forceinline__ void tmem_free(unsigned at) {
  asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(at), "n"(COLS));
}
__device__ __forceinline__ void tmem_load8(unsigned at, float* r) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7])
               : "r"(at));
}
__device__ __forceinline__ void tmem_store8(unsigned at, const float* r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%8], {%0,%1,%2,%3,%4,%5,%6,%7};" ::"f"(r[0]), "f"(r[1]),
               "f"(r[2]), "f"(r[3]), "f"(r[4]), "f"(r[5]), "f"(r[6]), "f"(r[7]), "r"(at)
               : "memory");
}
__device__ __forceinline__ void tmem_store16(unsigned at, const unsigned (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};" ::"r"(r[0]),
      "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
      "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(at)
      : "memory");
}
__device__ __forceinline__ void tmem_wait_load() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_store() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tensor_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tensor_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_to_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
// All products issued before arrive at `bar` when they are done; and this thread does, so that who waits there
// sees what this thread has seen.
__device__ __forceinline__ void tensor_commit(unsigned long long* bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory");
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
// D (+)= A B, fp16 products and fp32 sums: A in tensor memory, or in shared memory.
__device__ __forceinline__ void tensor_mma_t(unsigned d, unsigned a, uint64_t b, unsigned form, bool add) {
  asm volatile(
      "{ .reg .pred p; setp.ne.u32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p; }" ::"r"(d), "r"(a), "l"(b), "r"(form),
      "r"(static_cast<unsigned>(add))
      : "memory");
}
__device__ __forceinline__ void tensor_mma_s(unsigned d, uint64_t a, uint64_t b, unsigned form, bool add) {
  asm volatile(
      "{ .reg .pred p; setp.ne.u32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p; }" ::"r"(d), "l"(a), "l"(b), "r"(form),
      "r"(static_cast<unsigned>(add))
      : "memory");
}
// Of operands in shared memory in rows of 128 bytes whose 16-byte chunk c lies at c ^ (row % 8): the
// distances of 64-element blocks (`lead`, where rows run along the sum) and of eights of rows (`stride`).
__device__ __forceinline__ uint64_t tensor_operand(unsigned at, unsigned lead, unsigned stride) {
  return static_cast<uint64_t>((at & 0x3FFFF) >> 4) | static_cast<uint64_t>(lead >> 4) << 16 |
         static_cast<uint64_t>(stride >> 4) << 32 | 1ull << 46 | 2ull << 61;
}
// The same of rows of `row` = 32, 64 or 128 bytes along N, the 16-byte chunk c of row r at c ^ weights_turn(row, r).
__device__ __forceinline__ uint64_t tensor_operand_across(unsigned at, int row) {
  const uint64_t kind = row == 128 ? 2 : row == 64 ? 4 : 6;
  return static_cast<uint64_t>((at & 0x3FFFF) >> 4) | 1ull << 16 | static_cast<uint64_t>(row / 2) << 32 | 1ull << 46 | kind << 61;
}
__device__ __forceinline__ int weights_turn(int row, int r) {
  return row == 128 ? r & 7 : row == 64 ? (r >> 1) & 3 : (r >> 2) & 1;
}
// fp16 operands, fp32 result, M = 128; both operands' rows along the sum, or (across) along M and N.
__host__ __device__ constexpr unsigned tensor_form(int n, bool across) {
  return 1u << 4 | (across ? 3u << 15 : 0u) | static_cast<unsigned>(n / 8) << 17 | 8u << 24;
}

// The largest of a warp's numbers; a NaN where all are.
__device__ __forceinline__ float warp_max(float x) {
  float y;
  asm volatile("redux.sync.max.f32 %0, %1, 0xFFFFFFFF;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ bool elected() {
  unsigned r;
  asm volatile("{ .reg .pred p; elect.sync _|p, 0xFFFFFFFF; selp.u32 %0, 1, 0, p; }" : "=r"(r));
  return r != 0;
}
// One warp waits for all, the others go on.
template <int ID>
__device__ __forceinline__ void barrier_sync() { asm volatile("bar.sync %0, 128;" ::"n"(ID) : "memory"); }
template <int ID>
__device__ __forceinline__ void barrier_arrive() { asm volatile("bar.arrive %0, 128;" ::"n"(ID) : "memory"); }

// 32 bytes.
__device__ __forceinline__ void load32(unsigned* r, const char* p) {
  asm volatile("ld.global.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "l"(p));
}
__device__ __forceinline__ void load16(unsigned* r, const char* p) {
  asm volatile("ld.global.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "l"(p));
}
template <int N>
__device__ __forceinline__ void load_scales(unsigned (&r)[N], const char* p) {
  if constexpr (N == 4) load16(r, p);
  else if constexpr (N == 2) asm volatile("ld.global.v2.b32 {%0,%1}, [%2];" : "=r"(r[0]), "=r"(r[1]) : "l"(p));
  else asm volatile("ld.global.b32 %0, [%1];" : "=r"(r[0]) : "l"(p));
}

__host__ __device__ constexpr int tensor_blocks(int DP) { return (DP + 127) / 128; }  // 128s of a head's elements
__host__ __device__ constexpr int tensor_columns(int DP, int NR) {
  const int n = DP / 2 + NR + tensor_blocks(DP) * NR;  // keys, scores, what is summed
  return n <= 64 ? 64 : n <= 128 ? 128 : n <= 256 ? 256 : 512;
}
__host__ __device__ constexpr int tensor_rows(int rows) { return rows < 16 ? 16 : rows; }
__host__ __device__ constexpr int tensor_query_blocks(int DP) { return DP > 64 ? DP / 64 : 1; }  // 64s of elements
constexpr size_t tensor_smem_bytes(int DP, int NR) {
  return static_cast<size_t>(tensor_blocks(DP)) * 32768 + static_cast<size_t>(NR) * (256 + tensor_query_blocks(DP) * 128) +
         static_cast<size_t>(NR) * 4 * 10 + 1024;
}

// The keys are split evenly over the CTAs as attend_split's are, in steps of 128, one a thread.  Of a step, both
// products have the keys' side as their 128 rows and the queries of the kv head as their columns, so a few
// queries cost what one does:
//
//   S = K Q^T     K, 128 keys: codes times scales as fp16 (exact), from the registers into tensor memory
//   O += V^T P^T  V^T, 128 elements of a head: the same in shared memory, a key a row, and the weights P beside it
//
// A thread turns its key and its value into fp16 and has the key's scores, a number for each query.  S of a
// step is formed a step ahead, while the threads turn the values of the step and make its weights, and O is
// while they turn the next keys; codes come from memory a step ahead of that.  O stays in tensor memory, and is
// touched only when a score rises far above its row's reference, and every 64 steps.  The weights are one fp16 piece,
// 2^-11: an eighth of the output's own rounding to bf16; a second piece would double the second product and its stores.
// What it takes, of 16 requests of 4096 to 131072 tokens with 32 rows a kv head (8 of 128): 247 us, the bytes 106, issue
// 48 %, DRAM 48 %, the tensor core a quarter: nothing is full, a step's chain of dependent parts (keys turned, scores
// read, references compared by all threads, weights, values turned) and its barriers are not hidden by the two other
// CTAs of the SM.  64 requests of 64 to 8192 tokens, 4 rows: 44 us, the bytes 18; a step costs 0.55 us an SM (its bytes
// 0.41), an item about three, the launch, the first loads and the join 13 us together.  The same products on the
// warps' matrix instructions (as attend4_split's) took 449 and 56 us; with warps of their own for loading, weighing and
// starting the products, one CTA less an SM or two, 482 and 60.
// RR: rows that an item has at most (NR columns of the products, 16 at least).  FAST: codes and scales lie on
// the vectors' boundaries, D = DP.
template <int DP, int RR, int PER_SM, bool FAST>
__global__ void __launch_bounds__(kTThreads, PER_SM) attend4_tensor(const __grid_constant__ Attend4Params P) {
  using T = __nv_bfloat16;
  constexpr int NR = tensor_rows(RR), MB = tensor_blocks(DP), kCols = tensor_columns(DP, NR);
  constexpr int CW = DP / 8, SW = DP / 64;  // words of a key's codes, and of its scales
  constexpr size_t kInfoBytes = attend_info_bytes(PER_SM * kASms), kMlBytes = attend_ml_bytes(RR, PER_SM * kASms);
  constexpr float kBelow = 7.f, kSlack = 8.f, kGuess = -7.f, kLow = 7.f;
  extern __shared__ __align__(1024) unsigned char a_smem[];
  const AttendParams& p = P.a;
  unsigned char* const s_v = a_smem + (-smem_u32(a_smem) & 1023u);  // (the operands' rows are 1024-byte patterns)
  unsigned char* const s_p = s_v + MB * 32768;
  unsigned char* const s_q = s_p + NR * 256;
  float* const s_m = reinterpret_cast<float*>(s_q + NR * tensor_query_blocks(DP) * 128);
  float* const s_factor = s_m + NR;  // (an item's references, factors and last keys, and what its rows need beside)
  int* const s_last = reinterpret_cast<int*>(s_factor + NR);
  float* const s_red = reinterpret_cast<float*>(s_last + NR);  // [4][NR]
  float* const s_up = s_red + 4 * NR;
  float* const s_fall = s_up + NR;
  float* const s_sub = s_fall + NR;  // what scores are taken less: the reference, or 0 where there is none yet
  __shared__ __align__(8) unsigned long long s_bar[3];  // scores, what is summed; all, after a wait that gave up
  __shared__ unsigned s_tmem;
  __shared__ int64_t s_scan[kTThreads / 32], s_find[2];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int c = blockIdx.x, ctas = gridDim.x;
  const int HR = p.kv_heads * p.row_tiles;
  unsigned err = 0;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  if (tid == 0) {
    mbar_init(&s_bar[0], 2);
    mbar_init(&s_bar[1], 2);
    mbar_init(&s_bar[2], 4);
    fence_mbar_init();
  }
  if (warp == 0) tmem_alloc<kCols>(smem_u32(&s_tmem));

  // this CTA's share of the units, and where it begins
  const int per = (p.B + kTThreads - 1) / kTThreads;
  int64_t mine = 0;
  for (int b = tid * per; b < min((tid + 1) * per, p.B); ++b) {
    const int len = attend_len(p, b);
    if (len != p.lens[b]) err |= ASYMSPEC_DATA_BAD_LENGTH;
    mine += tensor_tiles(p, len) + kAItem;
  }
  int64_t upto = mine;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int64_t o = __shfl_up_sync(~0u, upto, d);
    if (lane >= d) upto += o;
  }
  if (lane == 31) s_scan[warp] = upto;
  tensor_fence_before();
  __syncthreads();
  tensor_fence_after();
  const unsigned tm_k = s_tmem, tm_s = tm_k + DP / 2, tm_o = tm_s + NR;
  const unsigned tm_warp = static_cast<unsigned>(warp * 32) << 16;  // this warp's lanes
  int64_t total = 0;
  for (int w = 0; w < kTThreads / 32; ++w) {
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
      const int64_t n = static_cast<int64_t>(tensor_tiles(p, attend_len(p, b)) + kAItem) * HR;
      if (v < n) break;
      v -= n;
    }
    s_find[0] = b;
    s_find[1] = v;
  }
  __syncthreads();
  AttendInfo* info = reinterpret_cast<AttendInfo*>(p.ws) + c;
  int b = 0, len = 0, n_tiles = 0, hr = 0, at_unit = 0;
  if (u >= u_end) {
    if (tid == 0) info->tiles = 0;
  } else {
    b = static_cast<int>(s_find[0]);
    len = attend_len(p, b), n_tiles = tensor_tiles(p, len);
    hr = static_cast<int>(div64(s_find[1], n_tiles + kAItem));
    at_unit = static_cast<int>(s_find[1] - static_cast<int64_t>(hr) * (n_tiles + kAItem));
    if (tid == 0) {
      info->total = total;
      info->first = u - at_unit;
      info->b = b;
      info->hr = hr;
      // (the first CTA that goes on with an item: the one before has its first tile)
      info->tiles = at_unit > kAItem && shares.start(c - 1) <= u - at_unit + kAItem ? n_tiles : 0;
    }
  }

  unsigned parity_s = 0, parity_o = 0;
  // (a thread that gave up waits no more, and starts no products)
  auto gave_up = [&] { return (err & ASYMSPEC_DATA_TIMEOUT) != 0; };
  auto wait = [&](int which, unsigned& parity) {
    // (looked at once more when the time is over: it may have passed while nothing here ran)
    if (!gave_up() && ((!mbar_wait_bounded(&s_bar[which], parity, kTWaitNs) && !mbar_try_wait(&s_bar[which], parity)) || kTestLate))
      err |= ASYMSPEC_DATA_TIMEOUT;
    parity ^= 1;
    tensor_fence_after();
  };
  const unsigned swizzle = (tid & 7) << 4;
  unsigned char* const v_row = s_v + (tid >> 3) * 1024 + (tid & 7) * 128;  // this thread's value in a 64 of elements
  unsigned char* const p_row = s_p + tid * (NR * 2);  // this thread's weights
  const int p_turn = weights_turn(NR * 2, tid);
  const uint64_t q_operand = tensor_operand(smem_u32(s_q), 16, 1024), p_operand = tensor_operand_across(smem_u32(s_p), NR * 2);
  const uint64_t v_operand = tensor_operand(smem_u32(s_v), 16384, 1024);

  for (; u < u_end; at_unit = 0, ++hr) {
    if (hr == HR) {
      hr = 0;
      ++b;
      len = attend_len(p, b);
      n_tiles = tensor_tiles(p, len);
    }
    const int end_unit = static_cast<int>(min(static_cast<int64_t>(n_tiles + kAItem), at_unit + (u_end - u)));
    const int t0 = max(0, at_unit - kAItem), t1 = end_unit - kAItem;
    u += end_unit - at_unit;
    if (t1 <= t0) continue;  // (the item's first tile is the next CTA's)
    const int kh = hr / p.row_tiles, R0 = (hr % p.row_tiles) * RR;
    const int lo = attend_first(p, len);
    const int rows = min(RR, p.rows - R0);  // of the item
    const int end_key = min(len, lo + t1 * kTKeys);
    const int32_t* table = p.tables + b * p.table_ld;

    // this thread's key of a step: where it is (key), and whether it is there.  Looked up two steps ahead of
    // the one whose keys are turned, loaded one step ahead; values go a step after the keys.
    int next_key = lo + t0 * kTKeys + tid, next_page, next_at;
    auto find = [&] {
      const int block = static_cast<int>(__umulhi(2u * static_cast<unsigned>(next_key), P.divide) >> P.shift);
      next_at = next_key - block * p.block_size;
      next_page = next_key < end_key ? __ldg(table + block) : INT_MIN;
    };
    unsigned kc[CW], ks[SW], vc[CW], vs[SW];
    int page = 0, at = 0, page_v = 0, at_v = 0;
    bool there = false, there_v = false;
    const char* codes[2];
    const char* scales[2];
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      codes[w] = P.codes[w] + kh * P.head_codes[w];
      scales[w] = P.scales[w] + kh * P.head_scales[w];
    }
    auto take = [&] {  // the step that was looked up becomes the one whose keys are loaded
      there = static_cast<unsigned>(next_page) < static_cast<unsigned>(p.num_blocks);
      // (up to 15 keys are before the window of every query: their block may be gone)
      if (!there && next_key < end_key && (p.window == 0 || next_key > len - p.Q - p.window)) err |= ASYMSPEC_DATA_BAD_INDEX;
      // (for a key that does not exist some codes of block 0, finite in any case, and zeros for scales)
      page = there ? next_page : 0, at = there ? next_at : 0;
      next_key += kTKeys;
      find();
    };
    auto load = [&](int w, int page_of, int at_of, unsigned (&code)[CW], unsigned (&scale)[SW]) {
      const char* from = stepped(stepped(codes[w], page_of, P.codes_of[w][0]), at_of, P.codes_of[w][1]);
      const char* scales_at = stepped(stepped(scales[w], page_of, P.scales_of[w][0]), at_of, P.scales_of[w][1]);
      if constexpr (FAST) {
#pragma unroll
        for (int i = 0; i < CW; i += 8) load32(code + i, from + 4 * i);
        load_scales<SW>(scale, scales_at);
      } else {
#pragma unroll
        for (int i = 0; i < CW; i += 4) {
          if (i * 8 < p.D) load16(code + i, from + 4 * i);
          else code[i] = code[i + 1] = code[i + 2] = code[i + 3] = 0;
        }
#pragma unroll
        for (int i = 0; i < SW; ++i) {
          scale[i] = 0;
          if (i * 64 < p.D) scale[i] = *reinterpret_cast<const uint16_t*>(scales_at + 4 * i);
          if (i * 64 + 32 < p.D) scale[i] |= static_cast<unsigned>(*reinterpret_cast<const uint16_t*>(scales_at + 4 * i + 2)) << 16;
        }
      }
    };
    auto turn_keys = [&] {  // into tensor memory, and the next step's are loaded
#pragma unroll
      for (int i = 0; i < SW; ++i) ks[i] = there ? ks[i] : 0u;
#pragma unroll
      for (int i = 0; i < CW; i += 4) {
        unsigned f[16];
        const unsigned s2 = e4m3_to_f16(ks[i / 8] >> (i % 8 ? 16 : 0));
        const unsigned sa = __byte_perm(s2, s2, 0x1010), sb = __byte_perm(s2, s2, 0x3232);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          unsigned x[4];
          e2m1_to_f16(kc[i + w], x);
#pragma unroll
          for (int k = 0; k < 4; ++k) f[4 * w + k] = mul_f16x2(x[k], w < 2 ? sa : sb);
        }
        tmem_store16(tm_k + tm_warp + 4 * i, f);
      }
      there_v = there, page_v = page, at_v = at;
      take();
      load(0, page, at, kc, ks);
      tmem_wait_store();
    };
    // Warps 1 to 3 say that a step's keys are turned and go on; warp 0 looks for that later, when it need not wait,
    // and starts the products.  Neighbouring steps have a barrier each: without the wait for the scores (after one
    // that gave up) a warp may be a step ahead of warp 0, but no more, as each step has a barrier of the CTA; with
    // one for all steps its second arrival would stand in for another's.
    auto keys_turned = [&](int step) {
      tensor_fence_before();
      if (warp == 0) return;
      step & 1 ? barrier_arrive<2>() : barrier_arrive<1>();
    };
    auto start_scores = [&](int step) {
      if (warp != 0) return;
      step & 1 ? barrier_sync<2>() : barrier_sync<1>();
      if (elected() && !gave_up()) {
        tensor_fence_after();
#pragma unroll
        for (int k = 0; k < DP / 16; ++k)
          tensor_mma_t(tm_s, tm_k + k * 8, q_operand + ((k >> 2) * (NR * 128) + (k & 3) * 32) / 16, tensor_form(NR, false),
                       k > 0);
        tensor_commit(&s_bar[0]);
      }
      __syncwarp();
    };
    find();
    take();
    load(0, page, at, kc, ks);
    load(1, page, at, vc, vs);

    // the item's queries, each row times the power of two that takes its largest element to 2^13
    const int least = len - p.Q + R0 / p.group;
    const int from = p.window ? len - p.Q + (R0 + rows - 1) / p.group - p.window + 1 : 0;
    // A first reference: if every row sees all keys of the first step, kGuess is close enough to most rows'
    // largest scores (0 to 8) and saves looking for them; a row whose largest of a warp's 32 is below that, or that
    // has one above, raises the references all the same.  So a row's largest weight is never below 2^kBelow: fp16
    // loses 2^-25 at most of each small one, which many keys may have.
    const bool guess = lo + (t0 + 1) * kTKeys - 1 <= least && lo + t0 * kTKeys >= from && lo + (t0 + 1) * kTKeys <= end_key;
    constexpr int kBatch = RR / 4 < 4 ? RR / 4 : 4;  // rows of a warp that are on their way together
#pragma unroll 1
    for (int r0 = warp; r0 < rows; r0 += 4 * kBatch) {
      uint16_t y[kBatch][DP / 32];
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        const int R = R0 + min(r0 + 4 * k, rows - 1);
        const int i = static_cast<int>(__umulhi(2u * static_cast<unsigned>(R), P.divide_rows) >> P.shift_rows);
        const uint16_t* src = static_cast<const uint16_t*>(p.q) + b * p.qs[0] + i * p.qs[1] +
                              (kh * p.group + R - i * p.group) * p.qs[2] + lane;
#pragma unroll
        for (int d = 0; d < DP; d += 32) y[k][d / 32] = lane + d < p.D ? src[d] : uint16_t(0);
      }
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        const int r = r0 + 4 * k;
        if (r >= rows) continue;
        float x[DP / 32];
        unsigned most = 0;
#pragma unroll
        for (int d = 0; d < DP / 32; ++d) {
          x[d] = __uint_as_float(static_cast<unsigned>(y[k][d]) << 16);
          most = max(most, __float_as_uint(x[d]) & 0x7FFFFFFFu);
        }
        const unsigned e = min(max(__reduce_max_sync(~0u, most) >> 23, 14u), 254u);
        const float up = __uint_as_float((267u - e) << 23);  // 2^(13 - (e - 127))
#pragma unroll
        for (int d = 0; d < DP / 32; ++d)
          *reinterpret_cast<__half*>(s_q + (d >> 1) * (NR * 128) + r * 128 +
                                     (((lane + 32 * (d & 1)) * 2) ^ ((r & 7) << 4))) = __float2half_rn(x[d] * up);
        if (lane == 0) s_factor[r] = p.scale2 * __uint_as_float((e - 13u) << 23);
      }
    }
    if (tid < rows) {
      s_m[tid] = guess ? kGuess : -INFINITY;
      s_sub[tid] = guess ? kGuess : 0.f;
      s_last[tid] = len - p.Q + (R0 + tid) / p.group;
    }
    if (tid >= rows && tid < RR) s_factor[tid] = s_sub[tid] = 0.f;  // (scores beyond `rows` are 0 or NaN)
    float l[RR];
#pragma unroll
    for (int n = 0; n < RR; ++n) l[n] = 0.f;
    bool bad_values = false;  // a value with a NaN
    bool fresh = !guess;      // a row without a reference
    const bool few = RR == 8 && rows <= RR / 2;
    // The item's part in the workspace: its sums, each element of a head its thread's.  (An item that is all this CTA's
    // has the place of the one that the next CTA goes on with, which is the CTA's last.)
    auto part = [&] { return static_cast<size_t>(t0 > 0 ? 2 * c : 2 * c + 1); };
    auto sums_at = [&] { return reinterpret_cast<float*>(p.ws + kInfoBytes + kMlBytes) + part() * RR * DP + tid; };
    fence_to_async();
    turn_keys();
    keys_turned(t0);
    start_scores(t0);

    for (int t = t0; t < t1; ++t) {
      const int j = lo + t * kTKeys + tid;  // this thread's key
      const bool live = there_v;
      wait(0, parity_s);
      float S[RR];
#pragma unroll
      for (int n = 0; n < RR; n += 8) tmem_load8(tm_s + tm_warp + n, S + n);
      // the next step's keys, while the scores come
      if (t + 1 < t1) turn_keys();
      tmem_wait_load();
      if (t + 1 < t1) keys_turned(t + 1);
      if (t > t0) wait(1, parity_o);  // (O of the step before: its weights and values have been read)
      // Values, while the scores wait in registers (after the weights, us of 8 requests of 4096 to 32768 tokens, 64 heads
      // on 8 or fewer: heads of 128 at 8, 16, 32 and 64 rows 42.5, 52.6, 73.9, 124 as it is and 44.2, 54.6, 76.8, 129
      // after; of 64 33.7, 45.8, 68.6, 110 and 36.2, 45.6, 71.3, 114; of 256 82.8, 88.3, 113, 241 and 83.7, 97.1, 119,
      // 239).  A NaN is left out of the products, where a weight of zero would make it one in rows that do not see it.
#pragma unroll
      for (int i = 0; i < SW; ++i) {
        vs[i] = live ? vs[i] : 0u;
        const unsigned nan = ((vs[i] & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u;
        if (nan) {
          vs[i] &= ~((nan >> 7) * 0xFFu);
          bad_values = true;
        }
      }
#pragma unroll
      for (int w = 0; w < CW; ++w) {
        const unsigned s2 = e4m3_to_f16(vs[w / 8] >> (w % 8 >= 4 ? 16 : 0));
        const unsigned s = __byte_perm(s2, s2, w % 4 < 2 ? 0x1010 : 0x3232);
        unsigned x[4];
        e2m1_to_f16(vc[w], x);
#pragma unroll
        for (int k = 0; k < 4; ++k) x[k] = mul_f16x2(x[k], s);
        *reinterpret_cast<uint4*>(v_row + (w / 8) * 16384 + (((w % 8) * 16) ^ swizzle)) = make_uint4(x[0], x[1], x[2], x[3]);
      }
      if (t + 1 < t1) {
        load(1, page_v, at_v, vc, vs);
        start_scores(t + 1);
      }
      // scores less their references
      auto less = [&] {
#pragma unroll
        for (int n = 0; n < RR; n += 4) {
          if (few && n >= RR / 2) continue;
          const float4 f = *reinterpret_cast<const float4*>(s_factor + n), m = *reinterpret_cast<const float4*>(s_sub + n);
          S[n] = fmaf(S[n], f.x, -m.x);
          S[n + 1] = fmaf(S[n + 1], f.y, -m.y);
          S[n + 2] = fmaf(S[n + 2], f.z, -m.z);
          S[n + 3] = fmaf(S[n + 3], f.w, -m.w);
        }
      };
      const int k0 = lo + t * kTKeys;
      const bool whole = __all_sync(~0u, live) && k0 + kTKeys - 1 <= least && k0 >= from;
      auto hide = [&] {  // what a row does not see
#pragma unroll
        for (int n = 0; n < RR; ++n) {
          if (n >= rows) continue;
          const int last = s_last[n];
          if (!live || j > last || (p.window != 0 && j <= last - p.window)) S[n] = -INFINITY;
        }
      };
      less();
      if (!whole) hide();
      float top = -INFINITY;
#pragma unroll
      for (int n = 0; n < RR; n += 4)
        if (!few || n < RR / 2) top = fmaxf(fmaxf(top, fmaxf(S[n], S[n + 1])), fmaxf(S[n + 2], S[n + 3]));
      bool raise = top > kBelow + kSlack;
      if (fresh) {
#pragma unroll
        for (int n = 0; n < RR; ++n)
          if (n < rows) raise = raise || (S[n] > -INFINITY && s_m[n] == -INFINITY);
      } else if (t == t0) {
#pragma unroll
        for (int n = 0; n < RR; ++n)
          if (n < rows) {
            const bool low = !(warp_max(S[n]) >= kLow);  // (all lanes take part)
            raise = raise || low;
          }
      }
      // (sums go to the workspace now, and the products' begin anew)
      const bool put_by = t > t0 && ((t - t0) & (kTSteps - 1)) == 0;
      if (__syncthreads_or(raise || put_by)) {
        // references rise: each row's to kBelow under its largest score, and what has been summed goes down
#pragma unroll
        for (int n = 0; n < RR; ++n) {
          if (n >= rows) continue;
          const float v = warp_max(S[n]);
          if (lane == 0) s_red[warp * NR + n] = v;
        }
        __syncthreads();
        for (int n = tid; n < rows; n += kTThreads) {
          const float v = fmaxf(fmaxf(s_red[n], s_red[NR + n]), fmaxf(s_red[2 * NR + n], s_red[3 * NR + n]));
          // (a row that has nothing summed yet: to wherever its scores are, if there are any)
          const bool empty = t == t0 || s_m[n] == -INFINITY, none = empty && !(v > -INFINITY);
          const float up = none ? 0.f : empty ? v - kBelow : fmaxf(v - kBelow, 0.f);
          s_m[n] = none ? -INFINITY : s_sub[n] + up;
          s_sub[n] = none ? 0.f : s_sub[n] + up;
          s_up[n] = up;
          s_fall[n] = empty || up == 0.f ? 1.f : ex2(-up);
        }
        __syncthreads();
        fresh = false;
#pragma unroll
        for (int n = 0; n < RR; ++n)
          if (n < rows) {
            l[n] *= s_fall[n];
            S[n] -= s_up[n];
            fresh = fresh || s_m[n] == -INFINITY;
          }
        if (t > t0) {
          const bool kept = t - t0 > kTSteps;
          float* const ws_o = sums_at();
#pragma unroll 1
          for (int mb = 0; mb < MB; ++mb)
#pragma unroll 1
            for (int n = 0; n < rows; n += 8) {
              float o[8];
              tmem_load8(tm_o + mb * NR + tm_warp + n, o);
              tmem_wait_load();
#pragma unroll
              for (int e = 0; e < 8; ++e) {
                const float fall = n + e < rows ? s_fall[n + e] : 1.f;
                o[e] *= fall;
                if ((DP >= 128 || tid < DP) && (kept || put_by)) {
                  float* const sum = ws_o + (n + e) * DP + mb * 128;
                  const float old = kept ? *sum * fall : 0.f;
                  *sum = put_by ? old + o[e] : old;
                }
              }
              tmem_store8(tm_o + mb * NR + tm_warp + n, o);
            }
          tmem_wait_store();
        }
      }
#pragma unroll
      for (int n = 0; n < RR; n += 8) {
        unsigned w[4] = {0, 0, 0, 0};
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
          if (few && n + e >= RR / 2) continue;
          const float w0 = ex2(S[n + e]), w1 = ex2(S[n + e + 1]);
          l[n + e] += w0;
          l[n + e + 1] += w1;
          w[e / 2] = pack_f16(w0, w1);
        }
        // (a key a row, as the values: one store for 8 queries; a query a row took 16-bit stores, 261 us for 249)
        *reinterpret_cast<uint4*>(p_row + ((n / 8) ^ p_turn) * 16) = make_uint4(w[0], w[1], w[2], w[3]);
      }
      fence_to_async();
      tensor_fence_before();
      if (warp == 1) {
        barrier_sync<3>();
        if (elected() && !gave_up()) {
          tensor_fence_after();
#pragma unroll
          for (int mb = 0; mb < MB; ++mb)
#pragma unroll
            for (int k = 0; k < kTKeys / 16; ++k)
              tensor_mma_s(tm_o + mb * NR, v_operand + (mb * 32768 + k * 2048) / 16,
                           p_operand + k * (NR * 32) / 16, tensor_form(NR, true), (t > t0 && !put_by) || k > 0);
          tensor_commit(&s_bar[1]);
        }
        __syncwarp();
      } else {
        barrier_arrive<3>();
      }
    }

    // the rows' sums over the threads
#pragma unroll
    for (int n = 0; n < RR; ++n) {
      if (n >= rows) continue;
      float v = l[n];
#pragma unroll
      for (int d = 16; d; d >>= 1) v += __shfl_xor_sync(~0u, v, d);
      if (lane == 0) s_red[warp * NR + n] = v;
    }
    const bool nans = __syncthreads_or(bad_values);
    const bool all = t0 == 0 && t1 == n_tiles;
    float* ws_ml = reinterpret_cast<float*>(p.ws + kInfoBytes) + part() * RR * 2;
    float* const ws_o = sums_at();
    // a row's sum, and what its values are taken times
    if (tid < rows) {
      const int n = tid;
      const float L = s_red[n] + s_red[NR + n] + s_red[2 * NR + n] + s_red[3 * NR + n];
      s_up[n] = !all ? P.value_scale : L == 0.f ? 0.f : P.value_scale / L;
      if (!all) {
        *reinterpret_cast<float2*>(ws_ml + n * 2) = make_float2(s_m[n], L);
      } else if (p.lse) {
        const int i = (R0 + n) / p.group, h = kh * p.group + R0 + n - i * p.group;
        p.lse[(static_cast<int64_t>(b) * p.Q + i) * p.heads + h] = lse_of(s_m[n], L);
      }
    }
    wait(1, parity_o);
    if (nans) {
      // a value's NaN that was left out of the products, in the rows that see it
#pragma unroll 1
      for (int mb = 0; mb < MB; ++mb) {
        const int d = mb * 128 + tid;
        uint64_t hit = 0;
        for (int j = lo + t0 * kTKeys; j < end_key; ++j) {
          const int block = j / p.block_size, pg = table[block];
          if (static_cast<unsigned>(pg) >= static_cast<unsigned>(p.num_blocks) || d >= p.D) continue;
          const char* sc = stepped(stepped(scales[1], pg, P.scales_of[1][0]), j - block * p.block_size, P.scales_of[1][1]);
          if ((sc[d / 16] & 0x7F) == 0x7F)
            for (int n = 0; n < rows; ++n)
              if (j <= s_last[n] && (p.window == 0 || j > s_last[n] - p.window)) hit |= 1ull << n;
        }
#pragma unroll 1
        for (int n = 0; n < rows; n += 8) {
          __syncwarp();
          float o[8];
          tmem_load8(tm_o + mb * NR + tm_warp + n, o);
          tmem_wait_load();
#pragma unroll
          for (int e = 0; e < 8; ++e) o[e] = hit >> (n + e) & 1 ? NAN : o[e];
          tmem_store8(tm_o + mb * NR + tm_warp + n, o);
        }
      }
      tmem_wait_store();
    }
    // A CTA in which a thread gave up: nothing of the item is right, nor of a later one.  NaN, which the join carries.
    const bool late = __syncthreads_or(gave_up());
    if (late && tid < rows) {
      s_up[tid] = NAN;
      if (!all) {
        ws_ml[tid * 2 + 1] = NAN;
      } else if (p.lse) {
        const int i = (R0 + tid) / p.group;
        p.lse[(static_cast<int64_t>(b) * p.Q + i) * p.heads + kh * p.group + R0 + tid - i * p.group] = NAN;
      }
    }
    if (late) __syncthreads();
    int h = R0 % p.group;  // the row's head, of the kv head's, and its output
    T* out = static_cast<T*>(p.out) + b * p.os[0] + R0 / p.group * p.os[1] + (kh * p.group + h) * p.os[2] + tid;
    const int64_t next_query = p.os[1] - (p.group - 1) * p.os[2];
#pragma unroll 1
    for (int n0 = 0; n0 < rows; n0 += 8) {
      float o[MB][8];
#pragma unroll
      for (int mb = 0; mb < MB; ++mb) tmem_load8(tm_o + mb * NR + tm_warp + n0, o[mb]);
      tmem_wait_load();
      if (t1 - t0 > kTSteps) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
#pragma unroll
          for (int mb = 0; mb < MB; ++mb)
            if (DP >= 128 || tid < DP) o[mb][e] += ws_o[(n0 + e) * DP + mb * 128];
      }
      if (!all) {
        // (the rows past the item's last one have room there too)
#pragma unroll
        for (int e = 0; e < 8; ++e)
#pragma unroll
          for (int mb = 0; mb < MB; ++mb)
            if (DP >= 128 || tid < DP) ws_o[(n0 + e) * DP + mb * 128] = late ? NAN : o[mb][e] * P.value_scale;
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          if (n0 + e >= rows) continue;
          const float f = s_up[n0 + e];
#pragma unroll
          for (int mb = 0; mb < MB; ++mb)
            if (mb * 128 + tid < p.D) put(out + mb * 128, f == 0.f ? 0.f : o[mb][e] * f);
          const bool turn = ++h == p.group;
          out += turn ? next_query : p.os[2];
          if (turn) h = 0;
        }
      }
    }
    tensor_fence_before();
    __syncthreads();
    tensor_fence_after();
  }
  if (err && p.err) atomicOr(p.err, err);
  if (__syncthreads_or(gave_up())) {
    // products may be under way, of what is freed here
    if (warp < 2 && elected()) tensor_commit(&s_bar[2]);
    mbar_wait_bounded(&s_bar[2], 0, kTWaitNs);
    __syncthreads();
  }
  if (warp == 0) tmem_free<kCols>(tm_k);
}

}  // namespace asymspec_impl
