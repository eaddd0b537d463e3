// Instantiations of the attention over a paged cache (see kernel_attend.cuh).
#include "kernel_attend.cuh"
#include "k_attend.h"

namespace asymspec_impl {

template <int DP, int WR, int ST, int PER_SM, int kH = 2>
AttendKernels attend_pick() {
  constexpr int smem = static_cast<int>(attend_smem_bytes<float>(DP, WR, ST));
  static_assert(smem <= kMaxSmem - 8192 && PER_SM * (smem + 1024) <= 228 * 1024, "the rings fit");
  static_assert(PER_SM * 152 <= kAMaxCtas, "the workspace has room");
  return {reinterpret_cast<const void*>(&attend_split<float, DP, WR, ST, PER_SM, kH>),
          reinterpret_cast<const void*>(&attend_join<float, DP, 16 * WR>), DP, 16 * WR, 128 * WR, smem, PER_SM};
}

// As for bf16 (three CTAs an SM instead of two at 16 rows of 64: a window of 2000, 32 requests
// of 5 queries, 49 to 45 us), with two warps for a group's rows at most (the operands' pieces
// leave no registers for more).  Two CTAs an SM with one step a ring are faster than one with
// three at 16 rows of 128: 64 requests of 64 to 8192 tokens 186 us against 226, 256 of 16 to 300
// 89 against 124.  256 elements leave room for one CTA and one step.
// Up to 8 rows (half of the matrix instructions' 16) the other half's softmax, pieces and sums are
// left out: that window 39.1 to 37.1 us, heads of 128 186 to 162, of 256 632 to 547.
AttendKernels attend_kernels_f32(int D, int rows) {
  if (rows <= 8)
    return D <= 64    ? attend_pick<64, 1, 2, 3, 1>()
           : D <= 128 ? attend_pick<128, 1, 1, 2, 1>()
                      : attend_pick<256, 1, 1, 1, 1>();
  if (D <= 64) return rows <= 16 ? attend_pick<64, 1, 2, 3>() : attend_pick<64, 2, 2, 2>();
  if (D <= 128) return rows <= 16 ? attend_pick<128, 1, 1, 2>() : attend_pick<128, 2, 2, 1>();
  return attend_pick<256, 1, 1, 1>();
}

}  // namespace asymspec_impl
