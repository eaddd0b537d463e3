// Instantiations of the attention over a paged cache (see kernel_attend.cuh).
#include "kernel_attend.cuh"
#include "k_attend.h"

namespace asymspec_impl {

template <int DP, int WR, int ST, int PER_SM>
AttendKernels attend_pick() {
  constexpr int smem = static_cast<int>(attend_smem_bytes<float>(DP, WR, ST));
  static_assert(smem <= kMaxSmem - 8192 && PER_SM * (smem + 1024) <= 228 * 1024, "the rings fit");
  static_assert(PER_SM * 152 <= kAMaxCtas, "the workspace has room");
  return {reinterpret_cast<const void*>(&attend_split<float, DP, WR, ST, PER_SM>),
          reinterpret_cast<const void*>(&attend_join<float, DP, 16 * WR>), DP, 16 * WR, 128 * WR, smem, PER_SM};
}

// As for bf16 (three CTAs an SM instead of two at 16 rows of 64: a window of 2000, 32 requests
// of 5 queries, 49 to 45 us), with two warps for a group's rows at most (the operands' pieces
// leave no registers for more); a key of 256 elements leaves room for one step a ring.
AttendKernels attend_kernels_f32(int D, int rows) {
  if (D <= 64) return rows <= 16 ? attend_pick<64, 1, 2, 3>() : attend_pick<64, 2, 2, 2>();
  if (D <= 128) return rows <= 16 ? attend_pick<128, 1, 3, 1>() : attend_pick<128, 2, 2, 1>();
  return attend_pick<256, 1, 1, 1>();
}

}  // namespace asymspec_impl
