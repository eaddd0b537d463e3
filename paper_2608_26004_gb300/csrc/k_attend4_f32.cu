// Instantiations of the attention over a paged cache in 4 bits (see kernel_attend4.cuh).
#include "k_attend.h"
#include "kernel_attend4.cuh"

namespace asymspec_impl {

template <int DP, int NT, int WR, int ST, int PER_SM>
AttendKernels attend4_pick() {
  constexpr int rows = 8 * NT * WR;
  constexpr int smem = static_cast<int>(attend4_smem_bytes(DP, rows, ST, 2));
  static_assert(smem <= kMaxSmem - 8192 && PER_SM * (smem + 1024) <= 228 * 1024, "the rings fit");
  return {reinterpret_cast<const void*>(&attend4_split<DP, NT, WR, ST, PER_SM>),
          reinterpret_cast<const void*>(&attend4_join<float, DP, rows, PER_SM * kASms>), DP, rows, 128 * WR, smem, PER_SM,
          PER_SM * kASms, kATile};
}

// fp32 queries: on the warps' matrix instructions, whose sums stay in registers, as the tensor core's would be cut
// over a whole context (see attend4_split).  As many CTAs an SM as the registers allow.
AttendKernels attend4_kernels_f32(int D, int rows) {
  if (D <= 64)
    return rows <= 8    ? attend4_pick<64, 1, 1, 3, 3>()
           : rows <= 16 ? attend4_pick<64, 2, 1, 3, 3>()
           : rows <= 32 ? attend4_pick<64, 2, 2, 3, 2>()
                        : attend4_pick<64, 2, 4, 3, 1>();
  if (D <= 128)
    return rows <= 8    ? attend4_pick<128, 1, 1, 3, 3>()
           : rows <= 16 ? attend4_pick<128, 2, 1, 3, 2>()
           : rows <= 32 ? attend4_pick<128, 2, 2, 3, 1>()
                        : attend4_pick<128, 2, 4, 3, 1>();
  return rows <= 8 ? attend4_pick<256, 1, 1, 2, 2>() : attend4_pick<256, 2, 1, 3, 1>();
}

}  // namespace asymspec_impl
