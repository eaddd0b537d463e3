// Instantiations of the attention over a paged cache (see kernel_attend.cuh).
#include "kernel_attend.cuh"
#include "k_attend.h"

namespace asymspec_impl {

template <int DP, int MT, int ST>
AttendKernels attend_pick() {
  constexpr int smem = static_cast<int>(attend_smem_bytes<float>(DP, MT, ST));
  static_assert(smem <= kMaxSmem - 8192, "the rings fit");
  return {reinterpret_cast<const void*>(&attend_split<float, DP, MT, ST>),
          reinterpret_cast<const void*>(&attend_join<float, DP, MT>), DP, 16 * MT, smem,
          smem <= 112 * 1024 ? 2 : 1};
}

AttendKernels attend_kernels_f32(int D, int rows) {
  if (D <= 64) return rows <= 16 ? attend_pick<64, 1, 3>() : attend_pick<64, 2, 2>();
  if (D <= 128) return rows <= 16 ? attend_pick<128, 1, 3>() : attend_pick<128, 2, 2>();
  return attend_pick<256, 1, 1>();
}

}  // namespace asymspec_impl
