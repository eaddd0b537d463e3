// The attention kernels of one head size and row tile, as the host launches them.
#pragma once

#include <cstddef>

namespace asymspec_impl {

struct AttendKernels {
  const void *split, *join;
  int DP, rows, threads, smem, ctas_per_sm;
};

// The kernels for heads of D elements and `rows` queries a kv head (k_attend_bf16.cu,
// k_attend_f32.cu).
AttendKernels attend_kernels_bf16(int D, int rows);
AttendKernels attend_kernels_f32(int D, int rows);

}  // namespace asymspec_impl
