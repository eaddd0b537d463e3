// The attention kernels of one head size and row tile, as the host launches them.
#pragma once

#include <cstddef>
#include <cstdint>

namespace asymspec_impl {

// The window that the kernels work with: 0 (none) where it spans whatever a table row can hold.  A
// window that is left is below that, 2^30 at most, so that the kernels' 32-bit length - Q - window + 1
// stays above -2^31 (Q * heads is 2^20 at most).
inline int attend_window(int window, int table_width, int block_size) {
  return window >= static_cast<int64_t>(table_width) * block_size ? 0 : window;
}

struct AttendKernels {
  const void *split, *join;
  int DP, rows, threads, smem, ctas_per_sm;
  int most_ctas;  // that the workspace has room for
  int tile;       // keys of a unit of work
};

// The kernels for heads of D elements and `rows` queries a kv head (k_attend_bf16.cu,
// k_attend_f32.cu).
AttendKernels attend_kernels_bf16(int D, int rows);
AttendKernels attend_kernels_f32(int D, int rows);
// The same over a cache in 4 bits (k_attend4_bf16.cu, k_attend4_f32.cu: one kernel for all boundaries); fast: a
// token's codes and scales of a head lie on boundaries of 32 and of DP / 16 bytes, and D is DP.
AttendKernels attend4_kernels_bf16(int D, int rows, bool fast);
AttendKernels attend4_kernels_f32(int D, int rows);

}  // namespace asymspec_impl
