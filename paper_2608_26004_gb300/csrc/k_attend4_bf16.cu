// Instantiations of the attention of bf16 queries over a paged cache in 4 bits (see
// kernel_attend4_tensor.cuh).
#include "k_attend.h"
#include "kernel_attend4_tensor.cuh"

namespace asymspec_impl {

template <int DP, int NR, int PER_SM>
AttendKernels tensor_pick() {
  constexpr int smem = static_cast<int>(tensor_smem_bytes(DP, NR));
  static_assert(smem <= kMaxSmem - 8192 && PER_SM * (smem + 2048) <= 228 * 1024, "the operands fit");
  static_assert(PER_SM * tensor_columns(DP, NR) <= 512, "and the tensor memory");
  static_assert(PER_SM * 152 <= kAMaxCtas, "the workspace has room");
  return {reinterpret_cast<const void*>(&attend4_tensor<DP, NR, PER_SM>),
          reinterpret_cast<const void*>(&attend_join<__nv_bfloat16, DP, NR>), DP, NR, kTThreads, smem, PER_SM};
}

AttendKernels attend4_kernels_bf16(int D, int rows) {
  if (D <= 64)
    return rows <= 16 ? tensor_pick<64, 16, 4>() : rows <= 32 ? tensor_pick<64, 32, 4>() : tensor_pick<64, 64, 2>();
  if (D <= 128)
    return rows <= 16 ? tensor_pick<128, 16, 4>() : rows <= 32 ? tensor_pick<128, 32, 3>() : tensor_pick<128, 64, 2>();
  return rows <= 16 ? tensor_pick<256, 16, 2>() : rows <= 32 ? tensor_pick<256, 32, 2>() : tensor_pick<256, 64, 1>();
}

}  // namespace asymspec_impl
