// Instantiations of the attention of bf16 queries over a paged cache in 4 bits (see
// kernel_attend4_tensor.cuh).
#include "k_attend.h"
#include "kernel_attend4_tensor.cuh"

namespace asymspec_impl {

template <int DP, int RR, int PER_SM>
AttendKernels tensor_pick(bool fast) {
  constexpr int NR = tensor_rows(RR), smem = static_cast<int>(tensor_smem_bytes(DP, NR));
  static_assert(smem <= kMaxSmem - 8192 && PER_SM * (smem + 2048) <= 228 * 1024, "the operands fit");
  static_assert(PER_SM * tensor_columns(DP, NR) <= 512, "and the tensor memory");
  return {fast ? reinterpret_cast<const void*>(&attend4_tensor<DP, RR, PER_SM, true>)
               : reinterpret_cast<const void*>(&attend4_tensor<DP, RR, PER_SM, false>),
          reinterpret_cast<const void*>(&attend4_join<__nv_bfloat16, DP, RR, PER_SM * kASms>), DP, RR, kTThreads, smem, PER_SM,
          PER_SM * kASms, kTKeys};
}

// Rows of an item: the products' columns come in sixteens, but a thread's scores and sums are registers, so up to
// 8 rows have a kernel of their own.  CTAs an SM: as many as tensor memory and shared memory have room for (four
// of 128 columns), three where 32 rows need more registers.  us, and with one CTA less: 64 requests of 64 to 8192
// tokens, 4 rows 44.4 / 47.3, heads of 64 36.2 / 39.5; 8 of 4096 to 32768, 16 rows 52.6 / 53.5, 32 rows 73.9 / 76.6 (with
// four 94.7), 64 rows 124 / 160.
AttendKernels attend4_kernels_bf16(int D, int rows, bool fast) {
  if (D <= 64)
    return rows <= 8    ? tensor_pick<64, 8, 4>(fast)
           : rows <= 16 ? tensor_pick<64, 16, 4>(fast)
           : rows <= 32 ? tensor_pick<64, 32, 4>(fast)
                        : tensor_pick<64, 64, 2>(fast);
  if (D <= 128)
    return rows <= 8    ? tensor_pick<128, 8, 4>(fast)
           : rows <= 16 ? tensor_pick<128, 16, 4>(fast)
           : rows <= 32 ? tensor_pick<128, 32, 3>(fast)
                        : tensor_pick<128, 64, 2>(fast);
  return rows <= 8    ? tensor_pick<256, 8, 2>(fast)
         : rows <= 16 ? tensor_pick<256, 16, 2>(fast)
         : rows <= 32 ? tensor_pick<256, 32, 2>(fast)
                      : tensor_pick<256, 64, 1>(fast);
}

}  // namespace asymspec_impl
