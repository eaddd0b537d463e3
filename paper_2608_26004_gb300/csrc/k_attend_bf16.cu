// Instantiations of the attention over a paged cache (see kernel_attend.cuh).
#include "kernel_attend.cuh"
#include "k_attend.h"

namespace asymspec_impl {

template <int DP, int WR, int ST, int PER_SM, int kH = 2>
AttendKernels attend_pick() {
  constexpr int smem = static_cast<int>(attend_smem_bytes<__nv_bfloat16>(DP, WR, ST));
  static_assert(smem <= kMaxSmem - 8192 && PER_SM * (smem + 1024) <= 228 * 1024, "the rings fit");
  static_assert(PER_SM * 152 <= kAMaxCtas, "the workspace has room");
  return {reinterpret_cast<const void*>(&attend_split<__nv_bfloat16, DP, WR, ST, PER_SM, kH>),
          reinterpret_cast<const void*>(&attend_join<__nv_bfloat16, DP, 16 * WR>), DP, 16 * WR, 128 * WR, smem, PER_SM};
}

// One, two or four warps for the rows of a group: as many as the rows fill.  us, 8 requests of
// 4096 to 32768 tokens, 8 kv heads of 128 elements, with row tiles of 16 / 32 / 64:
//   24 rows 117 / 97 / 151     32 rows 119 / 99 / 152     48 rows 173 / 169 / 160     64 rows 181 / 174 / 167
// CTAs an SM: as many as the registers allow, with rings as deep as shared memory then does.  Three
// at 16 rows, where two with deeper rings are as fast for long contexts (64 requests of 64 to 8192
// tokens 74 both) and slower for short ones (256 of 16 to 300 tokens 39 to 34).
// Up to 8 rows (half of the matrix instructions' 16) the other half's softmax and pieces are left
// out: those 64 requests 74.3 to 73.7 us (heads of 64 45.0 to 43.9, of 256 163 to 157), those 256
// 33.6 to 31.3.
AttendKernels attend_kernels_bf16(int D, int rows) {
  if (rows <= 8)
    return D <= 64    ? attend_pick<64, 1, 3, 3, 1>()
           : D <= 128 ? attend_pick<128, 1, 2, 3, 1>()
                      : attend_pick<256, 1, 3, 1, 1>();
  if (D <= 64)
    return rows <= 16 ? attend_pick<64, 1, 3, 3>() : rows <= 32 ? attend_pick<64, 2, 5, 2>() : attend_pick<64, 4, 8, 1>();
  if (D <= 128)
    return rows <= 16 ? attend_pick<128, 1, 2, 3>() : rows <= 32 ? attend_pick<128, 2, 3, 2>() : attend_pick<128, 4, 5, 1>();
  return rows <= 16 ? attend_pick<256, 1, 3, 1>() : attend_pick<256, 2, 3, 1>();
}

}  // namespace asymspec_impl
