// Instantiations of the tensor-core attention kernel, one padded head_dim and cache format per translation unit.
#include "qknorm_attn_tc.cuh"

namespace qknorm {

#define QKNORM_CAT_(a, b, c) a##b##c
#define QKNORM_CAT(a, b, c) QKNORM_CAT_(a, b, c)

AttnTcKernel QKNORM_CAT(attn_tc_kernel_, QKNORM_IO_TAG, QKNORM_DP)(bool one_tile, bool tma, int* smem_bytes) {
  *smem_bytes = AttnSmem<QKNORM_DP, QKNORM_F8>::kBytes;
  if (tma) return one_tile ? attn_tc_kernel<QKNORM_DP, QKNORM_F8, true, true> : attn_tc_kernel<QKNORM_DP, QKNORM_F8, false, true>;
  return one_tile ? attn_tc_kernel<QKNORM_DP, QKNORM_F8, true, false> : attn_tc_kernel<QKNORM_DP, QKNORM_F8, false, false>;
}

}  // namespace qknorm
