// Instantiations of the tensor-core attention kernel, one padded head_dim and cache format per translation unit.
#include "qknorm_attn_tc.cuh"

namespace qknorm {

#define QKNORM_CAT_(a, b, c) a##b##c
#define QKNORM_CAT(a, b, c) QKNORM_CAT_(a, b, c)

AttnKernel QKNORM_CAT(attn_tc_kernel_, QKNORM_IO_TAG, QKNORM_DP)(bool one_tile, int* smem_bytes) {
  *smem_bytes = AttnSmem<QKNORM_DP, QKNORM_F8>::kBytes;
  return one_tile ? attn_tc_kernel<QKNORM_DP, QKNORM_F8, true> : attn_tc_kernel<QKNORM_DP, QKNORM_F8, false>;
}

}  // namespace qknorm
