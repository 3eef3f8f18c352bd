// Instantiations of the tensor-core attention kernel, one padded head_dim and cache format per translation unit.
#include "qknorm_attn_tc.cuh"

namespace qknorm {

#define QKNORM_CAT_(a, b, c) a##b##c
#define QKNORM_CAT(a, b, c) QKNORM_CAT_(a, b, c)

namespace {
template <bool TMA>
AttnTcKernel pick(int form) {
  switch (form) {
    case kAttnTwo: return attn_tc_kernel<QKNORM_DP, QKNORM_F8, kAttnTwo, TMA>;
    case kAttnOne: return attn_tc_kernel<QKNORM_DP, QKNORM_F8, kAttnOne, TMA>;
    default: return attn_tc_kernel<QKNORM_DP, QKNORM_F8, kAttnQuad, TMA>;
  }
}
}  // namespace

AttnTcKernel QKNORM_CAT(attn_tc_kernel_, QKNORM_IO_TAG, QKNORM_DP)(int form, bool tma, int* smem_bytes) {
  *smem_bytes = AttnSmem<QKNORM_DP, QKNORM_F8>::kBytes;
  return tma ? pick<true>(form) : pick<false>(form);
}

}  // namespace qknorm
