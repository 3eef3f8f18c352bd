// Instantiations of the tensor-core attention kernel, one padded head_dim and cache format per translation unit.
#include "qknorm_attn_tc.cuh"

namespace qknorm {

#define QKNORM_CAT_(a, b, c) a##b##c
#define QKNORM_CAT(a, b, c) QKNORM_CAT_(a, b, c)

namespace {
template <bool TMA>
AttnTcKernel pick(int form) {
  switch (form) {
    case kAttnTwo: return attn_tc_kernel<QKNORM_DP, QKNORM_KIO, QKNORM_VIO, kAttnTwo, TMA>;
    case kAttnOne: return attn_tc_kernel<QKNORM_DP, QKNORM_KIO, QKNORM_VIO, kAttnOne, TMA>;
    default:  // 32 rows or fewer, which a widened 4-bit cache is never attended to by
      if constexpr (std::is_same<QKNORM_VIO, IoF16>::value) return nullptr;
      else return attn_tc_kernel<QKNORM_DP, QKNORM_KIO, QKNORM_VIO, kAttnQuad, TMA>;
  }
}
}  // namespace

AttnTcKernel QKNORM_CAT(attn_tc_kernel_, QKNORM_IO_TAG, QKNORM_DP)(int form, bool tma, int* smem_bytes) {
  *smem_bytes = AttnSmem<QKNORM_DP, QKNORM_KIO::kBytes == 1>::kBytes;
  return tma ? pick<true>(form) : pick<false>(form);
}

}  // namespace qknorm
