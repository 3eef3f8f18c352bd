// Instantiations of the rotary and cache-write kernels, in a translation unit of their own so that they
// compile in parallel with the others.
#include "qknorm_rope.cuh"

namespace qknorm {

namespace {
template <class IO, class CIO, int NORM, bool CACHE>
RopeKernel pick(int upt, int threads) {
  if (upt == 1) return rope_kernel<IO, CIO, NORM, CACHE, 1, 1024>;
  return threads <= 256 ? rope_kernel<IO, CIO, NORM, CACHE, 4, 256> : rope_kernel<IO, CIO, NORM, CACHE, 4, 1024>;
}
template <class CIO>
RopeKernel pick_cache(int norm, int upt, int threads) {
  switch (norm) {
    case kNormNone: return pick<IoBf16, CIO, kNormNone, true>(upt, threads);
    case kNormLayer: return pick<IoBf16, CIO, kNormLayer, true>(upt, threads);
    default: return pick<IoBf16, CIO, kNormHead, true>(upt, threads);
  }
}
}  // namespace

RopeKernel rope_kernel_for(int elem_bytes, int cache_bytes, int norm, int upt, int threads) {
  if (cache_bytes == 0)
    return elem_bytes == 1 ? pick<IoE4m3, IoE4m3, kNormNone, false>(upt, threads) : pick<IoBf16, IoBf16, kNormNone, false>(upt, threads);
  return cache_bytes == 1 ? pick_cache<IoE4m3>(norm, upt, threads) : pick_cache<IoBf16>(norm, upt, threads);
}

RopeGeneralKernel rope_general_kernel_for(int elem_bytes, int cache_bytes) {
  if (cache_bytes == 0) return elem_bytes == 1 ? rope_general_kernel<IoE4m3, IoE4m3, false> : rope_general_kernel<IoBf16, IoBf16, false>;
  return cache_bytes == 1 ? rope_general_kernel<IoBf16, IoE4m3, true> : rope_general_kernel<IoBf16, IoBf16, true>;
}

}  // namespace qknorm
