// Instantiations of the rotary and cache-write kernels, in a translation unit of their own so that they
// compile in parallel with the others.
#include "qknorm_rope.cuh"

namespace qknorm {

namespace {
template <class IO, class CIO, int NORM, bool CACHE, bool INTER>
RopeKernel pick(int upt, int threads) {
  if (upt == 1) return rope_kernel<IO, CIO, NORM, CACHE, INTER, 1, 1024>;
  return threads <= 256 ? rope_kernel<IO, CIO, NORM, CACHE, INTER, 4, 256> : rope_kernel<IO, CIO, NORM, CACHE, INTER, 4, 1024>;
}
template <class IO, class CIO, int NORM, bool CACHE>
RopeKernel pick(bool interleaved, int upt, int threads) {
  return interleaved ? pick<IO, CIO, NORM, CACHE, true>(upt, threads) : pick<IO, CIO, NORM, CACHE, false>(upt, threads);
}
template <class CIO>
RopeKernel pick_cache(int norm, bool interleaved, int upt, int threads) {
  switch (norm) {
    case kNormNone: return pick<IoBf16, CIO, kNormNone, true>(interleaved, upt, threads);
    case kNormLayer: return pick<IoBf16, CIO, kNormLayer, true>(interleaved, upt, threads);
    default: return pick<IoBf16, CIO, kNormHead, true>(interleaved, upt, threads);
  }
}
}  // namespace

RopeKernel rope_kernel_for(int elem_bytes, int cache_bytes, int norm, bool interleaved, int upt, int threads) {
  if (cache_bytes == 0)
    return elem_bytes == 1 ? pick<IoE4m3, IoE4m3, kNormNone, false>(interleaved, upt, threads)
                           : pick<IoBf16, IoBf16, kNormNone, false>(interleaved, upt, threads);
  if (cache_bytes == kCacheE2m1) return pick_cache<IoE2m1>(norm, interleaved, upt, threads);
  return cache_bytes == 1 ? pick_cache<IoE4m3>(norm, interleaved, upt, threads) : pick_cache<IoBf16>(norm, interleaved, upt, threads);
}

RopeGeneralKernel rope_general_kernel_for(int elem_bytes, int cache_bytes) {
  if (cache_bytes == 0) return elem_bytes == 1 ? rope_general_kernel<IoE4m3, IoE4m3, false> : rope_general_kernel<IoBf16, IoBf16, false>;
  if (cache_bytes == kCacheE2m1) return rope_general_kernel<IoBf16, IoE2m1, true>;
  return cache_bytes == 1 ? rope_general_kernel<IoBf16, IoE4m3, true> : rope_general_kernel<IoBf16, IoBf16, true>;
}

}  // namespace qknorm
