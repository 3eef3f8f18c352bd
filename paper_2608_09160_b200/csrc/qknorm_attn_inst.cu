// Instantiations of the general attention kernel, and the kernel that joins split results.
#include "qknorm_attn.cuh"

namespace qknorm {

__global__ void __launch_bounds__(kAttnJoinThreads) attn_join_kernel(const __grid_constant__ AttnParams P) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int lane = threadIdx.x & 31;
  const long long items = (long long)P.seqs * P.max_q * P.heads_q;
  const long long it = (long long)blockIdx.x * (kAttnJoinThreads / 32) + (threadIdx.x >> 5);
  if (it >= items) return;
  const int head = (int)(it % P.heads_q);
  const long long r = it / P.heads_q;
  const int i = (int)(r % P.max_q), b = (int)(r / P.max_q);
  const AttnSeq s = attn_seq(P, b);
  if (i >= s.n) return;
  const long long row = s.row0 + (long long)i;
  const int per_item = P.tok_per_tile * P.tiles_per_item;
  int J0, J1, ulo, uhi;
  attn_span(P, s, i / per_item * per_item, J0, J1, ulo, uhi);
  const int parts = (J1 - J0 + P.chunk_tiles - 1) / P.chunk_tiles;
  const long long step = P.T * P.heads_q, at = row * P.heads_q + head;
  float z = kNegInf;
  for (int p = lane; p < parts; p += 32) {
    const float zp = P.part_z[p * step + at];
    z = zp != zp ? zp : fmaxf(z, zp);  // a part that is NaN makes the row NaN below, through its weight
  }
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) z = fmaxf(z, __shfl_xor_sync(0xffffffffu, z, off));
  float acc[4] = {0.f, 0.f, 0.f, 0.f}, sum = 0.f;
  const int d = lane * 4;
  for (int p = 0; p < parts; ++p) {
    const float zp = P.part_z[p * step + at];
    if (zp == kNegInf) continue;  // this part saw no key: its o was not written
    const float w = exp2f(zp - z);
    sum += w;
    const float* o = P.part_o + (p * step + at) * P.head_dim;
    if (d < P.head_dim) {
      const float4 x = *reinterpret_cast<const float4*>(o + d);
      acc[0] = fmaf(w, x.x, acc[0]);
      acc[1] = fmaf(w, x.y, acc[1]);
      acc[2] = fmaf(w, x.z, acc[2]);
      acc[3] = fmaf(w, x.w, acc[3]);
    }
  }
  const float inv = sum == 0.f ? 0.f : P.v_scale / sum;
  if (d < P.head_dim) {
    const uint2 w = make_uint2(bf_pack(acc[0] * inv, acc[1] * inv), bf_pack(acc[2] * inv, acc[3] * inv));
    *reinterpret_cast<uint2*>(P.out + row * P.ld_out + (long long)head * P.head_dim + d) = w;
  }
  if (P.lse != nullptr && lane == 0) P.lse[at] = sum == 0.f ? kNegInf : (z + log2f(sum)) * kLn2;
}

AttnKernel attn_general_kernel_for(bool e4m3) { return e4m3 ? attn_general_kernel<IoE4m3> : attn_general_kernel<IoBf16>; }
AttnKernel attn_join_kernel_for() { return attn_join_kernel; }

}  // namespace qknorm
