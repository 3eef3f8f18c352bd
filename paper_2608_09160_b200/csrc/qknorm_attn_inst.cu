// Instantiations of the general attention kernel, and the kernel that joins split results.
#include "qknorm_attn.cuh"

namespace qknorm {

__global__ void __launch_bounds__(kAttnJoinThreads) attn_join_kernel(const __grid_constant__ AttnParams P) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int* rec = P.starts + blockIdx.x * 8;
  const int parts = rec[3];
  if (parts == 0) return;  // the share starts with a unit, or the unit was cut before
  const int b = rec[0], qt = rec[1], kvh = rec[2];
  const AttnSeq s = attn_seq(P, b);
  const int tok0 = qt * P.tok_per_tile * P.tiles_per_item, lane = threadIdx.x & 31;
  // part p of row r lies with CTA blockIdx.x - 1 + p: in its slot 1 if it is the first, else in slot 0
  auto place = [&](int p, int r) { return ((long long)(blockIdx.x - 1 + p) * 2 + (p == 0 ? 1 : 0)) * P.part_rows + r; };
  for (int r = blockIdx.y * kAttnJoinRows + (threadIdx.x >> 5); r < (blockIdx.y + 1) * kAttnJoinRows; r += kAttnJoinThreads / 32) {
    const int in_tile = r % kAttnTile, i = tok0 + r / kAttnTile * P.tok_per_tile + in_tile / P.group;
    if (in_tile >= P.tok_per_tile * P.group || i >= s.n) continue;
    const long long row = s.row0 + (long long)i;
    const int head = kvh * P.group + in_tile % P.group;
    float z = kNegInf;
    for (int p = lane; p < parts; p += 32) z = fmaxf(z, P.part_z[place(p, r)]);  // NaN passes by; its weight below will be NaN
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) z = fmaxf(z, __shfl_xor_sync(0xffffffffu, z, o));
    float acc[4] = {0.f, 0.f, 0.f, 0.f}, sum = 0.f;
    const int d = lane * 4;
    for (int p0 = 0; p0 < parts; p0 += 32) {  // a lane each for the parts' weights, then four parts' rows at a time
      const float zp = p0 + lane < parts ? P.part_z[place(p0 + lane, r)] : kNegInf;
      const float wp = zp == kNegInf ? 0.f : z == kNegInf ? zp : exp2f(zp - z);
      const unsigned there = __ballot_sync(0xffffffffu, zp != kNegInf);  // a part that saw no key has written no row
      const int n = parts - p0 < 32 ? parts - p0 : 32;
      for (int p = 0; p < n; p += 4) {
        float4 x[4];
#pragma unroll
        for (int b = 0; b < 4; ++b)
          x[b] = (there >> (p + b)) & 1 && d < P.head_dim
                     ? *reinterpret_cast<const float4*>(P.part_o + place(p0 + p + b, r) * P.head_dim + d) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          const float w = __shfl_sync(0xffffffffu, wp, p + b);
          sum += w;
          acc[0] = fmaf(w, x[b].x, acc[0]);
          acc[1] = fmaf(w, x[b].y, acc[1]);
          acc[2] = fmaf(w, x[b].z, acc[2]);
          acc[3] = fmaf(w, x[b].w, acc[3]);
        }
      }
    }
    const float inv = sum == 0.f ? 0.f : P.v_scale / sum;
    if (d < P.head_dim) {
      const uint2 w = make_uint2(bf_pack(acc[0] * inv, acc[1] * inv), bf_pack(acc[2] * inv, acc[3] * inv));
      *reinterpret_cast<uint2*>(P.out + row * P.ld_out + (long long)head * P.head_dim + d) = w;
    }
    if (P.lse != nullptr && lane == 0) P.lse[row * P.heads_q + head] = sum == 0.f ? kNegInf : (z + log2f(sum)) * kLn2;
  }
}

AttnKernel attn_general_kernel_for(AttnFormat format) {
  return format == kAttnE4m3 ? attn_general_kernel<IoE4m3, IoE4m3>
                             : format == kAttnWidened ? attn_general_kernel<IoBf16, IoF16> : attn_general_kernel<IoBf16, IoBf16>;
}
AttnKernel attn_join_kernel_for() { return attn_join_kernel; }

}  // namespace qknorm
