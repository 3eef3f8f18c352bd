// Instantiations of the 4-bit attention kernel, one padded head_dim per translation unit; the smallest one also has the kernels that
// join its parts and that widen a cache.
#include "qknorm_attn_e2m1.cuh"

namespace qknorm {

#define QKNORM_PASTE_(a, b) a##b
#define QKNORM_PASTE(a, b) QKNORM_PASTE_(a, b)

namespace {
template <int NT>
AttnE2m1Kernel pick(int copy, int* smem, int* per_sm) {
  *smem = E2m1Cta<QKNORM_DP, NT>::kSmem;
  *per_sm = E2m1Cta<QKNORM_DP, NT>::kPerSm;
  return copy == 16 ? attn_e2m1_kernel<QKNORM_DP, NT, 16> : attn_e2m1_kernel<QKNORM_DP, NT, 8>;
}
}  // namespace

AttnE2m1Kernel QKNORM_PASTE(attn_e2m1_kernel_, QKNORM_DP)(int nt, int copy, int* smem, int* per_sm) {
  switch (nt) {
    case 1: return pick<1>(copy, smem, per_sm);
    case 2: return pick<2>(copy, smem, per_sm);
#if QKNORM_DP < 256
    case 4: return pick<4>(copy, smem, per_sm);
#endif
    default: return nullptr;
  }
}

#if QKNORM_DP == 64
__global__ void __launch_bounds__(kE2m1JoinThreads) attn_e2m1_join_kernel(const __grid_constant__ AttnE2m1Params P) {
  const AttnParams& A = P.A;
  const int lane = threadIdx.x & 31;
  const long long warps = (long long)gridDim.x * (kE2m1JoinThreads / 32), items = (long long)A.seqs * A.max_q * A.heads_q;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  for (long long it = (long long)blockIdx.x * (kE2m1JoinThreads / 32) + (threadIdx.x >> 5); it < items; it += warps) {
    const int head = (int)(it % A.heads_q), i = (int)(it / A.heads_q % A.max_q), b = (int)(it / A.heads_q / A.max_q);
    const AttnSeq s = attn_seq(A, b);
    if (i >= s.n) continue;
    const long long r = (long long)i * A.group + head % A.group;
    const E2m1Span u = e2m1_span(P, s, r - r % P.tile_rows);
    if (u.c0 == u.c1) continue;
    const long long row = s.row0 + (long long)i;
    const long long at = (row * A.heads_q + head) * P.splits;
    float z = kNegInf;
    for (int c = u.c0 + lane; c <= u.c1; c += 32) z = fmaxf(z, P.part_z[at + c]);  // NaN passes by; its weight below will be NaN
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) z = fmaxf(z, __shfl_xor_sync(0xffffffffu, z, o));
    for (int d0 = 0; d0 < A.head_dim; d0 += 128) {
      const int d = d0 + 4 * lane;
      float acc[4] = {0.f, 0.f, 0.f, 0.f}, sum = 0.f;
      for (int c0 = u.c0; c0 <= u.c1; c0 += 32) {  // a lane each for the parts' weights, then four parts' rows at a time
        const float zp = c0 + lane <= u.c1 ? P.part_z[at + c0 + lane] : kNegInf;
        const float wp = zp == kNegInf ? 0.f : z == kNegInf ? zp : exp2f(zp - z);
        const int n = u.c1 - c0 + 1 < 32 ? u.c1 - c0 + 1 : 32;
        for (int p = 0; p < n; p += 4) {
          float4 x[4];
#pragma unroll
          for (int k = 0; k < 4; ++k)
            x[k] = p + k < n && d < A.head_dim ? *reinterpret_cast<const float4*>(P.part_o + (at + c0 + p + k) * A.head_dim + d)
                                               : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const float w = __shfl_sync(0xffffffffu, wp, (p + k) & 31);
            if (p + k >= n) continue;
            sum += w;
            acc[0] = fmaf(w, x[k].x, acc[0]);
            acc[1] = fmaf(w, x[k].y, acc[1]);
            acc[2] = fmaf(w, x[k].z, acc[2]);
            acc[3] = fmaf(w, x[k].w, acc[3]);
          }
        }
      }
      const float inv = sum == 0.f ? 0.f : A.v_scale / sum;
      if (d < A.head_dim) {
        uint16_t* out = A.out + row * A.ld_out + (long long)head * A.head_dim + d;
#pragma unroll
        for (int k = 0; k < 4; ++k) IoBf16::store(out, k, acc[k] * inv);
      }
      if (A.lse != nullptr && lane == 0 && d == 0) A.lse[row * A.heads_q + head] = sum == 0.f ? kNegInf : (z + log2f(sum)) * kLn2;
    }
  }
}
AttnE2m1Kernel attn_e2m1_join_kernel_for() { return attn_e2m1_join_kernel; }

// A CTA per (sequence, page, head, side).
__global__ void __launch_bounds__(kE2m1WidenThreads) e2m1_widen_kernel(const __grid_constant__ WidenParams W) {
  const AttnParams& A = W.P.A;
  const int blocks = A.head_dim >> 4;
  unsigned idx = blockIdx.x;
  const int side = idx & 1;
  idx >>= 1;
  const int h = idx % (unsigned)A.heads_kv;
  idx /= (unsigned)A.heads_kv;
  const int j = idx % (unsigned)W.cols, b = idx / (unsigned)W.cols;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  if (side == 0 && h == 0 && threadIdx.x == 0) W.table[(long long)b * W.cols + j] = b * W.cols + j;
  const AttnSeq s = attn_seq(A, b);
  if (s.n == 0) return;
  const int lo = attn_lo(A, s, 0), hi = attn_hi(A, s, s.n - 1);
  const long long first = (long long)j * kE2m1Page;
  if (hi <= lo || first >= hi || first + kE2m1Page <= lo) return;
  const AttnSide& C = side ? A.v : A.k;
  const AttnSide& S = side ? W.P.vs : W.P.ks;
  uint16_t* out = (side ? W.v : W.k) + (((long long)b * W.cols + j) * A.heads_kv + h) * kE2m1Page * A.head_dim;
  for (int i = threadIdx.x; i < kE2m1Page * blocks; i += kE2m1WidenThreads) {
    const int in = i / blocks, blk = i - in * blocks;
    const long long key = first + in;
    uint32_t y[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (key >= lo && key < hi) {
      int within;
      const long long page = attn_page(A, b, (int)key, within);
      if (page >= 0) {
        const uint2 w = __ldg(reinterpret_cast<const uint2*>(reinterpret_cast<const char*>(C.base) + page * C.page + within * C.token + h * C.head) + blk);
        const uint32_t byte = __ldg(reinterpret_cast<const unsigned char*>(S.base) + page * S.page + within * S.token + h * S.head + blk);
        uint32_t f[4], sc, none;
        e4m3x4_to_f16x2(byte, sc, none);
        const float scale = __half2float(__ushort_as_half((unsigned short)(sc & 0xffffu)));
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          e2m1x8_to_f16x2(half ? w.y : w.x, f);
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&f[k]));
            y[4 * half + k] = bf_pack(v.x * scale, v.y * scale);
          }
        }
      }
    }
    uint4* to = reinterpret_cast<uint4*>(out + (long long)in * A.head_dim + 16 * blk);
    to[0] = make_uint4(y[0], y[1], y[2], y[3]);
    to[1] = make_uint4(y[4], y[5], y[6], y[7]);
  }
}
WidenKernel e2m1_widen_kernel_for() { return e2m1_widen_kernel; }
#endif

}  // namespace qknorm
