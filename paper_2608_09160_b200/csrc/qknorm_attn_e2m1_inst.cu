// Instantiations of the 4-bit attention kernel, one padded head_dim per translation unit; the smallest one also has the kernels that
// join its parts and that widen a cache.
#include "qknorm_attn_e2m1.cuh"

namespace qknorm {

#define QKNORM_PASTE_(a, b) a##b
#define QKNORM_PASTE(a, b) QKNORM_PASTE_(a, b)

namespace {
template <int NT, int COPY, int WARPS = e2m1_warps(NT, COPY)>
E2m1Launch one() {
  using C = E2m1Cta<QKNORM_DP, NT, COPY, WARPS>;
  return E2m1Launch{attn_e2m1_kernel<QKNORM_DP, NT, COPY, WARPS>, C::kSmem, C::kWarps, C::kPerSm};
}
template <int NT>
E2m1Launch pick(int copy) {
#if QKNORM_DP < 256
  if (copy == 0) return one<NT, 0>();
#endif
  return copy == 16 ? one<NT, 16>() : one<NT, 8>();
}
}  // namespace

E2m1Launch QKNORM_PASTE(attn_e2m1_kernel_, QKNORM_DP)(int nt, int copy, bool wide) {
  if (wide) return copy == 16 ? one<1, 16, 8>() : one<1, 8, 8>();
  return nt == 1 ? pick<1>(copy) : pick<2>(copy);
}

#if QKNORM_DP == 64
__global__ void __launch_bounds__(kE2m1JoinThreads) attn_e2m1_join_kernel(const __grid_constant__ AttnE2m1Params P) {
  const AttnParams& A = P.A;
  const int lane = threadIdx.x & 31, rows = P.heads_cta * P.tile_rows;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int* cut = P.cuts + blockIdx.x * 8;
  const int b = cut[0];
  if (b < 0) return;
  const int rt = cut[1], hg = cut[2], c0 = cut[3], slot0 = cut[4], parts = blockIdx.x - c0 + 1;
  const AttnSeq s = attn_seq(A, b);
  // part p of row k lies with CTA c0 + p, in slot 0 but for the first
  auto place = [&](int p, int k) { return ((long long)(c0 + p) * 2 + (p == 0 ? slot0 : 0)) * rows + k; };
  for (int k = blockIdx.y * (kE2m1JoinThreads / 32) + (threadIdx.x >> 5); k < rows; k += gridDim.y * (kE2m1JoinThreads / 32)) {
    const unsigned rr = (unsigned)rt * (unsigned)P.tile_rows + (unsigned)(k % P.tile_rows);
    if (rr >= (unsigned)s.n * (unsigned)A.group) continue;
    const int i = (int)(rr / (unsigned)A.group), head = (hg * P.heads_cta + k / P.tile_rows) * A.group + (int)(rr - (unsigned)i * (unsigned)A.group);
    const long long row = s.row0 + (long long)i;
    float z = kNegInf;
    for (int p = lane; p < parts; p += 32) z = fmaxf(z, P.part_z[place(p, k)]);  // NaN passes by; its weight below will be NaN
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) z = fmaxf(z, __shfl_xor_sync(0xffffffffu, z, o));
    for (int d0 = 0; d0 < A.head_dim; d0 += 128) {
      const int d = d0 + 4 * lane;
      float acc[4] = {0.f, 0.f, 0.f, 0.f}, sum = 0.f;
      for (int p0 = 0; p0 < parts; p0 += 32) {  // a lane each for the parts' weights, then eight parts' rows at a time
        const float zp = p0 + lane < parts ? P.part_z[place(p0 + lane, k)] : kNegInf;
        const float wp = zp == kNegInf ? 0.f : z == kNegInf ? zp : exp2f(zp - z);
        const int n = parts - p0 < 32 ? parts - p0 : 32;
        constexpr int kAhead = 8;
        for (int p = 0; p < n; p += kAhead) {
          float4 x[kAhead];
#pragma unroll
          for (int e = 0; e < kAhead; ++e)
            x[e] = p + e < n && d < A.head_dim ? *reinterpret_cast<const float4*>(P.part_o + place(p0 + p + e, k) * A.head_dim + d)
                                               : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
          for (int e = 0; e < kAhead; ++e) {
            const float w = __shfl_sync(0xffffffffu, wp, p + e);  // 0 behind the last part
            sum += w;
            acc[0] = fmaf(w, x[e].x, acc[0]);
            acc[1] = fmaf(w, x[e].y, acc[1]);
            acc[2] = fmaf(w, x[e].z, acc[2]);
            acc[3] = fmaf(w, x[e].w, acc[3]);
          }
        }
      }
      const float inv = sum == 0.f ? 0.f : A.v_scale / sum;
      if (d < A.head_dim) {
        uint16_t* out = A.out + row * A.ld_out + (long long)head * A.head_dim + d;
#pragma unroll
        for (int e = 0; e < 4; ++e) IoBf16::store(out, e, acc[e] * inv);
      }
      if (A.lse != nullptr && lane == 0 && d == 0) A.lse[row * A.heads_q + head] = sum == 0.f ? kNegInf : (z + log2f(sum)) * kLn2;
    }
  }
}
AttnE2m1JoinKernel attn_e2m1_join_kernel_for() { return attn_e2m1_join_kernel; }

// A CTA per (sequence, page, head): blocks of K and of V together, so that a page is looked up once for both.
__global__ void __launch_bounds__(kE2m1WidenThreads) e2m1_widen_kernel(const __grid_constant__ WidenParams W) {
  const AttnParams& A = W.P.A;
  const int blocks = A.head_dim >> 4;
  unsigned idx = blockIdx.x;
  const int h = idx % (unsigned)A.heads_kv;
  idx /= (unsigned)A.heads_kv;
  const int j = idx % (unsigned)W.cols, b = idx / (unsigned)W.cols;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  if (h == 0 && threadIdx.x == 0) W.table[(long long)b * W.cols + j] = b * W.cols + j;
  const AttnSeq s = attn_seq(A, b);
  if (s.n == 0) return;
  const int lo = attn_lo(A, s, 0), hi = attn_hi(A, s, s.n - 1);
  const long long first = (long long)j * kE2m1Page;
  if (hi <= lo || first >= hi || first + kE2m1Page <= lo) return;
  const long long to = (((long long)b * W.cols + j) * A.heads_kv + h) * kE2m1Page * A.head_dim;
  const char* const codes[2] = {reinterpret_cast<const char*>(A.k.base) + h * A.k.head, reinterpret_cast<const char*>(A.v.base) + h * A.v.head};
  const unsigned char* const scales[2] = {reinterpret_cast<const unsigned char*>(W.P.ks.base) + h * W.P.ks.head,
                                          reinterpret_cast<const unsigned char*>(W.P.vs.base) + h * W.P.vs.head};
  constexpr int kAhead = 4;  // blocks of a thread, of K and of V, whose loads are under way together
  const bool even = kE2m1WidenThreads % blocks == 0;  // a thread stays at its block of a token
  const int in0 = (int)threadIdx.x / blocks, blk0 = (int)threadIdx.x - in0 * blocks, step = kE2m1WidenThreads / blocks;
  for (int i0 = threadIdx.x, turn = 0; i0 < kE2m1Page * blocks; i0 += kAhead * kE2m1WidenThreads, ++turn) {
    uint2 w[kAhead][2];
    uint32_t byte[kAhead][2];
#pragma unroll
    for (int a = 0; a < kAhead; ++a) {
      const int i = i0 + a * kE2m1WidenThreads;
      int in = in0 + (turn * kAhead + a) * step, blk = blk0;
      if (!even) {
        in = i / blocks;
        blk = i - in * blocks;
      }
      const long long key = first + in;
      w[a][0] = w[a][1] = make_uint2(0, 0);
      byte[a][0] = byte[a][1] = 0;
      if (i < kE2m1Page * blocks && key >= lo && key < hi) {
        int within;
        const int page = (int)attn_page(A, b, (int)key, within);
        if (page >= 0) {
          const unsigned long long p = (unsigned)page, n = (unsigned)within;
          w[a][0] = __ldg(reinterpret_cast<const uint2*>(codes[0] + p * A.k.page + n * A.k.token) + blk);
          w[a][1] = __ldg(reinterpret_cast<const uint2*>(codes[1] + p * A.v.page + n * A.v.token) + blk);
          byte[a][0] = __ldg(scales[0] + p * W.P.ks.page + n * W.P.ks.token + blk);
          byte[a][1] = __ldg(scales[1] + p * W.P.vs.page + n * W.P.vs.token + blk);
        }
      }
    }
#pragma unroll
    for (int a = 0; a < kAhead; ++a) {
      const int i = i0 + a * kE2m1WidenThreads;
      if (i >= kE2m1Page * blocks) break;
#pragma unroll
      for (int side = 0; side < 2; ++side) {
        uint32_t y[8], twice, none;  // the block's scale in both halves
        e4m3x4_to_f16x2(byte[a][side] * 0x101u, twice, none);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          uint32_t f[4];
          e2m1x8_to_f16x2(half ? w[a][side].y : w[a][side].x, f);
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            y[4 * half + k] = hmul2(f[k], twice);
            if (side == 0) {
              const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&y[4 * half + k]));
              y[4 * half + k] = bf_pack(v.x, v.y);
            }
          }
        }
        // rows lie one after the other; 32 bytes at a time, a whole sector
        asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"((side ? W.v : W.k) + to + 16ll * i), "r"(y[0]), "r"(y[1]), "r"(y[2]),
                     "r"(y[3]), "r"(y[4]), "r"(y[5]), "r"(y[6]), "r"(y[7])
                     : "memory");
      }
    }
  }
}
WidenKernel e2m1_widen_kernel_for() { return e2m1_widen_kernel; }
#endif

}  // namespace qknorm
