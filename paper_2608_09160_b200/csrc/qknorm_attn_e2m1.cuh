// Attention of new tokens over a 4-bit paged cache (include/qknorm_attn.h: qknorm_attn_paged_e2m1).
//
// Mathematics: as in qknorm_attn.cuh, with k = code * scale * k_scale.  A code has two significant bits and a scale four, so code * scale
// has six and is exact in fp16; the products are fp16 in, fp32 out.
//
// What bounds it: single tokens read 9/16 byte per element of K and V, a quarter of a bf16 cache, and have to widen every one of
// them.  So nothing is staged for the matrix unit: a warp brings 32 keys at a time into shared memory by cp.async, widens them out of
// registers straight into the operands of mma.sync, and no widened element touches memory.  K and V are the 16-row operand and the query
// rows the 8-column one, S^T = K Q^T and O^T = V^T P^T: eight query heads of a key head fill a matrix instruction, where they would
// leave half (mma.sync) or fifteen sixteenths (tcgen05) of it empty as its rows.
//
// Which element stands where in an operand is free as long as both operands agree, and is chosen so that a thread's share is
// contiguous in the cache (g = lane / 4, t = lane % 4, DP = head_dim padded to 64, 128 or 256):
//   S^T: thread t holds dims [t DP/4, (t+1) DP/4) of keys g and g + 8 -- whole blocks, one scale per block;
//   O^T: thread g holds dims [g DP/8, (g+1) DP/8) of keys 2t, 2t+1, 2t+8, 2t+9 -- within blocks, one scale per key and block;
//        pairs of keys share a register, so the codes of two keys are interleaved by four bits before they are widened.
// Scores come out with keys along g and rows along t, and go back in transposed by movmatrix; a thread's output columns are the
// rows of its scores, so that maxima and rescaling need no exchange beyond the maximum itself.
//
// Work: (sequence, key head, up to 8 NT query rows) x chunks of keys, a CTA of four warps each, tiles of 32 keys dealt to the warps in
// turn.  Rows with more than one chunk leave parts in the workspace for attn_e2m1_join_kernel.
#pragma once
#include "qknorm_attn.cuh"

namespace qknorm {

constexpr int kE2m1Warps = 4, kE2m1Threads = 32 * kE2m1Warps, kE2m1Tile = 32;
constexpr float kE2m1Lift = 14.f;  // weights are 2^14 times themselves, so that the smallest are not lost in fp16

struct AttnE2m1Params {
  AttnParams A;     // k, v: the codes, strides in bytes
  AttnSide ks, vs;  // the scales, strides in bytes
  int chunk;        // keys of a CTA
  int splits;       // chunks that a row has at most
  int row_tiles;    // per sequence and key head, at most
  int tile_rows;    // 8 NT
  int scale_unit;   // bytes that scales are copied by: 8 or 4 with cp.async, 2 or 1 without
  int q_vec;        // rows of q are 16-byte aligned
  float* part_o;    // [tokens][heads_q][splits][head_dim], normalised
  float* part_z;    // [tokens][heads_q][splits], log2
};

template <int DP>
struct E2m1Stage {  // one tile of one warp; pitches that keep the reads below free of bank conflicts
  static constexpr int kKPitch = DP == 256 ? 144 : DP / 2;
  static constexpr int kVPitch = DP == 64 ? 48 : DP == 128 ? 80 : 144;
  static constexpr int kSPitch = DP / 16;
  static constexpr int kV = kE2m1Tile * kKPitch;
  static constexpr int kKs = kV + kE2m1Tile * kVPitch;
  static constexpr int kVs = kKs + kE2m1Tile * kSPitch;
  static constexpr int kBytes = kVs + kE2m1Tile * kSPitch;
};
template <int DP, int NT>
struct E2m1Cta {
  static constexpr int kStages = DP == 256 ? 2 : DP == 128 ? (NT == 4 ? 4 : 3) : 4;
  static constexpr bool kQShared = DP * NT > 256;  // the query operand does not fit the registers beside the output
  static constexpr int kQBytes = kQShared ? NT * (DP / 16) * 32 * 8 : 0;
  static constexpr int kRing = kStages * E2m1Stage<DP>::kBytes;  // of a warp
  static constexpr int kOPitch = DP + 8;                         // floats
  static constexpr int kJoin = kE2m1Warps * 8 * NT * kOPitch * 4;
  static constexpr int kSmem = kQBytes + (kJoin > kE2m1Warps * kRing ? kJoin : kE2m1Warps * kRing);
  static constexpr int kPerSm = DP == 256 ? 2 : NT == 4 ? 2 : 3;
};

// Which chunks the rows [first, first + tile_rows) of a sequence and key head need; keys: some row sees any.
struct E2m1Span {
  long long rows;
  int tok0, tok1, base, ulo, uhi, c0, c1;
};
__device__ __forceinline__ E2m1Span e2m1_span(const AttnE2m1Params& P, const AttnSeq& s, long long first) {
  E2m1Span u;
  u.rows = (long long)s.n * P.A.group;
  const long long end = first + P.tile_rows < u.rows ? first + P.tile_rows : u.rows;
  u.tok0 = (int)(first / P.A.group);
  u.tok1 = (int)((end - 1) / P.A.group);
  u.base = attn_lo(P.A, s, 0);
  u.ulo = attn_lo(P.A, s, u.tok0);
  u.uhi = attn_hi(P.A, s, u.tok1);
  if (u.uhi <= u.ulo) {
    u.ulo = u.uhi = u.base;
    u.c0 = u.c1 = 0;
  } else {
    u.c0 = (u.ulo - u.base) / P.chunk;
    u.c1 = (u.uhi - 1 - u.base) / P.chunk;
  }
  return u;
}

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t hmul2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ uint32_t f16_pack(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ uint32_t transpose8(uint32_t a) {
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(a));
  return r;
}
__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// Copies N bytes, or writes N zeros.
template <int N>
__device__ __forceinline__ void copy_or_zero(uint32_t dst, const void* src, bool there) {
  const int n = there ? N : 0;
  if constexpr (N == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(dst), "l"(src), "n"(N), "r"(n) : "memory");
}
template <int N>
__device__ __forceinline__ void load_words(const char* p, uint32_t (&w)[N]) {
  if constexpr (N == 1) {
    w[0] = *reinterpret_cast<const uint32_t*>(p);
  } else if constexpr (N == 2) {
    const uint2 v = *reinterpret_cast<const uint2*>(p);
    w[0] = v.x, w[1] = v.y;
  } else {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      const uint4 v = *reinterpret_cast<const uint4*>(p + 4 * i);
      w[i] = v.x, w[i + 1] = v.y, w[i + 2] = v.z, w[i + 3] = v.w;
    }
  }
}

// DP: head_dim padded; NT: tiles of 8 query rows; COPY: bytes of a copy.
template <int DP, int NT, int COPY>
__global__ void __launch_bounds__(kE2m1Threads, E2m1Cta<DP, NT>::kPerSm) attn_e2m1_kernel(const __grid_constant__ AttnE2m1Params P) {
  using L = E2m1Stage<DP>;
  using C = E2m1Cta<DP, NT>;
  constexpr int KS = DP / 16;   // steps of 16 dims
  constexpr int PT = DP / 4;    // dims of a thread in S^T
  constexpr int PG = DP / 8;    // dims of a thread in O^T
  extern __shared__ uint4 smem_e2m1[];
  __shared__ float row_m[kE2m1Warps][8 * NT], row_l[kE2m1Warps][8 * NT];
  const AttnParams& A = P.A;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  char* const smem = reinterpret_cast<char*>(smem_e2m1);
  char* const ring = smem + C::kQBytes + warp * C::kRing;
  const uint32_t ring32 = (uint32_t)__cvta_generic_to_shared(ring);

  unsigned idx = blockIdx.x;
  const int rt = idx % (unsigned)P.row_tiles;
  idx /= (unsigned)P.row_tiles;
  const int kvh = idx % (unsigned)A.heads_kv;
  idx /= (unsigned)A.heads_kv;
  const int chunk = idx % (unsigned)P.splits, b = idx / (unsigned)P.splits;
  if (A.head_dim < DP)  // what no copy writes has to be zero
    for (int i = lane; i < C::kRing / 16; i += 32) reinterpret_cast<uint4*>(ring)[i] = make_uint4(0, 0, 0, 0);
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const AttnSeq s = attn_seq(A, b);
  const long long first = (long long)rt * (8 * NT);
  if (first >= (long long)s.n * A.group) return;
  const E2m1Span u = e2m1_span(P, s, first);
  if (chunk < u.c0 || chunk > u.c1) return;
  const long long c_lo = u.base + (long long)chunk * P.chunk, c_hi = c_lo + P.chunk;
  const int k0 = c_lo > u.ulo ? (int)c_lo : u.ulo, k1 = c_hi < u.uhi ? (int)c_hi : u.uhi;
  const int tiles = (k1 - k0 + kE2m1Tile - 1) / kE2m1Tile;

  // ---- copies: a lane looks up the page of one key of the tile
  const char* const kb = reinterpret_cast<const char*>(A.k.base) + kvh * A.k.head;
  const char* const vb = reinterpret_cast<const char*>(A.v.base) + kvh * A.v.head;
  const char* const ksb = reinterpret_cast<const char*>(P.ks.base) + kvh * P.ks.head;
  const char* const vsb = reinterpret_cast<const char*>(P.vs.base) + kvh * P.vs.head;
  const int row_bytes = A.head_dim >> 1, scale_bytes = A.head_dim >> 4;
  long long page = -1;  // of this lane's key in the tile that is issued next
  int within = 0;
  auto look = [&](int tile) {
    const int key = k0 + tile * kE2m1Tile + lane;
    page = -1;
    if (tile < tiles && key < k1) page = attn_page(A, b, key, within);
  };
  auto issue = [&](int tile, int stage) {
    if (tile < tiles) {
      const uint32_t at = ring32 + stage * L::kBytes;
      const bool there = page >= 0;
      const unsigned long long ka = there ? (unsigned long long)(page * A.k.page + within * A.k.token) : ~0ull;
      const unsigned long long va = there ? (unsigned long long)(page * A.v.page + within * A.v.token) : 0ull;
      constexpr int kPer = DP / 2 / COPY;  // copies of a row
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const int key = (lane + 32 * i) / kPer, part = (lane + 32 * i) % kPer;
        const unsigned long long kk = __shfl_sync(0xffffffffu, ka, key), vv = __shfl_sync(0xffffffffu, va, key);
        const bool ok = kk != ~0ull;
        if (part * COPY < row_bytes) {
          copy_or_zero<COPY>(at + key * L::kKPitch + part * COPY, kb + (ok ? kk + part * COPY : 0), ok);
          copy_or_zero<COPY>(at + L::kV + key * L::kVPitch + part * COPY, vb + (ok ? vv + part * COPY : 0), ok);
        }
      }
      const char* ks = ksb + (there ? page * P.ks.page + within * P.ks.token : 0);
      const char* vs = vsb + (there ? page * P.vs.page + within * P.vs.token : 0);
      const uint32_t ksm = at + L::kKs + lane * L::kSPitch, vsm = at + L::kVs + lane * L::kSPitch;
      if (P.scale_unit == 8) {
        if constexpr (DP >= 128) {
#pragma unroll
          for (int i = 0; i < L::kSPitch; i += 8)
            if (i < scale_bytes) {
              copy_or_zero<8>(ksm + i, ks + i, there);
              copy_or_zero<8>(vsm + i, vs + i, there);
            }
        }
      } else if (P.scale_unit == 4) {
#pragma unroll
        for (int i = 0; i < L::kSPitch; i += 4)
          if (i < scale_bytes) {
            copy_or_zero<4>(ksm + i, ks + i, there);
            copy_or_zero<4>(vsm + i, vs + i, there);
          }
      } else {
        unsigned char* kd = reinterpret_cast<unsigned char*>(ring + stage * L::kBytes + L::kKs + lane * L::kSPitch);
        unsigned char* vd = reinterpret_cast<unsigned char*>(ring + stage * L::kBytes + L::kVs + lane * L::kSPitch);
        for (int i = 0; i < scale_bytes; ++i) {
          kd[i] = there ? (unsigned char)ks[i] : 0;
          vd[i] = there ? (unsigned char)vs[i] : 0;
        }
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  __syncwarp();
#pragma unroll
  for (int i = 0; i < C::kStages - 1; ++i) {
    look(warp + i * kE2m1Warps);
    issue(warp + i * kE2m1Warps, i);
  }
  look(warp + (C::kStages - 1) * kE2m1Warps);

  // ---- queries: row g of every tile of 8, dims [t PT, (t + 1) PT), as fp16 times 2^-e
  uint32_t qr[C::kQShared ? 1 : NT][C::kQShared ? 1 : KS][2];
  uint2* const qs = reinterpret_cast<uint2*>(smem);
  float lift[NT][2];  // 2^e of this thread's score rows 2t, 2t + 1
  int lo[NT][2], hi[NT][2];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const long long r = first + nt * 8 + g;
    const bool there = r < u.rows;
    const int i = there ? (int)(r / A.group) : 0, head = kvh * A.group + (there ? (int)(r % A.group) : 0);
    const uint16_t* row = A.q + (s.row0 + (long long)i) * A.ld_q + (long long)head * A.head_dim + t * PT;
    uint32_t w[PT / 2];
#pragma unroll
    for (int j = 0; j < PT / 2; j += 4) {
      uint4 v = make_uint4(0, 0, 0, 0);
      if (there && t * PT + 2 * j < A.head_dim) {
        if (P.q_vec) {
          v = __ldg(reinterpret_cast<const uint4*>(row + 2 * j));
        } else {
          v.x = __ldg(row + 2 * j) | (uint32_t)__ldg(row + 2 * j + 1) << 16;
          v.y = __ldg(row + 2 * j + 2) | (uint32_t)__ldg(row + 2 * j + 3) << 16;
          v.z = __ldg(row + 2 * j + 4) | (uint32_t)__ldg(row + 2 * j + 5) << 16;
          v.w = __ldg(row + 2 * j + 6) | (uint32_t)__ldg(row + 2 * j + 7) << 16;
        }
      }
      w[j] = v.x, w[j + 1] = v.y, w[j + 2] = v.z, w[j + 3] = v.w;
    }
    float top = 0.f;  // of the finite elements
#pragma unroll
    for (int j = 0; j < PT / 2; ++j) {
      const float x = fabsf(bf_lo(w[j])), y = fabsf(bf_hi(w[j]));
      top = fmaxf(top, x < __builtin_huge_valf() ? x : 0.f);
      top = fmaxf(top, y < __builtin_huge_valf() ? y : 0.f);
    }
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
    const int e = top > 0.f ? ilogbf(top) - 14 : 0;  // the row's largest element comes to [2^14, 2^15)
    const float f_a = ldexpf(1.f, -e / 2), f_b = ldexpf(1.f, -e + e / 2);  // 2^-e itself may not be an fp32 value
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      uint32_t f[2];
#pragma unroll
      for (int k = 0; k < 2; ++k) f[k] = f16_pack(bf_lo(w[2 * ks + k]) * f_a * f_b, bf_hi(w[2 * ks + k]) * f_a * f_b);
      if constexpr (C::kQShared) {
        if (warp == nt % kE2m1Warps) qs[(nt * KS + ks) * 32 + lane] = make_uint2(f[0], f[1]);
      } else {
        qr[nt][ks][0] = f[0];
        qr[nt][ks][1] = f[1];
      }
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      lift[nt][k] = ldexpf(1.f, __shfl_sync(0xffffffffu, e, 4 * (2 * t + k)));
      const long long rr = first + nt * 8 + 2 * t + k;
      lo[nt][k] = hi[nt][k] = 0;
      if (rr < u.rows) {
        const int ii = (int)(rr / A.group);
        lo[nt][k] = attn_lo(A, s, ii);
        hi[nt][k] = attn_hi(A, s, ii);
        if (hi[nt][k] > k1) hi[nt][k] = k1;
      }
    }
  }
  if constexpr (C::kQShared) __syncthreads();
  // keys that every row sees
  const int all_lo = attn_lo(A, s, u.tok1), all_hi0 = attn_hi(A, s, u.tok0), all_hi = all_hi0 < k1 ? all_hi0 : k1;

  float o[KS][NT][4];  // [DP / 16 pairs of dims][..][dim 2j: rows 2t, 2t + 1; dim 2j + 1: the same]
  float m[NT][2], l[NT][2];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    m[nt][0] = m[nt][1] = kNegInf;
    l[nt][0] = l[nt][1] = 0.f;
#pragma unroll
    for (int j = 0; j < KS; ++j) o[j][nt][0] = o[j][nt][1] = o[j][nt][2] = o[j][nt][3] = 0.f;
  }

  int stage = 0;
  for (int tile = warp; tile < tiles; tile += kE2m1Warps) {
    asm volatile("cp.async.wait_group %0;" ::"n"(C::kStages - 2) : "memory");
    __syncwarp();  // every lane's copies have landed, and nobody reads the stage that is filled next
    {
      int next = stage + C::kStages - 1;
      if (next >= C::kStages) next -= C::kStages;
      issue(tile + (C::kStages - 1) * kE2m1Warps, next);
      look(tile + C::kStages * kE2m1Warps);
    }
    char* const st = ring + stage * L::kBytes;
    const int key0 = k0 + tile * kE2m1Tile;
    const bool full = key0 >= all_lo && key0 + kE2m1Tile <= all_hi;
    // V blocks that stand for NaN, in a tile that some row does not see all of: taken out here, put into the rows that see them below
    unsigned nan_blocks = 0, nan_keys = 0;
    if (!full) {
      unsigned char* vs = reinterpret_cast<unsigned char*>(st + L::kVs + lane * L::kSPitch);
#pragma unroll
      for (int i = 0; i < L::kSPitch; ++i)
        if ((vs[i] & 0x7f) == 0x7f) {
          nan_blocks |= 1u << i;
          vs[i] = 0;
        }
      nan_keys = __ballot_sync(0xffffffffu, nan_blocks != 0);  // also: the zeros are there for the others
      __syncwarp();
    }

    // ---- S^T = K Q^T, two times 16 keys
    float x[2][NT][4];
#pragma unroll
    for (int mt = 0; mt < 2; ++mt) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) x[mt][nt][0] = x[mt][nt][1] = x[mt][nt][2] = x[mt][nt][3] = 0.f;
      const int ka = 16 * mt + g;
      uint32_t w0[PT / 8], w1[PT / 8];
      load_words(st + ka * L::kKPitch + t * (PT / 2), w0);
      load_words(st + (ka + 8) * L::kKPitch + t * (PT / 2), w1);
      uint32_t s0[PT / 16], s1[PT / 16];  // a block's scale, twice
      if constexpr (PT == 16) {
        const unsigned char* p = reinterpret_cast<const unsigned char*>(st + L::kKs + ka * L::kSPitch + t);
        uint32_t a, c;
        e4m3x4_to_f16x2(__byte_perm(p[0], p[8 * L::kSPitch], 0x4400), a, c);
        s0[0] = a, s1[0] = c;
      } else if constexpr (PT == 32) {
        const uint16_t* p = reinterpret_cast<const uint16_t*>(st + L::kKs + ka * L::kSPitch + 2 * t);
        e4m3x4_to_f16x2(__byte_perm(p[0], 0, 0x1100), s0[0], s0[1]);
        e4m3x4_to_f16x2(__byte_perm(p[4 * L::kSPitch], 0, 0x1100), s1[0], s1[1]);
      } else {
        const uint32_t p0 = *reinterpret_cast<const uint32_t*>(st + L::kKs + ka * L::kSPitch + 4 * t);
        const uint32_t p1 = *reinterpret_cast<const uint32_t*>(st + L::kKs + (ka + 8) * L::kSPitch + 4 * t);
        e4m3x4_to_f16x2(__byte_perm(p0, 0, 0x1100), s0[0], s0[1]);
        e4m3x4_to_f16x2(__byte_perm(p0, 0, 0x3322), s0[2], s0[3]);
        e4m3x4_to_f16x2(__byte_perm(p1, 0, 0x1100), s1[0], s1[1]);
        e4m3x4_to_f16x2(__byte_perm(p1, 0, 0x3322), s1[2], s1[3]);
      }
#pragma unroll
      for (int w = 0; w < PT / 8; ++w) {
        uint32_t f0[4], f1[4];
        e2m1x8_to_f16x2(w0[w], f0);
        e2m1x8_to_f16x2(w1[w], f1);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          f0[k] = hmul2(f0[k], s0[w / 2]);
          f1[k] = hmul2(f1[k], s1[w / 2]);
        }
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            uint32_t b0, b1;
            if constexpr (C::kQShared) {
              const uint2 q = qs[(nt * KS + 2 * w + k) * 32 + lane];
              b0 = q.x, b1 = q.y;
            } else {
              b0 = qr[nt][2 * w + k][0], b1 = qr[nt][2 * w + k][1];
            }
            mma16816(x[mt][nt], f0[2 * k], f1[2 * k], f0[2 * k + 1], f1[2 * k + 1], b0, b1);
          }
      }
    }

    // ---- weights
    bool grew = false;
    float base[NT][2], fac[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        float top = kNegInf;
#pragma unroll
        for (int mt = 0; mt < 2; ++mt)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            float& v = x[mt][nt][2 * h + k];
            v = v * lift[nt][k] * A.c;
            const int key = key0 + 16 * mt + 8 * h + g;
            if (!full && (key < lo[nt][k] || key >= hi[nt][k])) v = kNegInf;
            top = fmaxf(top, v);
          }
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 4));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 8));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 16));
        const float mn = fmaxf(m[nt][k], top);
        grew = grew || mn > m[nt][k];
        base[nt][k] = mn == kNegInf ? 0.f : mn;
        fac[nt][k] = ex2(m[nt][k] - base[nt][k]);
        m[nt][k] = mn;
      }
    }
    if (__any_sync(0xffffffffu, grew)) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        l[nt][0] *= fac[nt][0];
        l[nt][1] *= fac[nt][1];
#pragma unroll
        for (int j = 0; j < KS; ++j) {
          o[j][nt][0] *= fac[nt][0];
          o[j][nt][1] *= fac[nt][1];
          o[j][nt][2] *= fac[nt][0];
          o[j][nt][3] *= fac[nt][1];
        }
      }
    }
    uint32_t pb[2][NT][2];
#pragma unroll
    for (int mt = 0; mt < 2; ++mt)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float p0 = ex2(x[mt][nt][2 * h] - base[nt][0] + kE2m1Lift), p1 = ex2(x[mt][nt][2 * h + 1] - base[nt][1] + kE2m1Lift);
          l[nt][0] += p0;
          l[nt][1] += p1;
          pb[mt][nt][h] = transpose8(f16_pack(p0, p1));
        }
      }

    // ---- O^T += V^T P^T
#pragma unroll
    for (int mt = 0; mt < 2; ++mt) {
      const int ka = 16 * mt + 2 * t;
      const char* v = st + L::kV + ka * L::kVPitch + g * (PG / 2);
      uint32_t w0[PG / 8], w1[PG / 8], w2[PG / 8], w3[PG / 8];
      load_words(v, w0);
      load_words(v + L::kVPitch, w1);
      load_words(v + 8 * L::kVPitch, w2);
      load_words(v + 9 * L::kVPitch, w3);
      uint32_t s01[PG > 16 ? 2 : 1], s23[PG > 16 ? 2 : 1];  // scales of keys 2t, 2t+1 and of 2t+8, 2t+9
#pragma unroll
      for (int k = 0; k < (PG > 16 ? 2 : 1); ++k) {
        const unsigned char* p = reinterpret_cast<const unsigned char*>(st + L::kVs + ka * L::kSPitch + (g * PG) / 16 + k);
        const uint32_t lo2 = p[0] | (uint32_t)p[L::kSPitch] << 8, hi2 = p[8 * L::kSPitch] | (uint32_t)p[9 * L::kSPitch] << 8;
        e4m3x4_to_f16x2(lo2 | hi2 << 16, s01[k], s23[k]);
      }
#pragma unroll
      for (int w = 0; w < PG / 8; ++w) {
        uint32_t a0[4], a1[4], a2[4], a3[4];
        constexpr uint32_t kLow = 0x0f0f0f0fu;
        e2m1x8_to_f16x2((w0[w] & kLow) | ((w1[w] << 4) & ~kLow), a0);
        e2m1x8_to_f16x2(((w0[w] >> 4) & kLow) | (w1[w] & ~kLow), a1);
        e2m1x8_to_f16x2((w2[w] & kLow) | ((w3[w] << 4) & ~kLow), a2);
        e2m1x8_to_f16x2(((w2[w] >> 4) & kLow) | (w3[w] & ~kLow), a3);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const uint32_t e0 = hmul2(a0[k], s01[w / 2]), e1 = hmul2(a1[k], s01[w / 2]), e2 = hmul2(a2[k], s23[w / 2]), e3 = hmul2(a3[k], s23[w / 2]);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) mma16816(o[4 * w + k][nt], e0, e1, e2, e3, pb[mt][nt][0], pb[mt][nt][1]);
        }
      }
    }
    while (nan_keys != 0) {
      const int k = __ffs(nan_keys) - 1, key = key0 + k;
      nan_keys &= nan_keys - 1;
      const unsigned blocks = __shfl_sync(0xffffffffu, nan_blocks, k);
#pragma unroll
      for (int j = 0; j < KS; ++j)
        if ((blocks >> ((g * PG + 2 * j) / 16)) & 1) {
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e)
              if (key >= lo[nt][e] && key < hi[nt][e]) o[j][nt][e] = o[j][nt][2 + e] = __int_as_float(0x7fc00000);
        }
    }
    if (++stage == C::kStages) stage = 0;
  }
  asm volatile("cp.async.wait_all;" ::: "memory");

  // ---- the four warps' parts
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      float v = l[nt][k];
      v += __shfl_xor_sync(0xffffffffu, v, 4);
      v += __shfl_xor_sync(0xffffffffu, v, 8);
      v += __shfl_xor_sync(0xffffffffu, v, 16);
      if (g == 0) {
        row_m[warp][nt * 8 + 2 * t + k] = m[nt][k];
        row_l[warp][nt * 8 + 2 * t + k] = v;
      }
    }
  __syncthreads();  // nobody reads tiles any more
  float* const all = reinterpret_cast<float*>(smem + C::kQBytes);
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      float* at = all + ((warp * NT + nt) * 8 + 2 * t + k) * C::kOPitch + g * PG;
#pragma unroll
      for (int j = 0; j < KS; ++j) *reinterpret_cast<float2*>(at + 2 * j) = make_float2(o[j][nt][k], o[j][nt][2 + k]);
    }
  __syncthreads();
  const bool whole = u.c0 == u.c1;
  for (int r = warp; r < 8 * NT; r += kE2m1Warps) {
    const long long rr = first + r;
    if (rr >= u.rows) break;
    float top = row_m[0][r];
#pragma unroll
    for (int w = 1; w < kE2m1Warps; ++w) top = fmaxf(top, row_m[w][r]);
    const float from = top == kNegInf ? 0.f : top;
    float sum = 0.f, share[kE2m1Warps];
#pragma unroll
    for (int w = 0; w < kE2m1Warps; ++w) {
      share[w] = ex2(row_m[w][r] - from);
      sum = fmaf(row_l[w][r], share[w], sum);
    }
    const float z = sum == 0.f ? kNegInf : from + log2f(sum) - kE2m1Lift, inv = sum == 0.f ? 0.f : 1.f / sum;
    const int i = (int)(rr / A.group), head = kvh * A.group + (int)(rr % A.group);
    const long long row = s.row0 + (long long)i;
    const long long part = (row * A.heads_q + head) * P.splits + chunk;
    for (int d = 2 * lane; d < A.head_dim; d += 64) {
      float2 v = make_float2(0.f, 0.f);
#pragma unroll
      for (int w = 0; w < kE2m1Warps; ++w) {
        const float2 a = *reinterpret_cast<const float2*>(all + (w * 8 * NT + r) * C::kOPitch + d);
        v.x = fmaf(a.x, share[w], v.x);
        v.y = fmaf(a.y, share[w], v.y);
      }
      v.x *= inv;
      v.y *= inv;
      if (whole) {
        uint16_t* out = A.out + row * A.ld_out + (long long)head * A.head_dim + d;
        IoBf16::store(out, 0, v.x * A.v_scale);
        IoBf16::store(out, 1, v.y * A.v_scale);
      } else {
        *reinterpret_cast<float2*>(P.part_o + part * A.head_dim + d) = v;
      }
    }
    if (lane == 0) {
      if (!whole) P.part_z[part] = z;
      else if (A.lse != nullptr) A.lse[row * A.heads_q + head] = z * kLn2;
    }
  }
}

// A warp per row and head of the rows with several chunks.
constexpr int kE2m1JoinThreads = 256;
__global__ void __launch_bounds__(kE2m1JoinThreads) attn_e2m1_join_kernel(const __grid_constant__ AttnE2m1Params P);

typedef void (*AttnE2m1Kernel)(const AttnE2m1Params);
// in qknorm_attn_e2m1_inst.cu; nt 1, 2 or 4 (2 at most for dp 256); smem, per_sm: of a CTA
AttnE2m1Kernel attn_e2m1_kernel_64(int nt, int copy, int* smem, int* per_sm);
AttnE2m1Kernel attn_e2m1_kernel_128(int nt, int copy, int* smem, int* per_sm);
AttnE2m1Kernel attn_e2m1_kernel_256(int nt, int copy, int* smem, int* per_sm);
AttnE2m1Kernel attn_e2m1_join_kernel_for();

// The visible part of a 4-bit cache as bf16 -- exact, the largest product of a code and a scale has six significant bits -- in pages of
// kE2m1Page tokens, heads one after the other in a page, the sequences' pages in a row: what "attn_tc" reads fastest.
constexpr int kE2m1Page = 128, kE2m1WidenThreads = 256;
struct WidenParams {
  AttnE2m1Params P;
  uint16_t* k;
  uint16_t* v;
  int* table;  // [seqs][cols]
  int cols;
};
typedef void (*WidenKernel)(const WidenParams);
WidenKernel e2m1_widen_kernel_for();

}  // namespace qknorm
