// Attention of new tokens over a 4-bit paged cache (include/qknorm_attn.h: qknorm_attn_paged_e2m1).
//
// Mathematics: as in qknorm_attn.cuh, with k = code * scale * k_scale.  A code has two significant bits and a scale four, so code * scale
// has six and is exact in fp16; the products are fp16 in, fp32 out.
//
// What bounds it: single tokens read 9/16 byte per element of K and V, a quarter of a bf16 cache, and have to widen every one of
// them.  So nothing is staged for the matrix unit: a warp takes 32 keys at a time as they lie in the cache, from shared memory, widens them in
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
// What holds it then, at 64 sequences of up to 8192 keys, 64 / 8 heads of 128 (102 us; its 382 MB take 58 at the copy rate): without its copies the kernel
// takes 83 us, without its arithmetic 76.  A tile of 32 keys is 136 widening conversions at two cycles each on one pipe, 128 packed products
// at two cycles on another, 32 matrix instructions at 8.8 and about 180 others; four warps of a scheduler alone with the K and V steps, out of registers, take
// 612 cycles a tile, all of it together 1018.  Tried and dropped: 64 keys a tile by cp.async (124 us against 123), V's words
// loaded before the weights (no difference), the scores of the next tile beside the weights and products of this one (101 against 99), four tiles of
// eight rows (spills; 60 rows 97 us against 74 with two), copies of one head's 16 tokens (124: the copy engine's time goes by the copy).
//
// Work: a unit is up to 8 NT query rows of a sequence and one key head for each warp as far as the CTA has heads; further warps take
// other keys of the same heads, and their parts are joined in shared memory.  A round is 32 keys for every warp.  With many heads to a CTA a
// copy brings a page's tokens of all of them.  See E2m1Item for how units come to CTAs.
#pragma once
#include "qknorm_attn.cuh"

namespace qknorm {

constexpr int kE2m1Tile = 32;     // keys that a warp takes at a time
constexpr int kE2m1Whole = 8;     // rounds up to which a unit is not cut, see E2m1Item
constexpr int kE2m1Error = 10;    // the device's error word: a stage did not come
// Weights are taken against a maximum that follows the running one only when a weight would pass 2^8 (kE2m1Slack), and are 2^7 times
// themselves (kE2m1Lift), so that they stay below fp16's 2^16 and the smallest are not lost.
constexpr float kE2m1Slack = 8.f, kE2m1Lift = 7.f;

struct AttnE2m1Params {
  AttnParams A;     // k, v: the codes, strides in bytes
  AttnSide ks, vs;  // the scales, strides in bytes
  int shares;       // units are cut into equal shares, see E2m1Item
  int row_tiles;    // per sequence and key head, at most
  int tile_rows;    // 8 NT
  int heads_cta;    // key heads of a CTA: 1, or by TMA a power of two up to its warps
  int run_shift;    // TMA: log2 of the tokens of a copy, 4 or 5
  int scale_unit;   // bytes that scales are copied by: 8 or 4 with cp.async, 2 or 1 without
  int q_vec;        // rows of q are 16-byte aligned
  int out_vec;      // rows of out are
  int* cuts;        // [grid][8]: the unit that began before the CTA's share and ends in it
  float* part_o;    // [grid][2][heads_cta * tile_rows][head_dim], normalised
  float* part_z;    // [grid][2][heads_cta * tile_rows], log2
};

struct E2m1Maps {  // [page][head][a page's tokens, one after the other]; elements of 8 bytes (codes) and 4 (scales)
  CUtensorMap k, v, ks, vs;
};

// How tiles come and lie in shared memory.  COPY 0: by TMA, runs of 16 or 32 tokens of all the CTA's heads per copy; a stage holds a tile
// for every warp, [run][head][token].  COPY 8, 16: any layout, by cp.async of that many bytes; stages are a warp's own.  The pitches keep
// the reads free of bank conflicts, but for V by TMA (two ways; see key_of).  WARPS: eight by cp.async for few short units, one CTA an SM.
constexpr int e2m1_warps(int nt, int copy) { return copy == 0 && nt == 1 ? 8 : 4; }
template <int DP, int NT, int COPY, int WARPS = e2m1_warps(NT, COPY)>
struct E2m1Cta {
  static constexpr int kWarps = WARPS, kThreads = 32 * kWarps;
  static constexpr int kStages = DP == 256 ? 2 : 3;
  static constexpr int kTiles = COPY == 0 ? kWarps : 1;  // of a stage
  static constexpr int kKPitch = DP == 256 ? 144 : DP / 2;
  static constexpr int kVPitch = COPY == 0 ? DP / 2 : DP == 64 ? 48 : DP == 128 ? 80 : 144;
  static constexpr int kSPitch = DP / 16;
  static constexpr int kV = kTiles * kE2m1Tile * kKPitch;
  static constexpr int kKs = kV + kTiles * kE2m1Tile * kVPitch;
  static constexpr int kVs = kKs + kTiles * kE2m1Tile * kSPitch;
  static constexpr int kBytes = kVs + kTiles * kE2m1Tile * kSPitch;
  static constexpr bool kQShared = DP * NT > 256;  // the query operand does not fit the registers beside the output
  static constexpr int kQHead = kQShared ? NT * (DP / 16) * 32 * 8 : 0;
  static constexpr int kQBytes = COPY == 0 ? kWarps * kQHead : kQHead;
  static constexpr int kRing = kStages * kBytes;   // of the CTA (TMA) or of a warp
  static constexpr int kAll = COPY == 0 ? kRing : kWarps * kRing;
  static constexpr int kOPitch = DP + 8;           // floats
  static constexpr int kJoin = kWarps * 8 * NT * kOPitch * 4;
  static constexpr int kSmem = 128 + kQBytes + (kJoin > kAll ? kJoin : kAll);
  static constexpr int kPerSm = COPY != 0 && kWarps == 8 ? 1 : DP == 256 || kWarps == 8 ? 2 : 3;
};
constexpr int kE2m1Runs = 256;  // runs whose pages are looked up at a time

// What the rows [first, first + tile_rows) of a sequence and key head see.
struct E2m1Span {
  unsigned rows;  // of the sequence; the host has checked that max_q * group fits
  int tok0, tok1, ulo, uhi, from;  // keys [ulo, uhi) that some row sees; from: ulo, rounded down to a tile
  int rounds;     // 0: no such rows; rows that see nothing take a round, too
};
__device__ __forceinline__ E2m1Span e2m1_span(const AttnE2m1Params& P, const AttnSeq& s, int rt, int round) {
  E2m1Span u;
  u.rows = (unsigned)s.n * (unsigned)P.A.group;
  const unsigned first = (unsigned)rt * (unsigned)P.tile_rows;
  u.rounds = u.tok0 = u.tok1 = u.ulo = u.uhi = u.from = 0;
  if (first >= u.rows) return u;
  const unsigned end = u.rows - first > (unsigned)P.tile_rows ? first + P.tile_rows : u.rows;
  u.tok0 = (int)(first / (unsigned)P.A.group);
  u.tok1 = (int)((end - 1) / (unsigned)P.A.group);
  u.ulo = attn_lo(P.A, s, u.tok0);
  u.uhi = attn_hi(P.A, s, u.tok1);
  u.rounds = 1;
  if (u.uhi <= u.ulo) {
    u.ulo = u.uhi = 0;
  } else {
    u.from = u.ulo & ~(kE2m1Tile - 1);
    u.rounds = (int)((unsigned)(u.uhi - u.from + round - 1) / (unsigned)round);
  }
  return u;
}

// A unit (sequence b, row tile rt, group of heads hg) or a part of it, rounds [r0, r1).  Where the longest units have few rounds, a CTA takes
// a whole unit.  Otherwise (shares) all rounds of all units in a row -- sequences, row tiles, groups fastest -- are cut into `grid` equal lengths, one
// for each CTA the GPU holds, so that all take the same time whatever the lengths of the sequences.  A part of a cut unit goes to one of
// its CTA's two slots, 0 if it is the first in the share, else 1, and attn_e2m1_join_kernel puts them together.
struct E2m1Item {
  AttnSeq s;
  E2m1Span u;
  int b, rt, hg;
  int r0, r1;
};
struct E2m1Start {
  int b, rt, hg, off;     // the share begins `off` rounds into this unit
  long long left;         // rounds of the share
  long long unit;         // where its first unit begins
  long long total;
};
__device__ __forceinline__ long long e2m1_share(long long total, int grid, int c) {  // where share c begins
  const long long q = total >> 31 == 0 ? (long long)((unsigned)total / (unsigned)grid) : total / grid, more = total - q * grid;
  return c * q + (c < more ? c : more);
}
// The share that holds round `at`.
__device__ __forceinline__ int e2m1_share_of(long long total, int grid, long long at) {
  const long long q = total / grid, more = total - q * grid;
  return (int)(at < more * (q + 1) ? at / (q + 1) : more + (at - more * (q + 1)) / q);
}
// By the whole CTA.  scratch: a long long for every warp; both in shared memory.
__device__ __forceinline__ void e2m1_find(const AttnE2m1Params& P, int groups, int round, long long* scratch, E2m1Start* out) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, warps = blockDim.x >> 5;
  const int n = P.A.seqs * P.row_tiles;  // the host has checked that it fits
  const int per = (n + blockDim.x - 1) / blockDim.x;
  const int n0 = per * tid < n ? per * tid : n, n1 = n0 + per < n ? n0 + per : n;
  long long sum = 0;
  for (int i = n0; i < n1; ++i) {
    const int b = i / P.row_tiles;
    sum += (long long)e2m1_span(P, attn_seq(P.A, b), i - b * P.row_tiles, round).rounds * groups;
  }
  long long upto = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long v = __shfl_up_sync(0xffffffffu, upto, o);
    if (lane >= o) upto += v;
  }
  if (lane == 31) scratch[warp] = upto;
  if (tid == 0) out->left = 0;
  __syncthreads();
  long long before = 0, total = 0;
  for (int w = 0; w < warps; ++w) {
    if (w < warp) before += scratch[w];
    total += scratch[w];
  }
  long long at = before + upto - sum;  // this thread's first unit
  const long long begin = e2m1_share(total, P.A.grid, blockIdx.x), end = e2m1_share(total, P.A.grid, blockIdx.x + 1);
  if (begin < end && begin >= at && begin < at + sum) {
    for (int i = n0; i < n1; ++i) {
      const int b = i / P.row_tiles, rt = i - b * P.row_tiles;
      const int w = e2m1_span(P, attn_seq(P.A, b), rt, round).rounds;
      if (begin < at + (long long)w * groups) {
        const int hg = (int)((begin - at) / w);
        *out = E2m1Start{b, rt, hg, (int)(begin - at - (long long)hg * w), end - begin, at + (long long)hg * w, total};
        break;
      }
      at += (long long)w * groups;
    }
  }
  __syncthreads();
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
// One copy: [1 page][heads of the CTA][tokens of a run] from element x of the page, head, page.
__device__ __forceinline__ void e2m1_load(uint32_t dst, const CUtensorMap* map, int x, int head, int page, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.3d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst), "l"(map), "r"(x),
               "r"(head), "r"(page), "r"(bar)
               : "memory");
}

// What a warp holds: its rows' queries and running results; and what it does with a tile of 32 keys.
template <int DP, int NT, int COPY>
struct E2m1Core {
  using C = E2m1Cta<DP, NT, COPY>;
  static constexpr int KS = DP / 16;  // steps of 16 dims
  static constexpr int PT = DP / 4;   // dims of a thread in S^T
  static constexpr int PG = DP / 8;   // dims of a thread in O^T
  static constexpr int MT = kE2m1Tile / 16;

  uint32_t qr[C::kQShared ? 1 : NT][C::kQShared ? 1 : KS][2];
  float2 cl[NT];  // c 2^e of this thread's score rows 2t, 2t + 1
  int lo[NT][2], hi[NT][2];
  float o[KS][NT][4];  // [DP / 16 pairs of dims][..][dim 2j: rows 2t, 2t + 1; dim 2j + 1: the same]
  // rows 2t, 2t + 1: the score that weights are taken against -- the difference to it is what is multiplied by cl, so that the largest
  // weight is 1 however large the scores are -- and this thread's share of the weights' sum
  float2 m[NT], l[NT];

  // Which key stands in row r of a block of 8: by TMA the rows are 16 banks apart, and an order in which rows 0, 2, 4, 6 and
  // rows 2i, 2i + 1 are keys of both parities halves the conflicts.
  static __device__ __forceinline__ int key_of(int r) { return COPY == 0 ? r ^ ((r >> 1) & 1) : r; }

  // Queries: row g of every tile of 8, dims [t PT, (t + 1) PT), as fp16 times 2^-e.
  __device__ __forceinline__ void start(const AttnE2m1Params& P, const AttnSeq& s, int kvh, unsigned first, unsigned rows, uint2* qs, bool writes) {
    const AttnParams& A = P.A;
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const unsigned group = (unsigned)A.group;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const unsigned r = first + nt * 8 + g;
      const bool there = r < rows;
      const int i = there ? (int)(r / group) : 0, head = kvh * A.group + (there ? (int)(r - i * group) : 0);
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
      uint32_t top = 0;  // the larger bit patterns without their signs are the larger magnitudes
#pragma unroll
      for (int j = 0; j < PT / 2; ++j) top = __vmaxu2(top, w[j] & 0x7fff7fffu);
      top = __vmaxu2(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = __vmaxu2(top, __shfl_xor_sync(0xffffffffu, top, 2));
      top = (top & 0xffffu) > (top >> 16) ? top & 0xffffu : top >> 16;
      // the row's largest element comes to [2^14, 2^15); a row with an infinity or NaN is scaled as if its finite elements were the largest
      const int e = ((int)(top >> 7) < 254 ? (int)(top >> 7) : 254) - 127 - 14;
      const float f_a = __int_as_float((127 - e / 2) << 23), f_b = __int_as_float((127 - (e - e / 2)) << 23);  // 2^-e may not be an fp32 value
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        uint32_t f[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) f[k] = f16_pack(bf_lo(w[2 * ks + k]) * f_a * f_b, bf_hi(w[2 * ks + k]) * f_a * f_b);
        if constexpr (C::kQShared) {
          if (writes) qs[(nt * KS + ks) * 32 + lane] = make_uint2(f[0], f[1]);
        } else {
          qr[nt][ks][0] = f[0];
          qr[nt][ks][1] = f[1];
        }
      }
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        // positive and finite, whatever c and e: a score of 0 stays one, and of -inf too
        (k ? cl[nt].y : cl[nt].x) = fminf(fmaxf(ldexpf(A.c, __shfl_sync(0xffffffffu, e, 4 * (2 * t + k))), kAttnLeastC), 3.4e38f);
        const unsigned rr = first + nt * 8 + 2 * t + k;
        const int ii = __shfl_sync(0xffffffffu, i, 4 * (2 * t + k));
        lo[nt][k] = hi[nt][k] = 0;
        if (rr < rows) {
          lo[nt][k] = attn_lo(A, s, ii);
          hi[nt][k] = attn_hi(A, s, ii);
        }
      }
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      m[nt] = make_float2(kNegInf, kNegInf);
      l[nt] = make_float2(0.f, 0.f);
#pragma unroll
      for (int j = 0; j < KS; ++j) o[j][nt][0] = o[j][nt][1] = o[j][nt][2] = o[j][nt][3] = 0.f;
    }
  }

  // st_*: where the tile's first 16 keys lie in shared memory; its second 16 lie `jump` keys behind them.  full: every row sees all of it.
  __device__ __forceinline__ void tile(const char* st_k, const char* st_v, const char* st_ks, char* st_vs, int jump, int key0, bool full, const uint2* qs) {
    const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    // V blocks that stand for NaN, in a tile that some row does not see all of: taken out here, put into the rows that see them below
    unsigned nan_blocks = 0, nan_keys = 0;
    if (!full) {
      unsigned char* vs = reinterpret_cast<unsigned char*>(st_vs + ((lane & 15) + (lane >> 4) * jump) * C::kSPitch);
#pragma unroll
      for (int i = 0; i < C::kSPitch; ++i)
        if ((vs[i] & 0x7f) == 0x7f) {
          nan_blocks |= 1u << i;
          vs[i] = 0;
        }
      nan_keys = __ballot_sync(0xffffffffu, nan_blocks != 0);
      if (COPY == 0 && nan_keys != 0) ptx::fence_proxy_async();  // the stage's next copies come after these
      __syncwarp();  // the zeros are there for the others
    }

    // ---- S^T = K Q^T, 16 keys at a time
    float x[MT][NT][4];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) x[mt][nt][0] = x[mt][nt][1] = x[mt][nt][2] = x[mt][nt][3] = 0.f;
      const int ka = mt * jump + key_of(g);
      uint32_t w0[PT / 8], w1[PT / 8];
      load_words(st_k + ka * C::kKPitch + t * (PT / 2), w0);
      load_words(st_k + (ka + 8) * C::kKPitch + t * (PT / 2), w1);
      uint32_t s0[PT / 16], s1[PT / 16];  // a block's scale, twice
      if constexpr (PT == 16) {
        const unsigned char* p = reinterpret_cast<const unsigned char*>(st_ks + ka * C::kSPitch + t);
        uint32_t a, c;
        e4m3x4_to_f16x2(__byte_perm(p[0], p[8 * C::kSPitch], 0x4400), a, c);
        s0[0] = a, s1[0] = c;
      } else if constexpr (PT == 32) {
        const uint16_t* p = reinterpret_cast<const uint16_t*>(st_ks + ka * C::kSPitch + 2 * t);
        e4m3x4_to_f16x2(__byte_perm(p[0], 0, 0x1100), s0[0], s0[1]);
        e4m3x4_to_f16x2(__byte_perm(p[4 * C::kSPitch], 0, 0x1100), s1[0], s1[1]);
      } else {
        const uint32_t p0 = *reinterpret_cast<const uint32_t*>(st_ks + ka * C::kSPitch + 4 * t);
        const uint32_t p1 = *reinterpret_cast<const uint32_t*>(st_ks + (ka + 8) * C::kSPitch + 4 * t);
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
    if (!full) {
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int key = key0 + 16 * mt + 8 * h + key_of(g);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int k = 0; k < 2; ++k)
              if (key < lo[nt][k] || key >= hi[nt][k]) x[mt][nt][2 * h + k] = kNegInf;
        }
    }
    bool grew = false;
    float2 top[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {  // NaN passes by; its weight below will be NaN
      top[nt] = make_float2(fmaxf(x[0][nt][0], x[0][nt][2]), fmaxf(x[0][nt][1], x[0][nt][3]));
#pragma unroll
      for (int mt = 1; mt < MT; ++mt) {
        top[nt].x = fmaxf(top[nt].x, fmaxf(x[mt][nt][0], x[mt][nt][2]));
        top[nt].y = fmaxf(top[nt].y, fmaxf(x[mt][nt][1], x[mt][nt][3]));
      }
      grew = grew || (top[nt].x - m[nt].x) * cl[nt].x > kE2m1Slack || (top[nt].y - m[nt].y) * cl[nt].y > kE2m1Slack;
    }
    if (__any_sync(0xffffffffu, grew)) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        auto grow = [&](float v, float& now, float scale) {
          v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 4));
          v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 8));
          v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 16));
          v = fmaxf(v, now);
          const float f = v == now ? 1.f : ex2((now - v) * scale);
          now = v;
          return f;
        };
        float2 fac;
        fac.x = grow(top[nt].x, m[nt].x, cl[nt].x);
        fac.y = grow(top[nt].y, m[nt].y, cl[nt].y);
        l[nt] = __fmul2_rn(l[nt], fac);
#pragma unroll
        for (int j = 0; j < KS; ++j)
#pragma unroll
          for (int h = 0; h < 4; h += 2) {
            const float2 v = __fmul2_rn(make_float2(o[j][nt][h], o[j][nt][h + 1]), fac);
            o[j][nt][h] = v.x;
            o[j][nt][h + 1] = v.y;
          }
      }
    }
    uint32_t pb[MT][NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const float2 less = make_float2(m[nt].x == kNegInf ? 0.f : -m[nt].x, m[nt].y == kNegInf ? 0.f : -m[nt].y);
#pragma unroll
      for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float2 d = __fadd2_rn(make_float2(x[mt][nt][2 * h], x[mt][nt][2 * h + 1]), less);
          float2 p = __ffma2_rn(d, cl[nt], make_float2(kE2m1Lift, kE2m1Lift));
          p.x = ex2(p.x);
          p.y = ex2(p.y);
          l[nt] = __fadd2_rn(l[nt], p);
          pb[mt][nt][h] = transpose8(f16_pack(p.x, p.y));
        }
    }

    // ---- O^T += V^T P^T
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      const int ka = mt * jump + key_of(2 * t), kc = mt * jump + key_of(2 * t + 1);
      const char* va = st_v + ka * C::kVPitch + g * (PG / 2);
      const char* vc = st_v + kc * C::kVPitch + g * (PG / 2);
      uint32_t w0[PG / 8], w1[PG / 8], w2[PG / 8], w3[PG / 8];
      load_words(va, w0);
      load_words(vc, w1);
      load_words(va + 8 * C::kVPitch, w2);
      load_words(vc + 8 * C::kVPitch, w3);
      uint32_t s01[PG > 16 ? 2 : 1], s23[PG > 16 ? 2 : 1];  // scales of keys 2t, 2t+1 and of 2t+8, 2t+9
#pragma unroll
      for (int k = 0; k < (PG > 16 ? 2 : 1); ++k) {
        const unsigned char* pa = reinterpret_cast<const unsigned char*>(st_vs + ka * C::kSPitch + (g * PG) / 16 + k);
        const unsigned char* pc = reinterpret_cast<const unsigned char*>(st_vs + kc * C::kSPitch + (g * PG) / 16 + k);
        const uint32_t lo2 = pa[0] | (uint32_t)pc[0] << 8, hi2 = pa[8 * C::kSPitch] | (uint32_t)pc[8 * C::kSPitch] << 8;
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
  }
};

// DP: head_dim padded; NT: tiles of 8 query rows; COPY, WARPS: see E2m1Cta.
template <int DP, int NT, int COPY, int WARPS>
__global__ void __launch_bounds__(E2m1Cta<DP, NT, COPY, WARPS>::kThreads, E2m1Cta<DP, NT, COPY, WARPS>::kPerSm)
    attn_e2m1_kernel(const __grid_constant__ AttnE2m1Params P, const __grid_constant__ E2m1Maps maps) {
  using C = E2m1Cta<DP, NT, COPY, WARPS>;
  using Core = E2m1Core<DP, NT, COPY>;
  constexpr bool kTma = COPY == 0;
  constexpr int kWarps = C::kWarps;
  extern __shared__ __align__(128) uint4 smem_e2m1[];
  __shared__ float row_m[kWarps][8 * NT], row_l[kWarps][8 * NT], row_c[kWarps][8 * NT];
  __shared__ int run_page[kTma ? kE2m1Runs : 1];
  __shared__ __align__(8) unsigned long long bars[C::kStages];
  __shared__ unsigned done[C::kStages];  // warps that have read the stage
  __shared__ long long scratch[kWarps];
  __shared__ E2m1Start start;
  const AttnParams& A = P.A;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
  const int HP = kTma ? P.heads_cta : 1, slices = kWarps / HP, h = warp % HP, slice = warp / HP;
  const int round = slices * kE2m1Tile;  // keys that the CTA takes at a time
  char* const smem = reinterpret_cast<char*>(smem_e2m1) + (-ptx::smem_u32(smem_e2m1) & 127u);  // TMA wants 128 bytes
  char* const ring = smem + C::kQBytes + (kTma ? 0 : warp * C::kRing);
  const uint32_t ring32 = ptx::smem_u32(ring), bar32 = ptx::smem_u32(bars), done32 = ptx::smem_u32(done);

  const int groups = A.heads_kv / HP;
  if constexpr (kTma) {
    if (threadIdx.x == 0) {
#pragma unroll
      for (int i = 0; i < C::kStages; ++i) {
        ptx::mbar_init(bar32 + 8 * i, 1);
        done[i] = 0;
      }
      ptx::fence_barrier_init();
    }
    __syncthreads();
  }
  asm volatile("griddepcontrol.wait;" ::: "memory");

  E2m1Item w;
  long long left = 0;
  if (P.shares) {
    e2m1_find(P, groups, round, scratch, &start);
    left = start.left;
    w.b = start.b;
    w.rt = start.rt;
    w.hg = start.hg;
    w.r0 = start.off;
  } else {
    unsigned idx = blockIdx.x;
    w.rt = idx % (unsigned)P.row_tiles;
    idx /= (unsigned)P.row_tiles;
    w.hg = idx % (unsigned)groups;
    w.b = idx / (unsigned)groups;
    w.r0 = 0;
  }
  if (!P.shares || left > 0) {
    w.s = attn_seq(A, w.b);
    w.u = e2m1_span(P, w.s, w.rt, round);
    if (!P.shares) left = w.u.rounds;
  }
  bool first_item = true, failed = false;
  int stage = 0;
  Core core;
  unsigned parity = 0;

  if (left <= 0) {
    if (P.shares && threadIdx.x == 0) P.cuts[blockIdx.x * 8] = -1;
    return;
  }
  w.r1 = left < w.u.rounds - w.r0 ? w.r0 + (int)left : w.u.rounds;
  const unsigned group = (unsigned)A.group;

  // ---- TMA: round it of the unit; the pages of a stretch of rounds are looked up once
  int seg = 0, seg_end = 0;  // the rounds of the stretch
  auto fill = [&](int it, int stage) {  // by one warp
    const int run = 1 << P.run_shift, runs = round >> P.run_shift;
    const uint32_t at = ring32 + stage * C::kBytes, bar = bar32 + 8 * stage;
    if (lane == 0) ptx::mbar_arrive_expect_tx(bar, C::kBytes);
    __syncwarp();
    if (lane < runs) {
      const int page = run_page[(it - seg) * runs + lane];
      const int key = w.u.from + it * round + lane * run, head0 = w.hg * HP;
      const int in_page = A.page_shift >= 0 ? key & (A.page_size - 1) : (int)((unsigned)key % (unsigned)A.page_size);
      const int i0 = lane * HP * run;  // where the run starts in the stage, in tokens of a head
      e2m1_load(at + i0 * C::kKPitch, &maps.k, in_page * (DP / 16), head0, page, bar);
      e2m1_load(at + C::kV + i0 * C::kVPitch, &maps.v, in_page * (DP / 16), head0, page, bar);
      e2m1_load(at + C::kKs + i0 * C::kSPitch, &maps.ks, in_page * (DP / 64), head0, page, bar);
      e2m1_load(at + C::kVs + i0 * C::kSPitch, &maps.vs, in_page * (DP / 64), head0, page, bar);
    }
    __syncwarp();
  };
  // ---- cp.async: a lane looks up the page of one key of its warp's tile
  const int row_bytes = A.head_dim >> 1, scale_bytes = A.head_dim >> 4;
  int page = -1, within = 0;  // of this lane's key in the tile that is issued next
  auto look = [&](int it) {
    page = -1;
    within = 0;
    const int key = w.u.from + it * round + slice * kE2m1Tile + lane;
    if (it < w.r1 && key < w.u.uhi && key >= w.u.ulo) page = (int)attn_page(A, w.b, key, within);
  };
  auto issue = [&](int it, int stage) {
    if (it < w.r1) {
      const int kvh = w.hg * HP + h;
      const char* const kb = reinterpret_cast<const char*>(A.k.base) + kvh * A.k.head;
      const char* const vb = reinterpret_cast<const char*>(A.v.base) + kvh * A.v.head;
      const char* const ksb = reinterpret_cast<const char*>(P.ks.base) + kvh * P.ks.head;
      const char* const vsb = reinterpret_cast<const char*>(P.vs.base) + kvh * P.vs.head;
      const uint32_t at = ring32 + stage * C::kBytes;
      const bool there = page >= 0;
      const unsigned long long pp = there ? (unsigned)page : 0u;
      const unsigned long long ka = there ? pp * A.k.page + within * A.k.token : ~0ull;
      const unsigned long long va = pp * A.v.page + within * A.v.token;
      constexpr int kCopy = COPY == 0 ? 16 : COPY, kPer = DP / 2 / kCopy;  // copies of a row
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const int key = (lane + 32 * i) / kPer, part = (lane + 32 * i) % kPer;
        const unsigned long long kk = __shfl_sync(0xffffffffu, ka, key), vv = __shfl_sync(0xffffffffu, va, key);
        const bool ok = kk != ~0ull;
        if (part * kCopy < row_bytes) {
          copy_or_zero<kCopy>(at + key * C::kKPitch + part * kCopy, kb + (ok ? kk + part * kCopy : 0), ok);
          copy_or_zero<kCopy>(at + C::kV + key * C::kVPitch + part * kCopy, vb + (ok ? vv + part * kCopy : 0), ok);
        }
      }
      const char* ks = ksb + (there ? pp * P.ks.page + within * P.ks.token : 0);
      const char* vs = vsb + (there ? pp * P.vs.page + within * P.vs.token : 0);
      const int ks_at = C::kKs + lane * C::kSPitch, vs_at = C::kVs + lane * C::kSPitch;
      if (P.scale_unit == 8) {
        if constexpr (DP >= 128) {
#pragma unroll
          for (int i = 0; i < C::kSPitch; i += 8)
            if (i < scale_bytes) {
              copy_or_zero<8>(at + ks_at + i, ks + i, there);
              copy_or_zero<8>(at + vs_at + i, vs + i, there);
            }
        }
      } else if (P.scale_unit == 4) {
#pragma unroll
        for (int i = 0; i < C::kSPitch; i += 4)
          if (i < scale_bytes) {
            copy_or_zero<4>(at + ks_at + i, ks + i, there);
            copy_or_zero<4>(at + vs_at + i, vs + i, there);
          }
      } else {
        unsigned char* st = reinterpret_cast<unsigned char*>(ring + stage * C::kBytes);
        for (int i = 0; i < scale_bytes; ++i) {
          st[ks_at + i] = there ? (unsigned char)ks[i] : 0;
          st[vs_at + i] = there ? (unsigned char)vs[i] : 0;
        }
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  // The first copies of a stretch of w's rounds.  Whoever calls this again has seen to it that nobody reads the stages, or run_page, any more.
  auto prime = [&](int from) {
    seg = from;
    seg_end = w.r1;
    if (w.u.uhi <= w.u.ulo) return;  // a round without keys
    if constexpr (kTma) {
      const int most = (kE2m1Runs << P.run_shift) / round;
      if (seg_end - seg > most) seg_end = seg + most;
      const int runs = (seg_end - seg) * round >> P.run_shift;
      for (int i = threadIdx.x; i < runs; i += C::kThreads) {
        const long long key = w.u.from + (long long)seg * round + ((long long)i << P.run_shift);
        int in_page = 0, p = -1;  // -1 reads as zeros, as every coordinate outside does
        if (key < w.u.uhi && key + (1 << P.run_shift) > w.u.ulo) p = (int)attn_page(A, w.b, (int)key, in_page);
        run_page[i] = p;
      }
      __syncthreads();
      for (int i = warp; i < C::kStages && seg + i < seg_end; i += kWarps) fill(seg + i, (stage + i) % C::kStages);
    } else {
      stage = 0;
      if (A.head_dim < DP) {  // what no copy writes has to be zero
        for (int i = lane; i < C::kRing / 16; i += 32) reinterpret_cast<uint4*>(ring)[i] = make_uint4(0, 0, 0, 0);
        __syncwarp();
      }
#pragma unroll 1
      for (int i = 0; i < C::kStages - 1; ++i) {
        look(seg + i);
        issue(seg + i, i);
      }
      look(seg + C::kStages - 1);
    }
  };
  prime(w.r0);
  if (P.shares && threadIdx.x == 0) {  // for the join: the unit that this share ends but has not begun
    int* cut = P.cuts + blockIdx.x * 8;
    cut[0] = -1;
    if (start.off > 0 && w.r1 == w.u.rounds) {
      const int from = e2m1_share_of(start.total, A.grid, start.unit);
      cut[1] = start.rt;
      cut[2] = start.hg;
      cut[3] = from;
      cut[4] = e2m1_share(start.total, A.grid, from) == start.unit ? 0 : 1;
      cut[0] = start.b;
    }
  }

  for (;;) {
    uint2* const qs = reinterpret_cast<uint2*>(smem + h * C::kQHead);
    core.start(P, w.s, w.hg * HP + h, (unsigned)w.rt * (8 * NT), w.u.rows, qs, slice == 0);
    if constexpr (C::kQShared) __syncthreads();
    // keys that every row sees
    const int all_lo = attn_lo(A, w.s, w.u.tok1), all_hi = attn_hi(A, w.s, w.u.tok0), k1 = w.u.uhi;
    // the tile's place in a stage, in tokens of a head
    const int tile_at = kTma ? ((slice * kE2m1Tile >> P.run_shift) * HP + h) << P.run_shift : 0;
    const int jump = kTma && P.run_shift == 4 ? 16 * HP : 16;

    while (w.u.uhi > w.u.ulo) {
      const int end = seg_end;
      for (int it = seg; it < end; ++it) {
        if constexpr (kTma) {
          if (__any_sync(0xffffffffu, !ptx::mbar_wait_bounded(bar32 + 8 * stage, parity))) {
            // never seen: the rows come out wrong and the error word says so; what is still on its way gets the same time again
            if (lane == 0) *A.error = kE2m1Error;
            for (int i = 0; i < C::kStages; ++i)
              if (it + i < end) ptx::mbar_wait_bounded(bar32 + 8 * ((stage + i) % C::kStages), parity ^ (stage + i >= C::kStages ? 1u : 0u));
            failed = true;
            break;
          }
        } else {
          asm volatile("cp.async.wait_group %0;" ::"n"(C::kStages - 2) : "memory");
          __syncwarp();  // every lane's copies have landed, and nobody reads the stage that is filled next
          int next = stage + C::kStages - 1;
          if (next >= C::kStages) next -= C::kStages;
          issue(it + C::kStages - 1, next);
          look(it + C::kStages);
        }
        char* const st = ring + stage * C::kBytes;
        const int key0 = w.u.from + it * round + slice * kE2m1Tile;
        if (key0 < k1)
          core.tile(st + tile_at * C::kKPitch, st + C::kV + tile_at * C::kVPitch, st + C::kKs + tile_at * C::kSPitch, st + C::kVs + tile_at * C::kSPitch,
                    jump, key0, key0 >= all_lo && key0 + kE2m1Tile <= all_hi, qs);
        if constexpr (kTma) {  // the last warp that has read a stage fills it again: nobody waits for the others
          __syncwarp();
          if (it + C::kStages < end) {
            unsigned before = 0;
            if (lane == 0)
              asm volatile("atom.acq_rel.cta.shared::cta.inc.u32 %0, [%1], %2;" : "=r"(before) : "r"(done32 + 4 * stage), "r"(kWarps - 1) : "memory");
            if (__shfl_sync(0xffffffffu, before, 0) == kWarps - 1) fill(it + C::kStages, stage);
          }
        }
        if (++stage == C::kStages) {
          stage = 0;
          parity ^= 1;
        }
      }
      if constexpr (kTma) {
        if (__syncthreads_or(failed)) return;  // everybody has seen the stretch's copies land, or has given up on them
      }
      if (end == w.r1) break;
      prime(end);
    }
    if constexpr (!kTma) asm volatile("cp.async.wait_all;" ::: "memory");

    // ---- the next unit; where a warp has its head to itself, its first copies come while the results of this one leave
    const E2m1Item now = w;
    const int now_slot = first_item ? 0 : 1;
    left -= w.r1 - w.r0;
    if (left > 0) {
      first_item = false;
      w.r0 = 0;
      do {
        if (++w.hg == groups) {
          w.hg = 0;
          if (++w.rt == P.row_tiles) {
            w.rt = 0;
            if (++w.b == A.seqs) return;  // never: the shares add up to the units
            w.s = attn_seq(A, w.b);
          }
          w.u = e2m1_span(P, w.s, w.rt, round);
        }
      } while (w.u.rounds == 0);
      w.r1 = left < w.u.rounds ? (int)left : w.u.rounds;
      if (kTma && slices == 1) prime(0);
    }
    const AttnSeq& s = now.s;
    const E2m1Span& u = now.u;
    const unsigned first = (unsigned)now.rt * (8 * NT);
    const bool whole = now.r0 == 0 && now.r1 == u.rounds;
    if (slices == 1) {  // ---- a warp has its head to itself: straight from its registers
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          float sum = k ? core.l[nt].y : core.l[nt].x;
          sum += __shfl_xor_sync(0xffffffffu, sum, 4);
          sum += __shfl_xor_sync(0xffffffffu, sum, 8);
          sum += __shfl_xor_sync(0xffffffffu, sum, 16);
          const float top = k ? core.m[nt].y : core.m[nt].x, c = k ? core.cl[nt].y : core.cl[nt].x;
          const unsigned r = nt * 8 + 2 * t + k, rr = first + r;
          if (rr >= u.rows) continue;
          const float z = sum == 0.f ? kNegInf : fmaf(top == kNegInf ? 0.f : top, c, log2f(sum)) - kE2m1Lift, inv = sum == 0.f ? 0.f : 1.f / sum;
          const int i = (int)(rr / group), head = (now.hg * HP + h) * A.group + (int)(rr - i * group);
          const long long row = s.row0 + (long long)i;
          const long long part = ((long long)blockIdx.x * 2 + now_slot) * (HP * 8 * NT) + h * 8 * NT + r;
          if (whole) {
            const float scale = inv * A.v_scale;
            uint16_t* out = A.out + row * A.ld_out + (long long)head * A.head_dim + g * Core::PG;
#pragma unroll
            for (int j = 0; j < Core::KS; j += 4) {
              uint32_t v[4];
#pragma unroll
              for (int e = 0; e < 4; ++e) v[e] = bf_pack(core.o[j + e][nt][k] * scale, core.o[j + e][nt][2 + k] * scale);
              if (P.out_vec) {
                *reinterpret_cast<uint4*>(out + 2 * j) = make_uint4(v[0], v[1], v[2], v[3]);
              } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) out[2 * j + e] = (uint16_t)(v[e / 2] >> (16 * (e & 1)));
              }
            }
          } else {
            float* po = P.part_o + part * A.head_dim + g * Core::PG;
#pragma unroll
            for (int j = 0; j < Core::KS; j += 2)
              *reinterpret_cast<float4*>(po + 2 * j) = make_float4(core.o[j][nt][k] * inv, core.o[j][nt][2 + k] * inv, core.o[j + 1][nt][k] * inv,
                                                                   core.o[j + 1][nt][2 + k] * inv);
          }
          if (g == 0) {
            if (!whole) P.part_z[part] = z;
            else if (A.lse != nullptr) A.lse[row * A.heads_q + head] = z * kLn2;
          }
        }
    } else {  // ---- the parts of the warps of a head
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          float v = k ? core.l[nt].y : core.l[nt].x;
          v += __shfl_xor_sync(0xffffffffu, v, 4);
          v += __shfl_xor_sync(0xffffffffu, v, 8);
          v += __shfl_xor_sync(0xffffffffu, v, 16);
          if (g == 0) {
            row_m[warp][nt * 8 + 2 * t + k] = k ? core.m[nt].y : core.m[nt].x;
            row_c[warp][nt * 8 + 2 * t + k] = k ? core.cl[nt].y : core.cl[nt].x;
            row_l[warp][nt * 8 + 2 * t + k] = v;
          }
        }
      __syncthreads();  // nobody reads tiles any more
      float* const all = reinterpret_cast<float*>(smem + C::kQBytes);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          float* at = all + ((warp * NT + nt) * 8 + 2 * t + k) * C::kOPitch + g * Core::PG;
#pragma unroll
          for (int j = 0; j < Core::KS; ++j) *reinterpret_cast<float2*>(at + 2 * j) = make_float2(core.o[j][nt][k], core.o[j][nt][2 + k]);
        }
      __syncthreads();
      for (int item = warp; item < HP * 8 * NT; item += kWarps) {
        const int r = item / HP, w0 = item % HP;  // the head's warps: w0, w0 + HP, ...
        const unsigned rr = first + r;
        if (rr >= u.rows) break;
        float top = row_m[w0][r];
        for (int w = w0 + HP; w < kWarps; w += HP) top = fmaxf(top, row_m[w][r]);
        const float against = top == kNegInf ? 0.f : top, c = row_c[w0][r];
        float sum = 0.f;
        for (int w = w0; w < kWarps; w += HP) sum = fmaf(row_l[w][r], ex2((row_m[w][r] - against) * c), sum);
        const float z = sum == 0.f ? kNegInf : fmaf(against, c, log2f(sum)) - kE2m1Lift, inv = sum == 0.f ? 0.f : 1.f / sum;
        const int i = (int)(rr / group), head = (now.hg * HP + w0) * A.group + (int)(rr - i * group);
        const long long row = s.row0 + (long long)i;
        const long long part = ((long long)blockIdx.x * 2 + now_slot) * (HP * 8 * NT) + w0 * 8 * NT + r;
        for (int d = 2 * lane; d < A.head_dim; d += 64) {
          float2 v = make_float2(0.f, 0.f);
          for (int w = w0; w < kWarps; w += HP) {
            const float2 a = *reinterpret_cast<const float2*>(all + (w * 8 * NT + r) * C::kOPitch + d);
            const float share = ex2((row_m[w][r] - against) * c);
            v.x = fmaf(a.x, share, v.x);
            v.y = fmaf(a.y, share, v.y);
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
    if (left <= 0) break;
    if (!kTma || slices != 1) {
      if constexpr (kTma) ptx::fence_proxy_async();  // copies go where the parts were
      __syncthreads();
      prime(0);
    }
  }
}

// Puts the parts of cut units together: a CTA per share and eight rows of a unit, a warp per row.
constexpr int kE2m1JoinThreads = 256;
__global__ void __launch_bounds__(kE2m1JoinThreads) attn_e2m1_join_kernel(const __grid_constant__ AttnE2m1Params P);

typedef void (*AttnE2m1Kernel)(const AttnE2m1Params, const E2m1Maps);
typedef void (*AttnE2m1JoinKernel)(const AttnE2m1Params);
struct E2m1Launch {
  AttnE2m1Kernel fn;
  int smem, warps, per_sm;
};
// in qknorm_attn_e2m1_inst.cu; nt 1 or 2; copy 0 (not for dp 256), 8 or 16; wide: eight warps by cp.async, nt 1
E2m1Launch attn_e2m1_kernel_64(int nt, int copy, bool wide);
E2m1Launch attn_e2m1_kernel_128(int nt, int copy, bool wide);
E2m1Launch attn_e2m1_kernel_256(int nt, int copy, bool wide);
AttnE2m1JoinKernel attn_e2m1_join_kernel_for();

// The visible part of a 4-bit cache, K as bf16 and V as fp16 -- exact, the product of a code and a scale has six significant bits, and is 2^-10 at least and
// 2688 at most -- in pages of
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
