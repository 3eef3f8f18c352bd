// Rotary positions, and the fused norm + rotation + write into a paged cache (include/qknorm_attn.h).
//
// One kernel template does both: a group of threads owns a token, reads its Q, K (and V) rows once into
// registers, forms the statistic if there is a norm, rotates, and writes every element once.
//
// Mathematics.  The norm is Eq. 1 (layerwise) or its headwise form, as in the other kernels.  Pair
// (a, b) of a head then turns by angle = position * inv_freq[i]: (a c - b s, b c + a s).  The angle is
// formed in fp64 as a number of turns and reduced to [-1/2, 1/2] there -- position 10^6 times frequency 1
// is 1.6e5 turns, of which fp32 keeps only 1/64 -- then cos and sin are taken in fp32.  The rot_dim/2 angles are the same
// for every head, so a token's cos and sin are made once, in shared memory, not once per head.
//
// What bounds it: HBM traffic (each element read once, written once).  The unit of work is 16 elements of one
// head, the two 8-element chunks whose elements pair up: chunks j and j + rot_dim/16 of the head in the
// half layout, neighbours in the interleaved one and in the part that does not rotate.  So a pair never
// crosses a thread, and in-place calls are safe: a unit is read and written by one thread.  A head takes the power of two
// >= head_dim/16 lanes, which keeps the headwise sum a shuffle tree inside a lane group.
// The layerwise sum is a shuffle tree plus one slot per warp; the barrier it needs is the one that
// publishes cos and sin.
#pragma once
#include "qknorm_device.cuh"
#include "qknorm_ring.cuh"  // ptx helpers

namespace qknorm {

struct RopeSide {
  const void* x;          // [T, heads*head_dim]
  void* y;                // the same, or nullptr where the result goes to the cache
  const uint16_t* gamma;  // [heads*head_dim] bf16; nullptr without a norm
  long long ldx, ldy;     // elements between rows
  int heads;              // 0 = absent
  float inv_d;            // 1 / (heads*head_dim)
};

struct CacheSide {
  void* base;
  long long page, token, head;  // strides, elements (4-bit cache: bytes)
  float inv_scale;
};

// The 4-bit cache as the template's CIO: its stores work on blocks of 16, below.
struct IoE2m1 {
  static constexpr int kBytes = 0;
};

struct RopeParams {
  RopeSide q, k, v;  // v only with a cache
  CacheSide ck, cv;
  const long long* slots;
  long long num_slots;  // num_pages * page_size
  int page_size, page_shift;  // page_shift: log2(page_size), or -1
  const long long* positions;  // [T], or with several axes [axes][T], ld_pos apart
  const double* inv_freq;
  float mscale;
  int rot_dim, interleaved;
  double turns_sign;  // +-1 / (2 pi)
  long long T;
  int head_dim;
  int log_lph;   // log2 of the lanes per head
  int slots_per_token;  // (q.heads + k.heads + v.heads) << log_lph
  int tokens_per_cta, threads_per_token;
  float eps, inv_hd;
  const unsigned char* axis;   // which axis turns a pair; nullptr: the first
  long long ld_pos;
  int axes;
  CacheSide cks, cvs;  // the block scales of a 4-bit cache
};

enum { kNormNone = 0, kNormLayer = 1, kNormHead = 2 };
constexpr int kRopeMaxPairs = 256;  // QKNORM_MAX_HEAD_DIM / 2

// The position at which pair i of token t stands; `first` is its position along the first axis.
__device__ __forceinline__ long long rope_pos(const RopeParams& R, long long t, int i, long long first) {
  if (R.axis == nullptr) return first;
  const int a = R.axis[i];
  return a < R.axes ? R.positions[a * R.ld_pos + t] : 0;
}

// cos and sin of pair i of the token at `pos`
__device__ __forceinline__ float2 rope_cs(const RopeParams& R, long long pos, int i) {
  double turns = (double)pos * R.inv_freq[i] * R.turns_sign;
  turns -= rint(turns);
  float s, c;
  sincospif((float)(turns + turns), &s, &c);
  return make_float2(c * R.mscale, s * R.mscale);
}

// 8 elements as stored, and as four pairs in fp32 (pairs, because sm_100 multiplies and adds them two at a time)
template <class IO>
struct Chunk8;
template <>
struct Chunk8<IoBf16> {
  uint4 w;
  __device__ __forceinline__ void load(const void* base, int i) {
    w = ld_stream(reinterpret_cast<const uint4*>(reinterpret_cast<const uint16_t*>(base) + i));
  }
  __device__ __forceinline__ void store(void* base, long long i) const {
    st_stream(reinterpret_cast<uint4*>(reinterpret_cast<uint16_t*>(base) + i), w);
  }
  __device__ __forceinline__ void unpack(float2* f) const {
    f[0] = bf_unpack2(w.x);
    f[1] = bf_unpack2(w.y);
    f[2] = bf_unpack2(w.z);
    f[3] = bf_unpack2(w.w);
  }
  __device__ __forceinline__ void pack(const float2* f) {
    w = make_uint4(bf_pack(f[0].x, f[0].y), bf_pack(f[1].x, f[1].y), bf_pack(f[2].x, f[2].y), bf_pack(f[3].x, f[3].y));
  }
  // (x * gamma) * r; the product is exact
  __device__ __forceinline__ void scaled(const uint4& g, float2 r, float2* f) const {
    f[0] = __fmul2_rn(mul_bf16x2(w.x, g.x), r);
    f[1] = __fmul2_rn(mul_bf16x2(w.y, g.y), r);
    f[2] = __fmul2_rn(mul_bf16x2(w.z, g.z), r);
    f[3] = __fmul2_rn(mul_bf16x2(w.w, g.w), r);
  }
  __device__ __forceinline__ void sumsq(float& a, float& b) const {
    IoBf16::sumsq_word(w.x, a, b);
    IoBf16::sumsq_word(w.y, a, b);
    IoBf16::sumsq_word(w.z, a, b);
    IoBf16::sumsq_word(w.w, a, b);
  }
};
template <>
struct Chunk8<IoE4m3> {
  uint2 w;
  __device__ __forceinline__ void load(const void* base, int i) {
    w = __ldcs(reinterpret_cast<const uint2*>(reinterpret_cast<const uint8_t*>(base) + i));
  }
  __device__ __forceinline__ void store(void* base, long long i) const {
    __stcs(reinterpret_cast<uint2*>(reinterpret_cast<uint8_t*>(base) + i), w);
  }
  __device__ __forceinline__ void unpack(float2* f) const {
    const uint32_t u[2] = {w.x, w.y};
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      uint32_t f01, f23;
      e4m3x4_to_f16x2(u[e], f01, f23);
      f[2 * e] = __half22float2(*reinterpret_cast<const __half2*>(&f01));
      f[2 * e + 1] = __half22float2(*reinterpret_cast<const __half2*>(&f23));
    }
  }
  __device__ __forceinline__ void pack(const float2* f) {
    w = make_uint2(e4m3_pack2(f[0].x, f[0].y) | (e4m3_pack2(f[1].x, f[1].y) << 16),
                   e4m3_pack2(f[2].x, f[2].y) | (e4m3_pack2(f[3].x, f[3].y) << 16));
  }
};

// What goes into a 4-bit cache (include/qknorm_attn.h: qknorm_fwd_append_e2m1).  16384 tokens of 5120 + 1024 + 1024 take 88 us, where 64 would move the
// bytes and a bf16 cache takes 81; the issue slots are 70 % full.

// The largest of three, or NaN if any is.
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float max_nan(float a, float b, float c) {
  float r;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ __forceinline__ float absmax8(const float2 (&v)[4]) {
  float m = max_nan(fabsf(v[0].x), fabsf(v[0].y));
#pragma unroll
  for (int e = 1; e < 4; ++e) m = max_nan(m, fabsf(v[e].x), fabsf(v[e].y));
  return m;
}
// x / d correctly rounded, for a d of at most four significant bits: its reciprocal is r, rounded down, and what is left.  The sum of
// the two products is off by 2^-45 of itself before its one rounding, and these quotients stay 2^-29 away from the middle between two
// fp32 numbers.  Ties between two codes are common (bf16 values over such a scale), and an ulp would decide them wrongly.
struct Reciprocal {
  float r, rest;
};
__device__ __forceinline__ float2 quotient(float2 x, Reciprocal d) {
  return __ffma2_rn(x, make_float2(d.r, d.r), __fmul2_rn(x, make_float2(d.rest, d.rest)));
}
// The E4M3 scale of a block whose largest magnitude is amax, as its byte; returns the scale's reciprocal, 0 for a scale of 0 or NaN.
// For the scale 448, which infinities have, rest > 0: they stay infinite.
__device__ __forceinline__ Reciprocal e2m1_scale(float amax, uint32_t& byte) {
  float most;
  asm("min.NaN.f32 %0, %1, 0f7E967699;" : "=f"(most) : "f"(amax));  // 1e38
  byte = e4m3_pack2(quotient(make_float2(most, most), {0x1.555554p-3f, 0x1.555556p-27f}).x, 0.f) & 0xffu;
  uint32_t f01, f23;
  e4m3x4_to_f16x2(byte, f01, f23);
  const float f = __half2float(__ushort_as_half((unsigned short)(f01 & 0xffffu)));
  // from an estimate by one of Newton's steps, rounded down; the remainder f*r - 1 is exact
  Reciprocal d;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(d.r) : "f"(f));
  d.r = __fmaf_rz(d.r, fmaf(-f, d.r, 1.0f), d.r);
  d.rest = d.r * fmaf(-f, d.r, 1.0f);
  if (!(f > 0.f)) d.r = d.rest = 0.f;
  return d;
}
// Codes of eight elements of a block with that scale.
__device__ __forceinline__ uint32_t e2m1_codes8(const float2 (&v)[4], Reciprocal d) {
  float2 y[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) y[e] = quotient(v[e], d);
  return e2m1_pack8(y);
}

// Where token slot `slot` (in range) starts in a cache side.
__device__ __forceinline__ long long cache_at(const CacheSide& c, long long slot, int page_size, int page_shift) {
  long long page;
  if (page_shift >= 0) page = slot >> page_shift;
  else if (slot <= 0xffffffffll) page = (unsigned)slot / (unsigned)page_size;
  else page = slot / page_size;
  return page * c.page + (slot - page * page_size) * c.token;
}

// IO: storage of q, k, v and out_q.  CIO: storage of the cache.  INTER: interleaved pairs.  UPT: 16-element units per thread.
// MAXT: the largest CTA; CTAs of up to 256 threads get 80 registers a thread, which four units need -- 64 with an FP8 cache,
// whose conversions want more warps instead (8191 tokens of 8192 + 1024 + 1024: 58 us against 64; bf16 cache: 84 against 83).
// So does a 4-bit cache behind a layerwise norm (16384 tokens of 5120 + 1024 + 1024: 87 us against 91), not behind the others, which would spill
// more (per head 97 against 93).
template <class IO, class CIO, int NORM, bool CACHE, bool INTER, int UPT, int MAXT>
__global__ void __launch_bounds__(MAXT, MAXT != 256 ? 1 : CACHE && (CIO::kBytes == 1 || (CIO::kBytes == 0 && NORM == kNormLayer)) ? 4 : 3) rope_kernel(const __grid_constant__ RopeParams R) {
  extern __shared__ float4 cs_all[];  // [tokens_per_cta][4][rot_dim/16]: (c, c, s, s) of pairs 8j+2e, 8j+2e+1 at [e][j]
  __shared__ float red[32][2];        // per warp: sum of squares of Q, of K
  const int slot_of_token = threadIdx.x / R.threads_per_token;
  const int tid = threadIdx.x - slot_of_token * R.threads_per_token;
  const long long t = (long long)blockIdx.x * R.tokens_per_cta + slot_of_token;
  const bool live = t < R.T;
  const int r16 = R.rot_dim >> 4;
  float4* cs = cs_all + slot_of_token * 4 * r16;
  asm volatile("griddepcontrol.wait;" ::: "memory");

  const char* row_q = reinterpret_cast<const char*>(R.q.x) + t * R.q.ldx * IO::kBytes;
  const char* row_k = reinterpret_cast<const char*>(R.k.x) + t * R.k.ldx * IO::kBytes;
  const char* row_v = reinterpret_cast<const char*>(R.v.x) + t * R.v.ldx * IO::kBytes;
  Chunk8<IO> u[UPT][2];
  int head[UPT];
  int off[UPT];   // of the unit's first chunk in its row
  int side[UPT];  // 0 q, 1 k, 2 v, -1 none
  const int j = tid & ((1 << R.log_lph) - 1);  // which 16 elements of its head; threads_per_token is a multiple of 32, so the
                                               // same in every unit of the thread
  const bool turns = j < r16;
  const int c0 = turns && !INTER ? 8 * j : 16 * j;
  const int step = turns && !INTER ? 8 * r16 : 8;  // from the first chunk to the second
#pragma unroll
  for (int i = 0; i < UPT; ++i) {
    const int s = tid + i * R.threads_per_token;
    int h = s >> R.log_lph;
    side[i] = -1;
    if (live && s < R.slots_per_token && j * 16 < R.head_dim) {
      side[i] = 0;
      if (h >= R.q.heads) {
        h -= R.q.heads;
        side[i] = 1;
        if (CACHE && h >= R.k.heads) {
          h -= R.k.heads;
          side[i] = 2;
        }
      }
    }
    head[i] = h;
    off[i] = h * R.head_dim + c0;
    if (side[i] >= 0) {
      const char* row = side[i] == 0 ? row_q : (!CACHE || side[i] == 1) ? row_k : row_v;
      u[i][0].load(row, off[i]);
      u[i][1].load(row, off[i] + step);
    }
  }
  long long cslot = -1;
  if (CACHE && live) {
    cslot = R.slots[t];
    if (cslot >= R.num_slots) cslot = -1;
  }
  constexpr bool kBlocks = CACHE && CIO::kBytes == 0;
  // Where the token's slot starts in the pools.  Only the warps that write there work it out, after the norm -- but for norms per head,
  // which everything has to be ready for (16384 tokens of 5120 + 1024 + 1024, bf16 cache: 81.5 us instead of 83.7; per head 86.6, as
  // here 83.7.  4-bit cache: 88.5 instead of 94.3, per head 93.8 instead of 97.2, without a norm 86.5 instead of 92.3).
  constexpr bool kEarly = CACHE && !kBlocks && NORM != kNormLayer;
  long long slot_k = 0, slot_v = 0;
  if (kEarly && cslot >= 0) {
    slot_k = cache_at(R.ck, cslot, R.page_size, R.page_shift);
    slot_v = cache_at(R.cv, cslot, R.page_size, R.page_shift);
  }
  if (live && r16 > 0) {
    auto put = [&](int p, float2 f) {
      float* at = reinterpret_cast<float*>(cs + ((p & 7) >> 1) * r16 + (p >> 3)) + (p & 1);
      at[0] = f.x;
      at[2] = f.y;
    };
    const long long pos = R.positions[t];
    if (R.axis == nullptr) {
      for (int p = tid; p < 8 * r16; p += R.threads_per_token) put(p, rope_cs(R, pos, p));
    } else {
      for (int p = tid; p < 8 * r16; p += R.threads_per_token) put(p, rope_cs(R, rope_pos(R, t, p, pos), p));
    }
  }
  float rq = 1.f, rk = 1.f;
  if constexpr (NORM == kNormLayer) {
    float sq = 0.f, sk = 0.f;
#pragma unroll
    for (int i = 0; i < UPT; ++i) {
      if (side[i] == 0 || side[i] == 1) {
        float a = 0.f, b = 0.f;
        u[i][0].sumsq(a, b);
        u[i][1].sumsq(a, b);
        if (side[i] == 0) sq += a + b;
        else sk += a + b;
      }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      sq += __shfl_xor_sync(0xffffffffu, sq, o);
      sk += __shfl_xor_sync(0xffffffffu, sk, o);
    }
    if ((threadIdx.x & 31) == 0) {
      red[threadIdx.x >> 5][0] = sq;
      red[threadIdx.x >> 5][1] = sk;
    }
  }
  __syncthreads();
  if constexpr (NORM == kNormLayer) {
    const int wpt = R.threads_per_token >> 5, w0 = slot_of_token * wpt;
    float sq = 0.f, sk = 0.f;
    for (int w = 0; w < wpt; ++w) {  // fixed order
      sq += red[w0 + w][0];
      sk += red[w0 + w][1];
    }
    rq = rstd_of(sq, R.q.inv_d, R.eps);
    rk = rstd_of(sk, R.k.inv_d, R.eps);
  }
#pragma unroll
  for (int i = 0; i < UPT; ++i) {
    float r = side[i] == 0 ? rq : rk;
    if constexpr (NORM == kNormHead) {
      float a = 0.f, b = 0.f;
      if (side[i] >= 0) {
        u[i][0].sumsq(a, b);
        u[i][1].sumsq(a, b);
      }
      a += b;
      for (int o = 1 << R.log_lph >> 1; o > 0; o >>= 1) a += __shfl_xor_sync(0xffffffffu, a, o);
      r = rstd_of(a, R.inv_hd, R.eps);
    }
    if (side[i] < 0) continue;
    const bool to_cache = CACHE && side[i] != 0;
    const bool as_is = (side[i] == 2 || (NORM == kNormNone && !turns)) && (!to_cache || CIO::kBytes == IO::kBytes);
    float2 a[4], b[4];
    if (!as_is) {
      bool scale = false;
      if constexpr (NORM != kNormNone) {
        if (side[i] != 2) {
          const uint16_t* g = (side[i] == 0 ? R.q.gamma : R.k.gamma) + off[i];
          const uint4 g0 = __ldg(reinterpret_cast<const uint4*>(g)), g1 = __ldg(reinterpret_cast<const uint4*>(g + step));
          u[i][0].scaled(g0, make_float2(r, r), a);
          u[i][1].scaled(g1, make_float2(r, r), b);
          scale = true;
        }
      }
      if (!scale) {
        u[i][0].unpack(a);
        u[i][1].unpack(b);
      }
      if (turns && side[i] != 2) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float4 f = cs[e * r16 + j];  // pairs 8j+2e, 8j+2e+1
          if constexpr (INTER) {             // pairs 8j..8j+3 lie in a, 8j+4..8j+7 in b
            float2& p = e < 2 ? a[2 * e] : b[2 * e - 4];
            float2& q = e < 2 ? a[2 * e + 1] : b[2 * e - 3];
            p = __ffma2_rn(make_float2(p.y, p.x), make_float2(-f.z, f.z), __fmul2_rn(p, make_float2(f.x, f.x)));
            q = __ffma2_rn(make_float2(q.y, q.x), make_float2(-f.w, f.w), __fmul2_rn(q, make_float2(f.y, f.y)));
          } else {
            const float2 c = make_float2(f.x, f.y), sn = make_float2(f.z, f.w), x = a[e];
            a[e] = __ffma2_rn(b[e], make_float2(-sn.x, -sn.y), __fmul2_rn(x, c));
            b[e] = __ffma2_rn(x, sn, __fmul2_rn(b[e], c));
          }
        }
      }
    }
    if (to_cache) {
      if (cslot < 0) continue;
      const CacheSide& C = side[i] == 1 ? R.ck : R.cv;
      if constexpr (kBlocks) {
        // A chunk of the half layout is half a block; the other half is the neighbouring lane's (rot_dim is a multiple of 32
        // then, so it is a lane of the same head, and of the same part of it).
        const CacheSide& S = side[i] == 1 ? R.cks : R.cvs;
        const bool split = turns && !INTER;
        const float2 k2 = make_float2(C.inv_scale, C.inv_scale);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          a[e] = __fmul2_rn(a[e], k2);
          b[e] = __fmul2_rn(b[e], k2);
        }
        float ma = absmax8(a), mb = absmax8(b);
        if (split) {
          const unsigned pair = 3u << (threadIdx.x & 30);
          ma = max_nan(ma, __shfl_xor_sync(pair, ma, 1));
          mb = max_nan(mb, __shfl_xor_sync(pair, mb, 1));
        } else {
          ma = mb = max_nan(ma, mb);
        }
        uint32_t sa, sb = 0;
        const Reciprocal da = e2m1_scale(ma, sa);
        char* codes = reinterpret_cast<char*>(C.base) + cache_at(C, cslot, R.page_size, R.page_shift) + head[i] * C.head + (c0 >> 1);
        if (split) {
          const Reciprocal db = e2m1_scale(mb, sb);
          __stcs(reinterpret_cast<uint32_t*>(codes), e2m1_codes8(a, da));
          __stcs(reinterpret_cast<uint32_t*>(codes + (step >> 1)), e2m1_codes8(b, db));
        } else {
          __stcs(reinterpret_cast<uint2*>(codes), make_uint2(e2m1_codes8(a, da), e2m1_codes8(b, da)));
        }
        unsigned char* sc = reinterpret_cast<unsigned char*>(S.base) + cache_at(S, cslot, R.page_size, R.page_shift) + head[i] * S.head;
        if (!split || !(j & 1)) sc[c0 >> 4] = (unsigned char)sa;
        else sc[(c0 + step) >> 4] = (unsigned char)sb;
        continue;
      } else {
      const long long slot_at = !kEarly ? cache_at(C, cslot, R.page_size, R.page_shift) : side[i] == 1 ? slot_k : slot_v;
      const long long at = slot_at + head[i] * C.head + c0;
      Chunk8<CIO> o0, o1;
      if constexpr (CIO::kBytes == 1 || IO::kBytes == 1) {
        const float2 k = make_float2(C.inv_scale, C.inv_scale);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          a[e] = __fmul2_rn(a[e], k);
          b[e] = __fmul2_rn(b[e], k);
        }
        o0.pack(a);
        o1.pack(b);
      } else if (as_is) {
        o0 = u[i][0];
        o1 = u[i][1];
      } else {
        o0.pack(a);
        o1.pack(b);
      }
      o0.store(C.base, at);
      o1.store(C.base, at + step);
      }
    } else {
      const RopeSide& A = side[i] == 0 ? R.q : R.k;
      char* row = reinterpret_cast<char*>(A.y) + t * A.ldy * IO::kBytes;
      if (!as_is) {
        u[i][0].pack(a);
        u[i][1].pack(b);
      }
      u[i][0].store(row, off[i]);
      u[i][1].store(row, off[i] + step);
    }
  }
}

// Any head_dim, any alignment, any width: a CTA per token, element-wise.  A lane owns whole pairs, so in-place
// calls are safe here too.
constexpr int kRopeGeneralThreads = 256;

template <class IO, class CIO, bool CACHE>
__global__ void __launch_bounds__(kRopeGeneralThreads) rope_general_kernel(const __grid_constant__ RopeParams R, int norm) {
  __shared__ float2 cs[kRopeMaxPairs];
  __shared__ float red[kRopeGeneralThreads / 32];
  constexpr bool kBlocks = CACHE && CIO::kBytes == 0;
  __shared__ float whole[kBlocks ? kRopeGeneralThreads / 32 : 1][kBlocks ? kRopeMaxPairs : 1];  // a warp's head, before it is cut into blocks
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int pairs = R.rot_dim >> 1, singles = R.head_dim - R.rot_dim;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  for (long long t = blockIdx.x; t < R.T; t += gridDim.x) {
    __syncthreads();  // the previous token's cos and sin are no longer needed
    if (pairs > 0) {
      const long long pos = R.positions[t];
      for (int p = threadIdx.x; p < pairs; p += kRopeGeneralThreads) cs[p] = rope_cs(R, rope_pos(R, t, p, pos), p);
    }
    long long cslot = -1;
    if (CACHE) {
      cslot = R.slots[t];
      if (cslot >= R.num_slots) cslot = -1;
    }
    for (int side = 0; side < (CACHE ? 3 : 2); ++side) {
      const RopeSide& A = side == 0 ? R.q : side == 1 ? R.k : R.v;
      if (A.heads == 0) continue;
      const bool to_cache = CACHE && side != 0;
      const CacheSide& C = side == 2 ? R.cv : R.ck;
      const long long xrow = t * A.ldx;
      float r = 1.f;
      if (norm == kNormLayer && side != 2) {
        float acc = 0.f;
        const int d = A.heads * R.head_dim;
        for (int i = threadIdx.x; i < d; i += kRopeGeneralThreads) {
          const float v = IO::load(A.x, xrow + i);
          acc = fmaf(v, v, acc);
        }
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) acc += __shfl_xor_sync(0xffffffffu, acc, off);
        __syncthreads();  // the slots of the side before
        if (lane == 0) red[warp] = acc;
        __syncthreads();
        float sum = 0.f;
        for (int w = 0; w < kRopeGeneralThreads / 32; ++w) sum += red[w];
        r = rstd_of(sum, A.inv_d, R.eps);
      } else {
        __syncthreads();
      }
      for (int h = warp; h < A.heads; h += kRopeGeneralThreads / 32) {
        const long long x0 = xrow + (long long)h * R.head_dim;
        float rr = r;
        if (norm == kNormHead && side != 2) {
          float acc = 0.f;
          for (int i = lane; i < R.head_dim; i += 32) {
            const float v = IO::load(A.x, x0 + i);
            acc = fmaf(v, v, acc);
          }
#pragma unroll
          for (int off = 16; off > 0; off >>= 1) acc += __shfl_xor_sync(0xffffffffu, acc, off);
          rr = rstd_of(acc, R.inv_hd, R.eps);
        }
        auto value = [&](int i) {
          float v = IO::load(A.x, x0 + i);
          if (norm != kNormNone && side != 2) v *= IoBf16::load(A.gamma, (long long)h * R.head_dim + i) * rr;
          return v;
        };
        if (to_cache && cslot < 0) continue;
        const long long y0 = to_cache ? cache_at(C, cslot, R.page_size, R.page_shift) + h * C.head : t * A.ldy + (long long)h * R.head_dim;
        auto put = [&](int i, float v) {
          if constexpr (kBlocks) {
            if (to_cache) {
              whole[warp][i] = v * C.inv_scale;
              return;
            }
          } else if (to_cache) {
            CIO::store(C.base, y0 + i, CIO::kBytes == 1 ? v * C.inv_scale : v);
            return;
          }
          IO::store(A.y, y0 + i, v);
        };
        for (int p = lane; p < pairs; p += 32) {
          const int ia = R.interleaved ? 2 * p : p, ib = R.interleaved ? 2 * p + 1 : p + pairs;
          const float a = value(ia), b = value(ib);
          const float2 f = side != 2 ? cs[p] : make_float2(1.f, 0.f);
          put(ia, side != 2 ? a * f.x - b * f.y : a);
          put(ib, side != 2 ? b * f.x + a * f.y : b);
        }
        for (int i = lane; i < singles; i += 32) put(R.rot_dim + i, value(R.rot_dim + i));
        if constexpr (kBlocks) {
          if (to_cache) {
            const CacheSide& S = side == 2 ? R.cvs : R.cks;
            unsigned char* sc = reinterpret_cast<unsigned char*>(S.base) + cache_at(S, cslot, R.page_size, R.page_shift) + h * S.head;
            __syncwarp();
            for (int blk = lane; blk < R.head_dim / 16; blk += 32) {
              float2 lo[4], hi[4];
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                lo[e] = make_float2(whole[warp][16 * blk + 2 * e], whole[warp][16 * blk + 2 * e + 1]);
                hi[e] = make_float2(whole[warp][16 * blk + 8 + 2 * e], whole[warp][16 * blk + 9 + 2 * e]);
              }
              uint32_t byte;
              const Reciprocal d = e2m1_scale(max_nan(absmax8(lo), absmax8(hi)), byte);
              *reinterpret_cast<uint2*>(reinterpret_cast<char*>(C.base) + y0 + 8 * blk) =
                  make_uint2(e2m1_codes8(lo, d), e2m1_codes8(hi, d));
              sc[blk] = (unsigned char)byte;
            }
            __syncwarp();
          }
        }
      }
    }
  }
}

typedef void (*RopeKernel)(const RopeParams);
typedef void (*RopeGeneralKernel)(const RopeParams, int);
// in qknorm_rope_inst.cu; upt 1 or 4, threads: of the CTA; cache_bytes 0 = no cache, kCacheE2m1 = the 4-bit one
constexpr int kCacheE2m1 = 4;
RopeKernel rope_kernel_for(int elem_bytes, int cache_bytes, int norm, bool interleaved, int upt, int threads);
RopeGeneralKernel rope_general_kernel_for(int elem_bytes, int cache_bytes);

}  // namespace qknorm
