// Attention of new tokens over a paged cache (include/qknorm_attn.h): what every kernel of it shares --
// parameters, which keys a row sees, the row-at-a-time routine -- and the general kernel and the join of split results.
//
// Mathematics.  For one row, over the keys it sees, with c = scale * log2(e) (times the FP8 cache's k_scale):
//   s_j = q . k_j,  m = max s_j,  l = sum 2^(c (s_j - m)),  o = sum 2^(c (s_j - m)) v_j / l
// in one pass with a running m (l and o are multiplied by 2^(c (m_old - m_new)) when it grows).  Two parts
// (o1, z1), (o2, z2) of one row over different keys, z = c m + log2 l, join to (o1 2^(z1-z) + o2 2^(z2-z), z).
#pragma once
#include <cuda.h>  // CUtensorMap

#include "qknorm_device.cuh"
#include "qknorm_ring.cuh"  // ptx helpers

namespace qknorm {

constexpr int kAttnTile = 128;       // keys per tile, rows per query tile
constexpr int kAttnMaxEpl = 16;      // head_dim elements per lane of the row routine: QKNORM_MAX_HEAD_DIM / 32
constexpr float kNegInf = -__builtin_huge_valf();
// c is never 0, which a product with the -inf of a masked score would make NaN; this is the least fp32 value
constexpr float kAttnLeastC = 1.401298464e-45f;

struct AttnSide {
  const void* base;
  long long page, token, head;  // strides, elements
};

struct AttnParams {
  const uint16_t* q;  // bf16
  uint16_t* out;      // bf16
  long long ld_q, ld_out;
  AttnSide k, v;
  long long num_pages;
  int page_size, page_shift;  // page_shift: log2(page_size), or -1
  const int* table;
  long long ld_table;
  const int* kv_lens;
  const int* q_starts;
  int seqs;
  long long T;
  int max_q;
  long long max_keys;  // min(max_kv, table_cols * page_size)
  int heads_q, heads_kv, group, head_dim;
  float c;             // scale * k_scale * log2(e)
  float v_scale;
  int causal, window;
  float* lse;
  // where the CTAs of the tensor-core kernel start, and what they leave unfinished (see AttnItem)
  int* starts;    // [grid][8]
  float* part_o;  // [grid][2][part_rows][head_dim], normalised
  float* part_z;  // [grid][2][part_rows], log2
  int grid, part_rows;
  int own;  // what an item costs beside its tiles, in tiles
  int tok_per_tile;     // tokens of a query tile: 128 / group
  int tiles_per_item;   // query tiles an item holds: 1 or 2
  int q_items;          // items per (sequence, key head)
  int box_rows, box_shift;  // tokens of one TMA copy: the largest power of two that divides page_size and a tile; 0: no TMA
  int box_kind;      // what a TMA copy of K and V takes, below
  int q_box_tokens;  // tokens of one TMA copy of q
  unsigned wait_ns;  // how long the tensor-core kernel waits while nothing in the CTA moves; below 2^31
  int* error;
};

// What one of the tensor-core kernel's copies of K or V brings: tokens of a page times
//   kBoxHalf       64 columns of a head (FP8: all its columns), from [page][head][token][d];
//   kBoxHeadInRow  a whole head of 128, from [page][8 tokens][head and half][token][64 columns]: heads side by side in a token;
//   kBoxHeadInPage a whole head of 128, from [page and head][8 tokens][half][token][64 columns]: a page's heads one after the other.
// Whole heads, because the copy engine's time goes by the box: 64 x 8192 keys took 420 us by halves, 331 by heads.
constexpr int kBoxHalf = 0, kBoxHeadInRow = 1, kBoxHeadInPage = 2;
struct AttnMaps {
  CUtensorMap q, k, v;  // q as [token][head][d]
};

// What one sequence's place in the batch says; everything clamped to the call's buffers.
struct AttnSeq {
  int row0;       // first row of q
  int n;          // new tokens served (<= max_q)
  int keys;       // keys that may be looked at
  long long pos0; // position of the first new token (negative: it sees nothing)
};

__device__ __forceinline__ AttnSeq attn_seq(const AttnParams& P, int b) {
  AttnSeq s;
  const long long T = P.T;
  long long r0 = P.q_starts[b], r1 = P.q_starts[b + 1];
  const long long len = P.kv_lens[b];
  r0 = r0 < 0 ? 0 : r0 > T ? T : r0;
  r1 = r1 < r0 ? r0 : r1 > T ? T : r1;
  s.row0 = (int)r0;
  s.n = (int)(r1 - r0 < P.max_q ? r1 - r0 : P.max_q);
  s.keys = (int)(len < 0 ? 0 : len < P.max_keys ? len : P.max_keys);
  s.pos0 = len - (r1 - r0);
  return s;
}

// Keys [lo, hi) that new token i sees; hi <= lo: none.  Both grow with i.
__device__ __forceinline__ int attn_hi(const AttnParams& P, const AttnSeq& s, int i) {
  if (!P.causal) return s.keys;
  const long long e = s.pos0 + i + 1;
  return (int)(e < 0 ? 0 : e < s.keys ? e : s.keys);
}
__device__ __forceinline__ int attn_lo(const AttnParams& P, const AttnSeq& s, int i) {
  if (P.window == 0) return 0;
  const long long e = s.pos0 + i + 1 - P.window;
  return (int)(e < 0 ? 0 : e < s.keys ? e : s.keys);
}

// Page and token inside the page of a key; page < 0: an entry that names no page.
__device__ __forceinline__ long long attn_page(const AttnParams& P, int b, int key, int& within) {
  int idx;
  if (P.page_shift >= 0) {
    idx = key >> P.page_shift;
    within = key & (P.page_size - 1);
  } else {
    idx = (int)((unsigned)key / (unsigned)P.page_size);
    within = key - idx * P.page_size;
  }
  const int e = __ldg(P.table + (long long)b * P.ld_table + idx);
  return (e < 0 || e >= P.num_pages) ? -1 : e;
}

// The waits of the tensor-core kernel give up when the time that stands in a word of shared memory has passed (low 32 bits of
// the GPU's clock in ns); whoever gets work done now and then moves it on.
__device__ __forceinline__ unsigned attn_time() {
  unsigned t;
  asm volatile("mov.u32 %0, %%globaltimer_lo;" : "=r"(t));
  return t;
}
__device__ __forceinline__ void attn_moving(const AttnParams& P, uint32_t deadline) {
  asm volatile("st.volatile.shared::cta.u32 [%0], %1;" ::"r"(deadline), "r"(attn_time() + P.wait_ns) : "memory");
}

// One warp, one row and head, keys [lo, hi): o (normalised; lane holds elements lane + 32 e) and z = c m + log2 l.
// Reads nothing of a key outside the range, so what other keys hold cannot matter.
// EPL: elements per lane, at least head_dim / 32.  deadline: the word of attn_moving, or 0.
template <class KIO, class VIO, int EPL>
__device__ __forceinline__ void attn_row(const AttnParams& P, int b, long long row, int head, int lo, int hi, float (&o)[EPL],
                                         float& z_out, uint32_t deadline = 0) {
  const int lane = threadIdx.x & 31, D = P.head_dim;
  const int kvh = head / P.group;
  float q[EPL];
#pragma unroll
  for (int e = 0; e < EPL; ++e) {
    const int d = lane + 32 * e;
    q[e] = d < D ? IoBf16::load(P.q, row * P.ld_q + (long long)head * D + d) : 0.f;
    o[e] = 0.f;
  }
  float m = kNegInf, l = 0.f;
  for (int key = lo; key < hi; ++key) {
    if (deadline != 0 && (key & 63) == 0 && lane == 0) attn_moving(P, deadline);
    int within;
    const long long page = attn_page(P, b, key, within);
    const long long ka = page * P.k.page + within * P.k.token + kvh * P.k.head;
    const long long va = page * P.v.page + within * P.v.token + kvh * P.v.head;
    float s = 0.f;
    if (page >= 0) {
#pragma unroll
      for (int e = 0; e < EPL; ++e) {
        const int d = lane + 32 * e;
        if (d < D) s = fmaf(q[e], KIO::load(P.k.base, ka + d), s);
      }
    }
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
    if (s == kNegInf) continue;
    const float mn = fmaxf(m, s);  // a NaN score leaves m as it is and makes p, and the row, NaN
    const float f = m == kNegInf ? 0.f : exp2f((m - mn) * P.c);
    const float p = mn == kNegInf ? s : exp2f((s - mn) * P.c);
    l = fmaf(l, f, p);
#pragma unroll
    for (int e = 0; e < EPL; ++e) {
      const int d = lane + 32 * e;
      if (d < D) o[e] = fmaf(o[e], f, p * (page >= 0 ? VIO::load(P.v.base, va + d) : 0.f));
    }
    m = mn;
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
  for (int e = 0; e < EPL; ++e) o[e] *= inv;
  z_out = l == 0.f ? kNegInf : m == kNegInf ? l : fmaf(m, P.c, log2f(l));
}

constexpr float kLn2 = 0.693147180559945309f;

// Any head_dim, group, alignment: a warp per (new token, query head).  For what the tensor-core kernel does not take; each key costs
// a warp a dependent round trip, where the other kernel takes 128 of them at once.
constexpr int kAttnGeneralThreads = 128;

template <class KIO, class VIO>
__global__ void __launch_bounds__(kAttnGeneralThreads) attn_general_kernel(const __grid_constant__ AttnParams P) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int lane = threadIdx.x & 31;
  const long long items = (long long)P.seqs * P.max_q * P.heads_q;
  const long long warps = (long long)gridDim.x * (kAttnGeneralThreads / 32);
  for (long long it = (long long)blockIdx.x * (kAttnGeneralThreads / 32) + (threadIdx.x >> 5); it < items; it += warps) {
    const int head = (int)(it % P.heads_q);
    const long long r = it / P.heads_q;
    const int i = (int)(r % P.max_q), b = (int)(r / P.max_q);
    const AttnSeq s = attn_seq(P, b);
    if (i >= s.n) continue;
    const long long row = s.row0 + (long long)i;
    float o[kAttnMaxEpl], z;
    attn_row<KIO, VIO, kAttnMaxEpl>(P, b, row, head, attn_lo(P, s, i), attn_hi(P, s, i), o, z);
#pragma unroll
    for (int e = 0; e < kAttnMaxEpl; ++e) {
      const int d = lane + 32 * e;
      if (d < P.head_dim) IoBf16::store(P.out, row * P.ld_out + (long long)head * P.head_dim + d, o[e] * P.v_scale);
    }
    if (P.lse != nullptr && lane == 0) P.lse[row * P.heads_q + head] = z * kLn2;
  }
}

// The tensor-core kernel's work.  A unit is the query tiles of one item of one sequence (tiles_per_item tiles from token
// qt * tok_per_tile * tiles_per_item on) and one key head; it weighs as many key tiles as its rows see, and `own` more for its
// first and last steps.  All units in a row -- sequences, their items, key heads fastest -- are cut into `grid` equal lengths, one for
// each CTA, wherever the cuts fall: CTAs get the same number of tiles whatever the lengths of the sequences.  A CTA's
// share of a unit is an item.  A unit that lies in one CTA is finished there; of one that is cut, each CTA leaves its part
// (normalised rows and their log-sum) in one of its two slots -- 0 if the unit began before the CTA's share, 1 if it goes on
// behind it -- and the join kernel puts them together.  A cut close to a unit's end or start goes there (attn_snap).
struct AttnItem {
  AttnSeq s;
  int b, kvh;
  int tok0;      // first new token
  int j0, j1;    // key tiles of this item; none: j0 == j1
  int ulo, uhi;  // keys that some row of the unit sees
  bool whole;    // all of its unit
  int slot;
};

// Key tiles [J0, J1) of the unit that starts at token tok0, and its keys [ulo, uhi).
__device__ __forceinline__ void attn_span(const AttnParams& P, const AttnSeq& s, int tok0, int& J0, int& J1, int& ulo, int& uhi) {
  int last = tok0 + P.tok_per_tile * P.tiles_per_item - 1;
  if (last >= s.n) last = s.n - 1;
  ulo = attn_lo(P, s, tok0);
  uhi = attn_hi(P, s, last);
  if (uhi <= ulo) {
    J0 = J1 = 0;
    return;
  }
  J0 = ulo / kAttnTile;
  J1 = (uhi + kAttnTile - 1) / kAttnTile;
}
// What a unit of the sequence's item qt weighs; 0: the sequence has no such rows.
__device__ __forceinline__ int attn_weight(const AttnParams& P, const AttnSeq& s, int qt) {
  const int tok0 = qt * P.tok_per_tile * P.tiles_per_item;
  if (tok0 >= s.n) return 0;
  int J0, J1, ulo, uhi;
  attn_span(P, s, tok0, J0, J1, ulo, uhi);
  return J1 - J0 + P.own;
}

// Where a CTA's share starts: unit (b, qt, kvh) of sequence s, `off` into it; and how long it is.
struct AttnStart {
  AttnSeq s;
  int b, qt, kvh, off;
  int left;
};

// A cut costs its unit a part more and the join; it is worth that where shares are long.  Short shares (few tiles on many SMs) only
// cut units that weigh more than 16: a cut in a shorter one goes to the nearer end.  Both sides, single tokens, 8 key heads of 8 query heads
// of 128, us in a captured graph, units whole | cut:
//   sequences            1            4            8           12           18           19           30           37
//    500 keys   11.6 | 16.5  12.1 | 17.4  12.3 | 18.3  12.8 | 20.0  14.8 | 18.3  21.4 | 25.2  22.3 | 30.7  22.7 | 27.0
//   1000 keys   16.6 | 15.7  17.2 | 16.8  18.5 | 20.7  19.4 | 24.7  21.1 | 24.9  31.7 | 30.0  33.1 | 38.5  34.2 | 38.5
//   1900 keys   25.1 | 17.4  27.2 | 18.7  29.2 | 26.3  29.1 | 31.7  31.6 | 35.0  50.2 | 40.9  52.6 | 54.1  59.4 | 59.2
// (1 key head: 1000 keys 16.5 | 15.5, 1900 keys 25.5 | 17.5 up to 24 sequences.)  So 16 is right, or within 2 us, for units up to 8 tiles and for batches that
// give most SMs one unit; for 9 to 16 tiles it loses up to 9 us to cuts where there are fewer than 64 units, and just above one unit an SM.
constexpr int kAttnWhole = 16;
__host__ __device__ __forceinline__ int attn_snap(long long share, int own, int weight) {
  return share < 32 && weight <= kAttnWhole ? (weight + 1) / 2 : own;
}

// Found by the whole CTA (blockDim threads, a multiple of 32 up to 1024): a scan over the weights of (sequence, item).
// scratch: 36 long longs of shared memory, free again when this returns; `out` is in shared memory too.
__device__ __forceinline__ void attn_find_start(const AttnParams& P, long long* scratch, AttnStart* out) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, warps = blockDim.x >> 5;
  const int n = P.seqs * P.q_items;  // the host has checked that it fits
  const int per = (n + blockDim.x - 1) / blockDim.x;
  const int n0 = per * tid < n ? per * tid : n, n1 = n0 + per < n ? n0 + per : n;
  long long sum = 0;
  AttnSeq s = {};
  int b0 = 0, qt0 = 0;
  if (n1 > n0) {
    b0 = P.q_items == 1 ? n0 : n0 / P.q_items;
    qt0 = n0 - b0 * P.q_items;
    s = attn_seq(P, b0);
    int b = b0, qt = qt0;
    for (int i = n0; i < n1; ++i) {
      sum += attn_weight(P, s, qt);
      if (++qt == P.q_items) {
        qt = 0;
        if (i + 1 < n1) s = attn_seq(P, ++b);
      }
    }
  }
  long long incl = sum;
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const long long v = __shfl_up_sync(0xffffffffu, incl, off);
    if (lane >= off) incl += v;
  }
  if (lane == 31) scratch[warp] = incl;
  if (tid == 0) scratch[33] = scratch[34] = -1;  // snapped end; snapped start
  __syncthreads();
  long long before = incl - sum, total = 0;
  for (int w = 0; w < warps; ++w) {
    if (w < warp) before += scratch[w];
    total += scratch[w];
  }
  before *= P.heads_kv;
  total *= P.heads_kv;
  sum *= P.heads_kv;
  long long share = total <= 0x7fffffff ? ((unsigned)total + gridDim.x - 1) / gridDim.x : (total + gridDim.x - 1) / gridDim.x;
  if (share < P.own + 2) share = P.own + 2;
  // No room for parts: every cut moves to a unit's start.  The host has seen to it that none has to -- for starts that ascend; others
  // can make more units than the rows allow for.
  const bool cuts = P.starts != nullptr;
#pragma unroll
  for (int which = 0; which < 2; ++which) {  // this CTA's cut, and the next one's
    const long long cut = (blockIdx.x + which) * share;
    if (cut >= total) {
      if (which == 1 && tid == 0) scratch[33] = total;
      continue;
    }
    if (cut < before || cut >= before + sum) continue;
    int b = b0, qt = qt0;
    if (per > 1) s = attn_seq(P, b);
    long long at = before;
    int w = attn_weight(P, s, qt);
    while (cut >= at + (long long)w * P.heads_kv) {
      at += (long long)w * P.heads_kv;
      if (++qt == P.q_items) {
        qt = 0;
        s = attn_seq(P, ++b);
      }
      w = attn_weight(P, s, qt);
    }
    int kvh = 0;
    for (; cut >= at + w; at += w) ++kvh;
    int off = (int)(cut - at);
    const int raw = off, snap = cuts ? attn_snap(share, P.own, w) : 0x3fffffff;
    off = off <= snap ? 0 : w - off <= snap ? w : off;
    scratch[33 + (which ^ 1)] = at + off;
    if (which == 0) {
      out->s = s;
      out->b = b;
      out->qt = qt;
      out->kvh = kvh;
      out->off = off;
      if (cuts) {
        int* rec = P.starts + blockIdx.x * 8;
        const bool inside = off > 0 && off < w;
        rec[0] = b;
        rec[1] = qt;
        rec[2] = kvh;
        // parts that this cut and those behind it make, if it is the unit's first
        rec[3] = inside && raw - share <= snap ? 2 + (int)((w - snap - 1 - raw) / share) : 0;
      }
    }
  }
  __syncthreads();
  if (tid == 0) {
    if (scratch[34] < 0) {
      out->left = 0;  // past the last unit
      if (cuts) P.starts[blockIdx.x * 8 + 3] = 0;
    } else {
      out->left = (int)(scratch[33] - scratch[34]);
    }
  }
  __syncthreads();
}

// The items of a share, in order.
struct AttnWalk {
  AttnSeq s;
  int b, qt, kvh, off, left;
  int J0, J1, ulo, uhi;
  int unit, step;        // step > 0: no shares, this CTA takes every step-th (sequence, key head), one item per sequence
  bool have_seq, known;  // s is b's; the span is that of (b, qt)
  uint32_t deadline = 0;  // the word of attn_moving: many sequences without rows may have to be passed by
  __device__ __forceinline__ explicit AttnWalk(const AttnStart& st)
      : s(st.s), b(st.b), qt(st.qt), kvh(st.kvh), off(st.off), left(st.left), unit(0), step(0), have_seq(true), known(false) {}
  __device__ __forceinline__ AttnWalk(int first, int every) : qt(0), off(0), left(0), unit(first), step(every) {}
  __device__ __forceinline__ bool next_whole(const AttnParams& P, AttnItem& it) {
    for (; unit < P.seqs * P.heads_kv; unit += step) {
      it.b = unit / P.heads_kv;
      it.s = attn_seq(P, it.b);
      if (it.s.n <= 0) {
        attn_moving(P, deadline);
        continue;
      }
      it.kvh = unit - it.b * P.heads_kv;
      it.tok0 = 0;
      attn_span(P, it.s, 0, it.j0, it.j1, it.ulo, it.uhi);
      it.whole = true;
      it.slot = 0;
      unit += step;
      return true;
    }
    return false;
  }
  __device__ __forceinline__ bool next(const AttnParams& P, AttnItem& it) {
    const int per_item = P.tok_per_tile * P.tiles_per_item;
    while (left > 0 && b < P.seqs) {
      if (!known) {
        if (!have_seq) s = attn_seq(P, b);
        have_seq = true;
        if (qt * per_item >= s.n) {  // the rest of this sequence's items have no rows
          qt = 0;
          ++b;
          have_seq = false;
          attn_moving(P, deadline);
          continue;
        }
        attn_span(P, s, qt * per_item, J0, J1, ulo, uhi);
        known = true;
      }
      const int w = J1 - J0 + P.own;
      const int take = w - off < left ? w - off : left;  // 0: the share starts at the end of this unit
      it.s = s;
      it.b = b;
      it.kvh = kvh;
      it.tok0 = qt * per_item;
      it.ulo = ulo;
      it.uhi = uhi;
      it.j0 = off > 0 ? J0 + off - P.own : J0;
      it.j1 = J0 + off + take - P.own;
      it.whole = off == 0 && take == w;
      it.slot = off > 0 ? 0 : 1;
      left -= take;
      off = 0;
      if (++kvh == P.heads_kv) {
        kvh = 0;
        known = false;
        if (++qt == P.q_items) {
          qt = 0;
          ++b;
          have_seq = false;
        }
      }
      if (take > 0) return true;
    }
    return false;
  }
};

// Puts the units together that were cut: CTAs (c, *) do the one that c's share starts inside of, if that cut is the unit's first,
// 16 rows each, two a warp (a unit's 256 rows in one CTA were one latency after the other: 68 us).
constexpr int kAttnJoinThreads = 256;
constexpr int kAttnJoinRows = 16;  // divides part_rows

__global__ void __launch_bounds__(kAttnJoinThreads) attn_join_kernel(const __grid_constant__ AttnParams P);

typedef void (*AttnKernel)(const AttnParams);
// in qknorm_attn_inst.cu and qknorm_attn_tc_inst.cu
typedef void (*AttnTcKernel)(const AttnParams, const AttnMaps);
enum AttnFormat { kAttnBf16, kAttnE4m3, kAttnWidened };  // how a cache's elements are stored; the last: a 4-bit one, as K in bf16 and V in fp16
AttnKernel attn_general_kernel_for(AttnFormat format);
AttnKernel attn_join_kernel_for();
// forms of the tensor-core kernel: two query tiles per item, one, one of at most 32 rows
constexpr int kAttnTwo = 0, kAttnOne = 1, kAttnQuad = 2;
constexpr int kAttnTcThreads = 512;
constexpr int kAttnTcRegs = 128;  // registers per thread at launch that the kernel's register split counts on

}  // namespace qknorm
