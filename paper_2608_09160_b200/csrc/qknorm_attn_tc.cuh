// Attention over a paged cache on the tensor cores (tcgen05, accumulators in TMEM).
//
// A persistent CTA per SM walks over items: the query rows of one sequence that share a key head -- tokens
// times the group's query heads, packed into tiles of 128 rows -- and a range of key tiles of 128 keys.
//   warps 0-7    two softmax warpgroups; a thread owns a row of a 128 x 128 score tile
//   warp 13      copies K and V tiles into a ring in shared memory with TMA, a box per page (and tile)
//   warps 8-11   prepare what has arrived: widen FP8 tiles, blank V rows outside the item's keys; where a page is no
//                multiple of 8 tokens they gather the rows themselves with cp.async
//   warp 14      brings the query rows, by TMA where K and V come that way
//   warp 12      issues the tcgen05.mma
//   warp 15      says which items come next; with two query tiles it issues the second one's and warp 14 walks over the items
// Scores S_w = Q K^T land in TMEM (128 columns per warpgroup w).  The warpgroup reads them, keeps the running
// maximum and sum in registers, writes P = 2^(c (s - m)) back over S in 16 bits, and O_w += P V takes P from
// TMEM and V, keys by head_dim as it lies in the cache, as a transposed operand.  O_w stays in TMEM; it is rescaled only
// when the maximum has grown by more than 2^8, so a weight is at most 2^8 and the rescale is rare.
//
// Three forms:
//   two query tiles     (chunks): tile w belongs to warpgroup w, both use every K and V tile;
//   one query tile      (short chunks): key tiles alternate between the warpgroups, each with an O of its own over the
//                       same rows, joined through TMEM at the end of the item;
//   one tile of 32 rows (single tokens): as before, and the rows stand in all four quarters of the tile's 128 lanes.  A
//                       warp can only reach its own quarter; so the warp of quarter i takes keys 32 i .. 32 i + 31 of the
//                       tile (P is zero elsewhere in its quarter), four warps share what one would do alone, and the eight
//                       parts of a row are joined through shared memory at the end of the item.
// The first two keep the tensor pipe on one warpgroup's tile while the other one is in its exponentials.
//
// What shared memory holds beside the item's own: zeros in V rows outside the item's keys and in the columns behind head_dim, up to the
// next multiple of 64.  K rows outside the keys hold whatever the page holds there (their scores are masked), Q rows that no token fills
// hold other sequences' queries or what was there before (their results are stored nowhere).  Inside a tile that the causal
// edge or the window cuts, a V row with an infinity or a NaN would reach rows that do not see it (0 * inf): the loader looks at the V rows of such
// tiles and, if it finds one, has the item's rows done again one by one by attn_row, spread over the softmax warps that have them.
//
// Every wait is bounded: when for two seconds nothing has moved in the CTA -- 64 score tiles, 64 keys of a row done again, 64 items
// laid out, a sequence without rows passed by -- it sets the error word, and the CTA leaves.  Waiting for something slow (rows done again over
// a long context, an item of very many tiles) goes on for as long as that takes.  The time stands in shared memory and not
// with the one who waits, and there is no other sign to leave: the waiting loop stands in some 30 places between the instructions of
// the main loops, and with a count of what has moved beside each loop's own start time a prompt of 8192 took 850 to 940 us instead of 770.
//
// FP8 cache: K and V are staged raw and widened to fp16, which holds every E4M3 value exactly; Q is
// brought to fp16 with a power of two per row, which loses nothing but parts below 2^-30 of the row's largest element.
//
// Rounding: P is rounded for the second product, to bf16 (2^-8 relative) or, with an FP8 cache, to fp16 (2^-11 relative, and
// 2^-25 absolute below 2^-14; the sum l takes them unrounded).  So P stands for 2^7 times the weights there: what the maximum may lag
// behind still fits, and a weight keeps half a step of 2^-32 of the largest one instead of 2^-25.  (With weights as they are, a key that
// outweighs its row's others by 2^26 left them out of O and in l.)  Otherwise only the output is rounded; sums, maxima and O are fp32.
//
// What bounds it (B200; calls in a captured graph, 6448 GB/s and 1676 TFLOP/s measured copy and matrix rates):
//   single tokens, bf16   HBM: 64 sequences to 8192 keys, 64 query and 8 key heads: 233 us, 5.8 TB/s (268 us after a second of nothing
//                         else, when the power limit has brought the clock from 1965 to 1515 MHz)
//   single tokens, FP8    the tile workers and shared memory (a K and a V tile are written, read, written as fp16 and read by
//                         the products: 224 KB of 128-byte-a-cycle traffic): 16 sequences to 32000 keys: 199 us (217 at 1770 MHz), floor 102
//   few short sequences   latency: about 5 us until the first product, then a tile each 0.9 us: 8 x 1000 keys: 17.1 us, floor 3.3
//   chunks and prompts    exponentials and products of two tiles in turn, 3700 cycles a pair of 128 x 128 (products alone 2048,
//                         exponentials alone as many), and 8 to 10 thousand cycles a unit for its first and last steps: 8192 tokens, 40 heads:
//                         675 us (765 at 1740 MHz), floor 410; over an FP8 cache 1215, for the widening
// Tiles of 128 x 128: the largest M of one CTA's products, and two score tiles and two O of 128 columns fill the 512 columns of TMEM.
#pragma once
#include "qknorm_attn.cuh"

namespace qknorm {

namespace tc {

// Shared-memory matrix descriptor, 128-byte swizzle.  The low word holds the address in 16-byte units (moving on by n
// bytes adds n / 16 to it) and the leading stride, the high word the stride between groups of 8 rows: a constant of the tile.
__device__ __forceinline__ uint32_t desc_lo(uint32_t addr, uint32_t lbo) { return (addr >> 4) | ((lbo >> 4) << 16); }
__host__ __device__ constexpr uint32_t desc_hi(uint32_t group) { return (group >> 4) | (1u << 14) | (2u << 29); }
// fp32 accumulators, both operands bf16 (or both fp16), M = 128
__host__ __device__ constexpr uint32_t instr_desc(int n, bool f16, bool b_transposed) {
  return (1u << 4) | ((f16 ? 0u : 1u) << 7) | ((f16 ? 0u : 1u) << 10) | ((b_transposed ? 1u : 0u) << 16) |
         ((uint32_t)(n >> 3) << 17) | ((128u >> 4) << 24);
}
__device__ __forceinline__ void mma_ss(uint32_t d, uint32_t a_lo, uint32_t a_hi, uint32_t b_lo, uint32_t b_hi, uint32_t idesc, bool acc) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\tsetp.ne.u32 p, %4, 0;\n\t"
      "mov.b64 a, {%1, %5};\n\tmov.b64 b, {%2, %6};\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, p;\n\t}" ::"r"(d), "r"(a_lo), "r"(b_lo), "r"(idesc), "r"((uint32_t)acc),
      "r"(a_hi), "r"(b_hi)
      : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint32_t b_lo, uint32_t b_hi, uint32_t idesc, bool acc) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 b;\n\tsetp.ne.u32 p, %4, 0;\n\t"
      "mov.b64 b, {%2, %5};\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %3, p;\n\t}" ::"r"(d), "r"(a), "r"(b_lo), "r"(idesc), "r"((uint32_t)acc),
      "r"(b_hi)
      : "memory");
}
__device__ __forceinline__ void commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}

#define QKNORM_R8(m, i) m(i), m(i + 1), m(i + 2), m(i + 3), m(i + 4), m(i + 5), m(i + 6), m(i + 7)
#define QKNORM_O(i) "=r"(r[i])
#define QKNORM_I(i) "r"(r[i])
// 32 columns of this lane's row
__device__ __forceinline__ void ld32(uint32_t addr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : QKNORM_R8(QKNORM_O, 0), QKNORM_R8(QKNORM_O, 8), QKNORM_R8(QKNORM_O, 16), QKNORM_R8(QKNORM_O, 24)
      : "r"(addr));
}
// 16 columns
__device__ __forceinline__ void ld16(uint32_t addr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : QKNORM_R8(QKNORM_O, 0), QKNORM_R8(QKNORM_O, 8)
      : "r"(addr));
}
__device__ __forceinline__ void st16(uint32_t addr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, "
      "%15};" ::QKNORM_R8(QKNORM_I, 0),
      QKNORM_R8(QKNORM_I, 8), "r"(addr)
      : "memory");
}
#undef QKNORM_O
#undef QKNORM_I
#undef QKNORM_R8

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
__device__ __forceinline__ uint32_t pack_f16(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
// The same; what lies beyond the format becomes its largest value (NaN stays NaN).
__device__ __forceinline__ uint32_t pack_f16_sat(float a, float b) {
  uint32_t r;
  asm("cvt.rn.satfinite.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
  return r;
}
// Has the phase completed?  Does not wait: try_wait may suspend the thread for a while.
__device__ __forceinline__ bool test(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(bar), "r"(parity)
      : "memory");
  return ok != 0;
}
__device__ __forceinline__ void arrive_n(uint32_t bar, uint32_t n) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(n) : "memory");
}
// One box: column x, token t of its page, head h, page p; what lies outside the pool is zeros.
__device__ __forceinline__ void tma4(uint32_t dst, const CUtensorMap* map, int x, int t, int h, int p, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst),
      "l"(map), "r"(x), "r"(t), "r"(h), "r"(p), "r"(bar)
      : "memory");
}
// Whole rows of 128 columns: half column h of the row (or of the head), 8-token group t, page (or page and head) p.
__device__ __forceinline__ void tma5(uint32_t dst, const CUtensorMap* map, int h, int t, int p, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.5d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %2, %3, %4, %5}], [%6];" ::"r"(dst),
      "l"(map), "r"(0), "r"(h), "r"(t), "r"(p), "r"(bar)
      : "memory");
}
__device__ __forceinline__ void tma3(uint32_t dst, const CUtensorMap* map, int x, int h, int t, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
      "l"(map), "r"(x), "r"(h), "r"(t), "r"(bar)
      : "memory");
}
// 16 bytes from global to shared memory, or 16 zero bytes
__device__ __forceinline__ void cp16(uint32_t dst, const void* src, bool take) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(take ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void cp_wait_all() { asm volatile("cp.async.wait_all;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ void sts128(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}

}  // namespace tc

// Shared memory, byte offsets from a 1024-byte aligned base.
template <int DP, bool F8>
struct AttnSmem {
  static constexpr int kTile = kAttnTile * DP * 2;  // a 16-bit tile of Q, K or V
  static constexpr int kRaw = kAttnTile * DP;       // an FP8 tile: 32 rows at a time land in the upper half of the place that
                                                    // their fp16 form takes, and one warp widens them over themselves
  static constexpr int kStages = DP == 128 ? 5 : 10;
  static constexpr int kLag = kStages - 2;  // gathered tiles that stay in flight when the next is issued
  static constexpr int kQ0 = 0;             // two Q tiles
  static constexpr int kRing = 2 * kTile;
  static constexpr int kFull = kRing + kStages * kTile;  // mbarriers, 8 bytes each
  static constexpr int kEmpty = kFull + 8 * kStages;
  static constexpr int kQFull = kEmpty + 8 * kStages;
  static constexpr int kQEmpty = kQFull + 16;
  static constexpr int kSFull = kQEmpty + 16;
  static constexpr int kPFull = kSFull + 16;
  static constexpr int kPMost = kPFull + 16;  // the first 96 keys' weights are there (not QUAD)
  static constexpr int kOFull = kPMost + 16;
  static constexpr int kOFree = kOFull + 16;
  static constexpr int kMl = kOFree + 16;
  static constexpr int kMlFree = kMl + 8;
  static constexpr int kDrain = kMlFree + 8;
  static constexpr int kRawFull = kDrain + 8;         // per stage: an FP8 tile, or a bf16 V tile that wants looking at, is there
  static constexpr int kQRaw = kRawFull + 8 * kStages;  // [2] FP8 cache: a bf16 Q tile is there
  static constexpr int kTurn = kQRaw + 16;            // [2] two forms: whose turn it is to issue
  static constexpr int kPass = kTurn + 16;            // the softmax warps' steps through the join of an item
  static constexpr int kTmem = kPass + 8;             // TMEM base address
  static constexpr int kAbort = kTmem + 4;            // a wait ran out: everybody leaves
  static constexpr int kDeadline = kAbort + 4;        // see attn_moving
  static constexpr int kPoison = kDeadline + 8;       // [4] 1 + number of an item that holds a V row to be careful with
  // FP8 cache: [4][128] bytes, the exponent taken out of a Q row (0: none).  Four sets, because a set is read until the
  // item's last score tile is done with, which can be after its Q buffer has been given to a later item; a set comes
  // round again only after the tensor warp has seen the scores of the item before last consumed.
  static constexpr int kQScale = kPoison + 16;
  static constexpr int kItemSlots = F8 ? 2 : 4;              // items ahead of the slowest reader
  static constexpr int kItems = kQScale + (F8 ? 512 : 0);    // [kItemSlots][16] ints, see put_item
  static constexpr int kItemFull = kItems + 64 * kItemSlots;
  static constexpr int kItemEmpty = kItemFull + 8 * kItemSlots;
  static constexpr int kMlRows = kItemEmpty + 8 * kItemSlots;             // [8 softmax warps][32] float2, one-tile forms: (m, l) of their parts
  static constexpr int kBytes = kMlRows + 2048;
};

static_assert(AttnSmem<128, false>::kBytes <= 232448 && AttnSmem<128, true>::kBytes <= 232448, "shared memory of one CTA");

// Key tiles [a, b) that query tile w of the item uses, and how its rows' ranges spread.
struct AttnTileRange {
  int a, b;
  int rows;            // rows in use
  int hi_min, lo_max;  // end of the first token's keys, start of the last token's
};
__device__ __forceinline__ AttnTileRange attn_tile_range(const AttnParams& P, const AttnItem& it, int w) {
  AttnTileRange r;
  const int t0 = it.tok0 + w * P.tok_per_tile;
  const int t1 = t0 + P.tok_per_tile < it.s.n ? t0 + P.tok_per_tile : it.s.n;
  r.a = r.b = r.rows = r.hi_min = r.lo_max = 0;
  if (t0 >= t1) return r;
  r.rows = (t1 - t0) * P.group;
  r.hi_min = attn_hi(P, it.s, t0);
  r.lo_max = attn_lo(P, it.s, t1 - 1);
  const int lo = attn_lo(P, it.s, t0), hi = attn_hi(P, it.s, t1 - 1);
  if (hi <= lo) return r;
  const int a = lo / kAttnTile, b = (hi + kAttnTile - 1) / kAttnTile;
  r.a = a > it.j0 ? a : it.j0;
  r.b = b < it.j1 ? b : it.j1;
  if (r.b <= r.a) r.a = r.b = 0;
  return r;
}
// Does the causal edge or the window cut through this tile's keys in use for some row of the query tile?
__device__ __forceinline__ bool attn_cut(const AttnItem& it, const AttnTileRange& r, int j) {
  const int k0 = j * kAttnTile, k1 = k0 + kAttnTile;
  return j >= r.a && j < r.b && ((k1 < it.uhi ? k1 : it.uhi) > r.hi_min || (k0 > it.ulo ? k0 : it.ulo) < r.lo_max);
}

template <int DP, bool F8, int FORM, bool TMA>
struct AttnTc {
  using L = AttnSmem<DP, F8>;
  static constexpr bool ONE = FORM != kAttnTwo;
  static constexpr bool QUAD = FORM == kAttnQuad;
  // Tiles of 64 columns: rows of 128 bytes, 16-byte pieces swizzled within 8 rows.  Q: its 64-column halves one after the
  // other.  K and V: groups of 8 rows, a group's halves side by side -- so that one TMA box can bring whole rows of a page.
  static constexpr int kHalf = kAttnTile * 128;
  static constexpr int kGroup = 8 * 2 * DP;  // bytes of 8 rows of K or V
  // Where row r of a raw FP8 tile lies: with the 31 rows that the same warp widens, behind the start of their fp16 form.
  __device__ __forceinline__ static uint32_t raw_at(int r) { return (r >> 5) * (64 * DP) + 32 * DP + (r & 31) * DP; }
  __device__ __forceinline__ static uint32_t kv_at(int r, int c) {  // row r, 16-byte piece c
    return (r >> 3) * kGroup + (c >> 3) * 1024 + (r & 7) * 128 + (((c ^ r) & 7) << 4);
  }

  static constexpr float kUp = F8 ? 7.f : 0.f;  // P = 2^(c (s - m) + kUp), and l is the sum of those

  const AttnParams& P;
  const AttnMaps& maps;
  uint32_t smem;
  unsigned char* smem_ptr;

  __device__ __forceinline__ volatile int* abort_flag() const { return reinterpret_cast<volatile int*>(smem_ptr + L::kAbort); }
  __device__ __forceinline__ volatile int* poison() const { return reinterpret_cast<volatile int*>(smem_ptr + L::kPoison); }

  __device__ __forceinline__ volatile unsigned* deadline() const { return reinterpret_cast<volatile unsigned*>(smem_ptr + L::kDeadline); }
  __device__ __forceinline__ void moving() const { attn_moving(P, smem + L::kDeadline); }

  // Bounded (see above); false: leave.
  __device__ __forceinline__ bool wait(uint32_t bar, uint32_t parity) const {
    if (ptx::mbar_try_wait(bar, parity)) return true;
    return wait_slow(bar, parity);
  }
  __device__ __forceinline__ bool wait_slow(uint32_t bar, uint32_t parity) const {
    while (!ptx::mbar_try_wait(bar, parity)) {
      if ((int)(attn_time() - *deadline()) > 0) {
        *abort_flag() = 1;
        *P.error = 7;
        return false;
      }
    }
    return true;
  }
  // Without a look at the abort flag: what is waited for is on its way whatever else happened.
  __device__ __forceinline__ void wait_drain(uint32_t bar, uint32_t parity) const {
    const unsigned long long t0 = ptx::globaltimer_ns();
    while (!ptx::mbar_try_wait(bar, parity))
      if (ptx::globaltimer_ns() - t0 > 2000000000ull) {
        *P.error = 9;
        return;
      }
  }
  __device__ __forceinline__ uint32_t full(uint32_t pos) const { return smem + L::kFull + 8 * (pos % L::kStages); }
  __device__ __forceinline__ uint32_t empty(uint32_t pos) const { return smem + L::kEmpty + 8 * (pos % L::kStages); }
  __device__ __forceinline__ uint32_t stage(uint32_t pos) const { return smem + L::kRing + (pos % L::kStages) * L::kTile; }

  // ---- items ----------------------------------------------------------------------------------------
  // One warp (15; 14 in the two-tile form) walks over the CTA's share and lays the items down for everybody else, some ahead.
  static constexpr int kReaders = 8 + 4 + 1 + (ONE ? 1 : 2) + (TMA ? 1 : 0);  // softmax and tile warps, Q, matrix threads, producer

  __device__ __forceinline__ volatile int* item_at(uint32_t i) const {
    return reinterpret_cast<volatile int*>(smem_ptr + L::kItems) + (i % L::kItemSlots) * 16;
  }
  // Lays down item i, or that there are no more; one thread.  False: that was the last, or leave.
  __device__ __forceinline__ bool put_item(AttnWalk& walk, uint32_t i) const {
    AttnItem it;
    const bool more = walk.step > 0 ? walk.next_whole(P, it) : walk.next(P, it);
    if (i >= (uint32_t)L::kItemSlots && !wait(smem + L::kItemEmpty + 8 * (i % L::kItemSlots), ((i / L::kItemSlots) - 1) & 1)) return false;
    volatile int* at = item_at(i);
    at[0] = more ? it.b : -1;
    if ((i & 63) == 63) moving();
    if (more) {
      at[1] = it.s.row0;
      at[2] = it.s.n;
      at[3] = it.s.keys;
      at[4] = (int)(it.s.pos0 & 0xffffffffll);
      at[5] = (int)(it.s.pos0 >> 32);
      at[6] = it.kvh;
      at[7] = it.tok0;
      at[8] = it.j0;
      at[9] = it.j1;
      at[10] = it.ulo;
      at[11] = it.uhi;
      at[12] = (it.whole ? 1 : 0) | it.slot << 1;
    }
    tc::arrive(smem + L::kItemFull + 8 * (i % L::kItemSlots));
    return more;
  }
  __device__ __forceinline__ void get_item(uint32_t i, AttnItem& it) const {
    const volatile int* at = item_at(i);
    it.b = at[0];
    it.s.row0 = at[1];
    it.s.n = at[2];
    it.s.keys = at[3];
    it.s.pos0 = (long long)(uint32_t)at[4] | (long long)at[5] << 32;
    it.kvh = at[6];
    it.tok0 = at[7];
    it.j0 = at[8];
    it.j1 = at[9];
    it.ulo = at[10];
    it.uhi = at[11];
    it.whole = at[12] & 1;
    it.slot = at[12] >> 1;
  }
  __device__ __forceinline__ bool item_wait(uint32_t i) const {
    return wait(smem + L::kItemFull + 8 * (i % L::kItemSlots), (i / L::kItemSlots) & 1);
  }
  __device__ __forceinline__ void item_done(uint32_t i) const { tc::arrive(smem + L::kItemEmpty + 8 * (i % L::kItemSlots)); }
  // Item i for a whole warp, which keeps it in registers; false: there are no more, or leave.
  __device__ __forceinline__ bool take_item(uint32_t i, AttnItem& it) const {
    if (!__all_sync(0xffffffffu, item_wait(i))) return false;
    get_item(i, it);
    __syncwarp();
    if ((threadIdx.x & 31) == 0) item_done(i);
    return it.b >= 0;
  }

  // ---- K and V tiles --------------------------------------------------------------------------------
  // V rows outside the item's keys have to be zeros (a weight of 0 times a NaN would be one), and the rows of a cut tile
  // looked through.  K may hold anything there: its scores are masked.
  struct VJob {
    bool blank, look;
  };
  __device__ __forceinline__ static VJob v_job(const AttnItem& it, const AttnTileRange& r0, const AttnTileRange& r1, int j) {
    const int k0 = j * kAttnTile;
    return VJob{k0 < it.ulo || k0 + kAttnTile > it.uhi, attn_cut(it, r0, j) || (!ONE && attn_cut(it, r1, j))};
  }

  // Warp 13.  A lane issues one box: tokens of a page, whole heads or 64 columns of them.
  __device__ __forceinline__ void run_producer(int lane) const {
    const uint32_t all = 0xffffffffu;
    // at most 32 boxes: one has at least 8 tokens; half heads (kBoxHalf) only come in boxes of 8
    const int halves = !F8 && P.box_kind == kBoxHalf ? DP / 64 : 1;
    const int boxes = (kAttnTile >> P.box_shift) * halves;
    const int box = lane / halves, half = lane % halves;
    const uint32_t at = F8 ? raw_at(box * P.box_rows) : box * P.box_rows * 2 * DP + half * 1024;
    uint32_t pos = 0, waiting_raw = 0, raw_ph = 0;  // bits by stage: its newest tile went to kRawFull; phase of kRawFull
    bool ok = true;
    // page and token of this lane's box of tile j; the page past the last one stands for zeros
    auto look_up = [&](const AttnItem& it, int j, int& within) {
      const int key = j * kAttnTile + box * P.box_rows;
      within = 0;
      long long page = P.num_pages;
      if (lane < boxes && key < it.uhi && key + P.box_rows > it.ulo) {
        const long long e = attn_page(P, it.b, key, within);
        if (e >= 0) page = e;
      }
      return (int)page;
    };
    AttnItem it;
    for (uint32_t n_item = 0; ok && take_item(n_item, it); ++n_item) {
      if (it.j0 >= it.j1) continue;
      const AttnTileRange r0 = attn_tile_range(P, it, 0);
      AttnTileRange r1 = r0;
      if (!ONE) r1 = attn_tile_range(P, it, 1);
      int next_within, next = look_up(it, it.j0, next_within);
      for (int j = it.j0; ok && j < it.j1; ++j) {
        const int page = next, within = next_within;
        if (j + 1 < it.j1) next = look_up(it, j + 1, next_within);
        const VJob job = v_job(it, r0, r1, j);
#pragma unroll
        for (int v = 0; v < 2; ++v) {
          uint32_t bar, dst;
          const uint32_t st = pos % L::kStages, round = pos / L::kStages;
          if (round > 0 && !(ok = __all_sync(all, wait(empty(pos), (round - 1) & 1)))) break;
          const bool raw = F8 || (v == 1 && (job.blank || job.look));
          bar = raw ? smem + L::kRawFull + 8 * st : full(pos);
          dst = stage(pos);
          waiting_raw = (waiting_raw & ~(1u << st)) | (raw ? 1u << st : 0u);
          if (raw) raw_ph ^= 1u << st;
          if (lane == 0) {
            if (!raw) tc::arrive_n(bar, 3);  // the four warps that would otherwise have had to look
            ptx::mbar_arrive_expect_tx(bar, F8 ? L::kRaw : L::kTile);
          }
          __syncwarp();
          if (lane < boxes) {
            const CUtensorMap* map = v ? &maps.v : &maps.k;
            if (P.box_kind == kBoxHalf) tc::tma4(dst + at, map, half * 64, within, it.kvh, page, bar);
            else if (P.box_kind == kBoxHeadInRow) tc::tma5(dst + at, map, 2 * it.kvh, within >> 3, page, bar);
            else tc::tma5(dst + at, map, 0, within >> 3, page * P.heads_kv + it.kvh, bar);
          }
          ++pos;
        }
      }
    }
    if (*abort_flag()) {  // nobody consumes what is still on its way, but it must have landed before the CTA ends
      const uint32_t n = L::kStages;
      for (uint32_t p = pos > n ? pos - n : 0; p < pos; ++p) {
        if ((waiting_raw >> (p % n)) & 1) wait_drain(smem + L::kRawFull + 8 * (p % n), ((raw_ph >> (p % n)) & 1) ^ 1);
        else wait_drain(full(p), (p / n) & 1);
      }
    }
  }

  __device__ __forceinline__ void signal(uint32_t bar, int lane) const {
    ptx::fence_proxy_async();
    __syncwarp();
    if (lane == 0) tc::arrive(bar);
  }
  __device__ __forceinline__ static bool odd_bf16(uint32_t u) { return (u & 0x7f80u) == 0x7f80u || (u & 0x7f800000u) == 0x7f800000u; }
  __device__ __forceinline__ static bool odd_f16(uint32_t u) { return (u & 0x7c00u) == 0x7c00u || (u & 0x7c000000u) == 0x7c000000u; }

  static constexpr int kChunks = F8 ? DP / 16 : DP / 8;  // 16-byte pieces of a stored row; also steps per tile
  static constexpr int kRowsAt = 32 / kChunks;           // rows a warp handles in one step
  __device__ __forceinline__ static int row_of(int tid, int step) { return (tid & ~31) + step * kRowsAt + (tid & 31) / kChunks; }

  // Looks through the rows [from, to) of a bf16 tile for infinities and NaN; blanks the others if asked to.
  __device__ __forceinline__ bool inspect(uint32_t tile_at, int tid, int from, int to, bool blank, bool look) const {
    const int c = tid % kChunks;
    bool bad = false;
#pragma unroll 4
    for (int i = 0; i < kChunks; ++i) {
      const int r = row_of(tid, i);
      const uint32_t at = tile_at + kv_at(r, c);
      if (r < from || r >= to) {
        if (blank) tc::sts128(at, 0u, 0u, 0u, 0u);
      } else if (look) {
        const uint4 v = ptx::lds128(at);
        bad |= odd_bf16(v.x) || odd_bf16(v.y) || odd_bf16(v.z) || odd_bf16(v.w);
      }
    }
    return bad;
  }

  // The first row of a thread's pieces of FP8 rows.  With 128 columns, 8 lanes take the first half of one row and the second of
  // its neighbour: the two halves of one widened row lie on the same banks, but the swizzle puts neighbours on different ones.
  // (Both halves of one row, one of them written in the other order: that choice became branches, 897 cycles a tile against 413.)
  __device__ __forceinline__ static int raw_row(int tid) { return row_of(tid, 0) ^ (DP == 128 ? (tid >> 2) & 1 : 0); }

  // This warp's 32 rows of an FP8 tile to fp16, over themselves: all read before any is written.  CARE: rows outside [from, to)
  // become zeros, the others are looked through for NaN.
  template <bool CARE>
  __device__ __forceinline__ bool widen(uint32_t tile_at, int tid, int from, int to) const {
    const int c = tid % kChunks, r0 = raw_row(tid);
    const uint32_t src = tile_at + raw_at(r0) + c * 16;
    // Pieces 2c and 2c + 1 of row r0; the next rows of this thread are kRowsAt further each, which is 4 or 8: half a group or one.
    const uint32_t dst = tile_at + kv_at(r0 & ~7, 2 * c & ~7), row = (r0 & 7) * 128;
    const uint32_t turn = (((2 * c) ^ r0) & 7) << 4;
    bool bad = false;
    uint4 v[kChunks];
#pragma unroll
    for (int i = 0; i < kChunks; ++i) v[i] = ptx::lds128(src + i * kRowsAt * DP);
    __syncwarp();
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
      if (CARE && (r0 + i * kRowsAt < from || r0 + i * kRowsAt >= to)) v[i] = make_uint4(0u, 0u, 0u, 0u);
      uint32_t h[8];
      e4m3x4_to_f16x2(v[i].x, h[0], h[1]);
      e4m3x4_to_f16x2(v[i].y, h[2], h[3]);
      e4m3x4_to_f16x2(v[i].z, h[4], h[5]);
      e4m3x4_to_f16x2(v[i].w, h[6], h[7]);
      if (CARE) {
#pragma unroll
        for (int e = 0; e < 8; ++e) bad |= odd_f16(h[e]);
      }
      // the swizzle of row r0 + i * kRowsAt differs from row r0's by a constant: r0 % 8 < kRowsAt, or kRowsAt is 8
      const uint32_t at = dst + (i * kRowsAt >> 3) * kGroup + ((i * kRowsAt) & 7) * 128 + row + (turn ^ (((i * kRowsAt) & 7) << 4));
      tc::sts128(at, h[0], h[1], h[2], h[3]);
      tc::sts128(at ^ 16, h[4], h[5], h[6], h[7]);
    }
    return bad;
  }

  // Warps 8-11 behind TMA copies.
  __device__ __forceinline__ void run_workers(int tid) const {
    const uint32_t all = 0xffffffffu;
    const int lane = tid & 31;
    uint32_t pos = 0, raw_ph = 0;
    int count = 0;  // items with keys
    AttnItem it;
    for (uint32_t n_item = 0; take_item(n_item, it); ++n_item) {
      if (it.j0 >= it.j1) continue;
      const AttnTileRange r0 = attn_tile_range(P, it, 0);
      AttnTileRange r1 = r0;
      if (!ONE) r1 = attn_tile_range(P, it, 1);
      if constexpr (F8) {
        for (int n = 0; n < 2 * (it.j1 - it.j0); ++n, ++pos) {
          const int j = it.j0 + (n >> 1), k0 = j * kAttnTile;
          const VJob job = v_job(it, r0, r1, j);
          const uint32_t st = pos % L::kStages;
          if (!__all_sync(all, wait(smem + L::kRawFull + 8 * st, (pos / L::kStages) & 1))) return;
          if ((n & 1) && (job.blank || job.look)) {
            if (widen<true>(stage(pos), tid, it.ulo - k0, it.uhi - k0) && job.look) poison()[count & 3] = count + 1;
          } else {
            widen<false>(stage(pos), tid, 0, 0);
          }
          signal(full(pos), lane);
        }
      } else {
        for (int j = it.j0; j < it.j1; ++j) {
          const VJob job = v_job(it, r0, r1, j);
          if (!job.blank && !job.look) continue;
          const uint32_t vp = pos + 2 * (j - it.j0) + 1, st = vp % L::kStages;
          if (!__all_sync(all, wait(smem + L::kRawFull + 8 * st, (raw_ph >> st) & 1))) return;
          raw_ph ^= 1u << st;
          const int k0 = j * kAttnTile;
          if (inspect(stage(vp), tid, it.ulo - k0, it.uhi - k0, true, job.look)) poison()[count & 3] = count + 1;
          signal(full(vp), lane);
        }
        pos += 2 * (it.j1 - it.j0);
      }
      ++count;
    }
  }

  // Warps 8-11 where a page is no whole number of 8 tokens: they copy the rows themselves.  A warp fills 32 rows of a tile.
  // A lane looks up one row's place; 32 / kRowsAt lanes then copy that row side by side, the place handed round by
  // shuffle: one table read per row, and it is made a tile ahead.
  struct Loader {
    uint32_t pos = 0;    // tiles issued
    int pending = 0;     // issued, not handed over
    int look_item = -1;  // the newest pending tile is V and cut: look through it, name this item
  };

  // The oldest pending tile has arrived (its cp.async group is complete): hand it over.
  __device__ __forceinline__ bool hand_over(Loader& ld, int tid) const {
    const int lane = tid & 31;
    const uint32_t pos = ld.pos - ld.pending;
    const bool look = ld.look_item >= 0 && ld.pending == 1;
    bool bad = false;
    if constexpr (F8) {
      bad = look ? widen<true>(stage(pos), tid, 0, kAttnTile) : widen<false>(stage(pos), tid, 0, 0);
    } else if (look) {
      bad = inspect(stage(pos), tid, 0, kAttnTile, false, true);
    }
    if (look) {
      if (bad) poison()[ld.look_item & 3] = ld.look_item + 1;
      ld.look_item = -1;
    }
    signal(full(pos), lane);
    // The wait before this call covered this lane's own copies; widen reads pieces that the lanes beside it copied (raw_row).
    __syncwarp();
    --ld.pending;
    return true;
  }
  __device__ __forceinline__ bool flush(Loader& ld, int tid) const {
    tc::cp_wait<0>();
    while (ld.pending > 0)
      if (!hand_over(ld, tid)) return false;
    return true;
  }
  // Page-table entry of the key this lane looks up in tile j (-1: nothing to load).
  __device__ __forceinline__ int lane_entry(int tid, const AttnItem& it, int j, int& within) const {
    const int key = j * kAttnTile + tid;
    within = 0;
    return key >= it.ulo && key < it.uhi ? (int)attn_page(P, it.b, key, within) : -1;
  }
  // One K or V tile.  off: where this lane's row starts, elements; negative: a row of zeros.
  __device__ __forceinline__ bool load_tile(Loader& ld, int tid, const void* from, long long off) const {
    const uint32_t pos = ld.pos;
    // wait, but never while sitting on tiles that somebody else waits for
    if (pos >= (uint32_t)L::kStages && !__all_sync(0xffffffffu, tc::test(empty(pos), ((pos / L::kStages) - 1) & 1)) &&
        !(flush(ld, tid) && __all_sync(0xffffffffu, wait(empty(pos), ((pos / L::kStages) - 1) & 1))))
      return false;
    const int c = tid % kChunks, src_lane = (tid & 31) / kChunks;
    const bool in_head = c * (F8 ? 16 : 8) < P.head_dim;
    const char* base = reinterpret_cast<const char*>(from);
    const uint32_t dst = stage(pos) + (F8 ? c * 16 : 0);
    constexpr int kBatch = 8 < kChunks ? 8 : kChunks;  // shuffles ahead of copies: one after the other they would wait in one queue
#pragma unroll
    for (int i0 = 0; i0 < kChunks; i0 += kBatch) {
      long long at[kBatch];
#pragma unroll
      for (int b = 0; b < kBatch; ++b) at[b] = __shfl_sync(0xffffffffu, off, (i0 + b) * kRowsAt + src_lane);
#pragma unroll
      for (int b = 0; b < kBatch; ++b) {
        const int r = row_of(tid, i0 + b);
        const bool take = in_head && at[b] >= 0;
        const char* src = take ? base + (at[b] + c * (F8 ? 16 : 8)) * (F8 ? 1 : 2) : base;
        tc::cp16(dst + (F8 ? raw_at(r) : kv_at(r, c)), src, take);
      }
    }
    tc::cp_commit();
    ++ld.pos;
    ++ld.pending;
    if (ld.pending > L::kLag) {
      tc::cp_wait<L::kLag>();
      return hand_over(ld, tid);
    }
    return true;
  }

  __device__ __forceinline__ void run_loader(int tid) const {
    Loader ld;
    int count = 0;  // items with keys
    bool ok = true;
    AttnItem it;
    for (uint32_t n_item = 0; ok; ++n_item) {
      // the next item may have to wait for rows that wait for tiles that are pending here
      if (!__all_sync(0xffffffffu, tc::test(smem + L::kItemFull + 8 * (n_item % L::kItemSlots), (n_item / L::kItemSlots) & 1)) &&
          !(ok = flush(ld, tid)))
        break;
      if (!take_item(n_item, it)) break;
      if (it.j0 >= it.j1) continue;
      const AttnTileRange r0 = attn_tile_range(P, it, 0);
      AttnTileRange r1 = r0;
      if (!ONE) r1 = attn_tile_range(P, it, 1);
      int within, entry = lane_entry(tid, it, it.j0, within);
      for (int j = it.j0; j < it.j1; ++j) {
        const int page = entry, tok = within;
        if (j + 1 < it.j1) entry = lane_entry(tid, it, j + 1, within);
        ok = load_tile(ld, tid, P.k.base, page < 0 ? -1 : page * P.k.page + tok * P.k.token + it.kvh * P.k.head);
        if (!ok) break;
        const bool look = v_job(it, r0, r1, j).look;
        if (look && !(ok = flush(ld, tid))) break;
        if (look) ld.look_item = count;
        ok = load_tile(ld, tid, P.v.base, page < 0 ? -1 : page * P.v.page + tok * P.v.token + it.kvh * P.v.head);
        if (!ok) break;
        if (look && !(ok = flush(ld, tid))) break;
      }
      ++count;
    }
    if (ok) flush(ld, tid);
    tc::cp_wait<0>();
  }

  // ---- query tiles ----------------------------------------------------------------------------------
  static constexpr int kQThreads = 32;  // warp 14

  // Query tile of `rows` rows from token tok0 into Q buffer `buf`; the rest of the last 32 rows in use is zeros.  QUAD: the
  // same 32 rows four times.
  __device__ __forceinline__ void load_q(int tid, const AttnItem& it, int tok0, int rows, int buf, int scale_set) const {
    constexpr int kQChunks = DP / 8, kStep = kQThreads / kQChunks;
    const int c = tid % kQChunks, r0 = tid / kQChunks;
    const uint32_t dst = smem + L::kQ0 + buf * L::kTile + (c >> 3) * kHalf;
    const bool in_head = c * 8 < P.head_dim;
    const int end = (rows + 31) & ~31;
    const uint16_t* from = P.q + (it.s.row0 + (long long)tok0) * P.ld_q + (long long)(it.kvh * P.group) * P.head_dim + c * 8;
    auto row_at = [&](int r) {
      const int tok = (int)((unsigned)r / (unsigned)P.group), g = r - tok * P.group;
      return from + tok * P.ld_q + g * P.head_dim;
    };
    if constexpr (!F8) {  // asynchronous: every row is on its way before the first is waited for
      for (int r = r0; r < end; r += kStep) {
        const bool take = in_head && r < rows;
#pragma unroll
        for (int k = 0; k < (QUAD ? 4 : 1); ++k)
          tc::cp16(dst + (r + 32 * k) * 128 + (((c ^ r) & 7) << 4), take ? row_at(r) : P.q, take);
      }
    } else {
      constexpr int kBatch = 4;  // kStep * kBatch divides 32
      for (int i0 = r0; i0 < end; i0 += kStep * kBatch) {
        uint4 v[kBatch];
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
          const int r = i0 + b * kStep;
          v[b] = in_head && r < rows ? *reinterpret_cast<const uint4*>(row_at(r)) : make_uint4(0u, 0u, 0u, 0u);
        }
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
          const int r = i0 + b * kStep;
          q_to_f16(v[b], r, c, scale_set);
#pragma unroll
          for (int k = 0; k < (QUAD ? 4 : 1); ++k) tc::sts128(dst + (r + 32 * k) * 128 + (((c ^ r) & 7) << 4), v[b].x, v[b].y, v[b].z, v[b].w);
        }
      }
    }
  }

  // FP8 cache: 8 elements of Q row r (the row's other pieces are in the neighbouring lanes) from bf16 to fp16, the row's largest
  // exponent brought to 2^8; rows of zeros, tiny rows and rows with infinities or NaN as they are.
  __device__ __forceinline__ void q_to_f16(uint4& v, int r, int c, int scale_set) const {
    uint32_t u[4] = {v.x, v.y, v.z, v.w};
    uint32_t mag = 0;  // largest magnitude of the row, as bf16 bits
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t lo = u[e] & 0x7fffu, hi = (u[e] >> 16) & 0x7fffu;
      mag = max(mag, max(lo, hi));
    }
#pragma unroll
    for (int off = DP / 16; off > 0; off >>= 1) mag = max(mag, __shfl_xor_sync(0xffffffffu, mag, off));
    const int e = (int)(mag >> 7);
    const bool scaled = e > 16 && e < 255;
    const float f = scaled ? __uint_as_float((uint32_t)(127 + 135 - e) << 23) : 1.f;
#pragma unroll
    for (int k = 0; k < 4; ++k) u[k] = tc::pack_f16(bf_lo(u[k]) * f, bf_hi(u[k]) * f);
    v = make_uint4(u[0], u[1], u[2], u[3]);
    if (c == 0) smem_ptr[L::kQScale + scale_set * 128 + r] = (unsigned char)(scaled ? e : 0);
  }

  // The rows of a Q tile that a TMA copy has brought, to fp16 in place; QUAD: and into the other quarters.
  __device__ __forceinline__ void convert_q(int lane, int rows, int buf, int scale_set) const {
    constexpr int kQChunks = DP / 8, kStep = 32 / kQChunks, kBatch = 4;
    const int c = lane % kQChunks;
    const uint32_t base = smem + L::kQ0 + buf * L::kTile + (c >> 3) * kHalf;
    const int end = (rows + kStep * kBatch - 1) / (kStep * kBatch) * (kStep * kBatch);  // at most 128, QUAD 32
    for (int i0 = lane / kQChunks; i0 < end; i0 += kStep * kBatch) {
      uint4 v[kBatch];
#pragma unroll
      for (int b = 0; b < kBatch; ++b) {
        const int r = i0 + b * kStep;
        v[b] = ptx::lds128(base + r * 128 + (((c ^ r) & 7) << 4));
      }
#pragma unroll
      for (int b = 0; b < kBatch; ++b) {
        const int r = i0 + b * kStep;
        q_to_f16(v[b], r, c, scale_set);
#pragma unroll
        for (int k = 0; k < (QUAD ? 4 : 1); ++k)
          tc::sts128(base + (r + 32 * k) * 128 + (((c ^ r) & 7) << 4), v[b].x, v[b].y, v[b].z, v[b].w);
      }
    }
  }

  __device__ __forceinline__ void run_q(int tid, AttnWalk& walk) const {
    const uint32_t all = 0xffffffffu;
    if (!ONE && tid == 0) put_item(walk, 0);
    uint32_t qph = 0, qany = 0;  // bit w: phase of Q buffer w, and whether it was in use before
    int count = 0;
    AttnItem it;
    for (uint32_t n_item = 0; take_item(n_item, it); ++n_item) {
      const bool keys = it.j0 < it.j1;
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        const AttnTileRange r = attn_tile_range(P, it, ONE ? 0 : w);
        if (!keys || (ONE ? w != (count & 1) : r.a >= r.b)) continue;
        if (((qany >> w) & 1) && !__all_sync(all, wait(smem + L::kQEmpty + 8 * w, ((qph >> w) & 1) ^ 1))) {
          if (TMA) drain_q(qph, -1);
          return;
        }
        const int tok0 = it.tok0 + (ONE ? 0 : w * P.tok_per_tile), set = ONE ? count & 3 : w + 2 * ((qph >> w) & 1);
        const uint32_t q_full = smem + L::kQFull + 8 * w;
        if constexpr (TMA) {
          // the tile's tokens and heads as one box per 64 columns (QUAD: four times, unless they are written again anyway); tokens of
          // other sequences that come along stand in rows nobody looks at
          constexpr int kCopies = QUAD && !F8 ? 4 : 1;
          const uint32_t bar = F8 ? smem + L::kQRaw + 8 * w : q_full;
          if (tid == 0) {
            ptx::mbar_arrive_expect_tx(bar, (DP / 64) * kCopies * P.q_box_tokens * P.group * 128);
#pragma unroll
            for (int k = 0; k < kCopies; ++k)
#pragma unroll
              for (int h = 0; h < DP / 64; ++h)
                tc::tma3(smem + L::kQ0 + w * L::kTile + h * kHalf + k * 32 * 128, &maps.q, h * 64, it.kvh * P.group, it.s.row0 + tok0, bar);
          }
          if constexpr (F8) {
            if (!__all_sync(all, wait(bar, (qph >> w) & 1))) return drain_q(qph, w);
            convert_q(tid, r.rows, w, set);
            signal(q_full, tid);
          }
        } else {
          load_q(tid, it, tok0, r.rows, w, set);
          if (!F8) tc::cp_wait_all();
          signal(q_full, tid);
        }
        qph ^= 1u << w;
        qany |= 1u << w;
      }
      if (keys) ++count;
      if (!ONE && tid == 0) put_item(walk, n_item + 1);
      __syncwarp();
    }
    if (TMA && *abort_flag()) drain_q(qph, -1);
  }
  // Left early: the copies under way into the Q buffers have to land first.  qph: phases that have been asked for; open: a buffer
  // whose newest copy is not counted in it yet.
  __device__ __forceinline__ void drain_q(uint32_t qph, int open) const {
    for (int w = 0; w < 2; ++w) {
      const uint32_t bar = smem + (F8 ? L::kQRaw : L::kQFull) + 8 * w;
      wait_drain(bar, w == open ? (qph >> w) & 1 : ((qph >> w) & 1) ^ 1);
    }
  }

  // ---- tensor-core issue ----------------------------------------------------------------------------
  __device__ __forceinline__ void issue_qk(uint32_t tmem, int w, int qbuf, uint32_t pos) const {
    constexpr uint32_t idesc = tc::instr_desc(kAttnTile, F8, false);
    const uint32_t q = tc::desc_lo(smem + L::kQ0 + qbuf * L::kTile, 16), k = tc::desc_lo(stage(pos), 16);
#pragma unroll
    for (int s = 0; s < DP / 16; ++s) {  // 16 columns of head_dim: 32 bytes inside the 128-byte swizzle span
      tc::mma_ss(tmem + w * kAttnTile, q + (((s >> 2) * kHalf + (s & 3) * 32) >> 4), tc::desc_hi(1024), k + (((s >> 2) * 1024 + (s & 3) * 32) >> 4),
                 tc::desc_hi(kGroup), idesc, s > 0);
    }
    tc::commit(smem + L::kSFull + 8 * w);
  }
  // The first 96 keys' weights have been waited for (not QUAD); waits for the rest.
  __device__ __forceinline__ bool issue_pv(uint32_t tmem, int w, uint32_t pos, bool acc, uint32_t p_phase) const {
    constexpr uint32_t idesc = tc::instr_desc(DP, F8, true);
    const uint32_t v = tc::desc_lo(stage(pos), 1024);
    if (!QUAD) {
      tc::fence_after();
#pragma unroll
      for (int s = 0; s < 6; ++s)  // 16 keys: 8 TMEM columns of P, 16 rows of V
        tc::mma_ts(tmem + 2 * kAttnTile + w * DP, tmem + w * kAttnTile + s * 8, v + s * (2 * kGroup >> 4), tc::desc_hi(kGroup), idesc, acc || s > 0);
    }
    if (!wait(smem + L::kPFull + 8 * w, p_phase)) return false;
    tc::fence_after();
#pragma unroll
    for (int s = QUAD ? 0 : 6; s < kAttnTile / 16; ++s)
      tc::mma_ts(tmem + 2 * kAttnTile + w * DP, tmem + w * kAttnTile + s * 8, v + s * (2 * kGroup >> 4), tc::desc_hi(kGroup), idesc, acc || s > 0);
    return true;
  }

  // One query tile: one thread issues for both warpgroups.
  __device__ __forceinline__ void run_mma_one(uint32_t tmem) const {
    uint32_t pos = 0, count = 0;
    uint32_t qph = 0, pph = 0, oph = 0, oany = 0;  // bit w: phase of a barrier pair's w-th barrier; oany: O_w was in use before
    AttnItem it;
    for (uint32_t n_item = 0;; ++n_item) {
      if (!item_wait(n_item)) return;
      get_item(n_item, it);
      item_done(n_item);
      if (it.b < 0) return;
      if (it.j0 >= it.j1) continue;
      const int nt = it.j1 - it.j0;
      const int qb = count & 1;
      for (int r = -2; r < nt; ++r) {
        const int w = r & 1;
        if (r >= 0) {
          const uint32_t vp = pos + 2 * r + 1;
          if (!wait(full(vp), (vp / L::kStages) & 1)) return;
          if (r < 2 && ((oany >> w) & 1) && !wait(smem + L::kOFree + 8 * w, ((oph >> w) & 1) ^ 1)) return;
          if (!QUAD && !wait(smem + L::kPMost + 8 * w, (pph >> w) & 1)) return;
          if (!issue_pv(tmem, w, vp, r >= 2, (pph >> w) & 1)) return;
          pph ^= 1u << w;
          tc::commit(empty(vp));
          if (r + 2 >= nt) {
            tc::commit(smem + L::kOFull + 8 * w);
            oph ^= 1u << w;
            oany |= 1u << w;
          }
        }
        if (r + 2 < nt) {
          const uint32_t kp = pos + 2 * (r + 2);
          if (r == -2) {
            if (!wait(smem + L::kQFull + 8 * qb, (qph >> qb) & 1)) return;
            qph ^= 1u << qb;
          }
          if (!wait(full(kp), (kp / L::kStages) & 1)) return;
          tc::fence_after();
          issue_qk(tmem, w, qb, kp);
          tc::commit(empty(kp));
          if (r + 2 == nt - 1) tc::commit(smem + L::kQEmpty + 8 * qb);
        }
      }
      pos += 2 * nt;
      ++count;
    }
  }

  // Two query tiles: a thread for each (warps 12 and 15), issuing in turn.  The turns keep one warpgroup in its exponentials while
  // the other's products are made; if the products of the two interleaved, both would wait for them and then both compute
  // (measured at the time, 8192 tokens: 1024 us against 768).  Two threads, because what a thread does between products -- waiting for tiles and
  // weights, announcing what is done -- then lies beside the other's products and not between them.
  __device__ __forceinline__ void run_mma_two(uint32_t tmem, int w) const {
    uint32_t pos = 0, round = 0;
    uint32_t qph = 0, pph = 0, oph = 0, oany = 0;
    const uint32_t my_turn = smem + L::kTurn + 8 * w, your_turn = smem + L::kTurn + 8 * (w ^ 1);
    AttnItem it;
    for (uint32_t n_item = 0;; ++n_item) {
      if (!item_wait(n_item)) return;
      get_item(n_item, it);
      item_done(n_item);
      if (it.b < 0) return;
      if (it.j0 >= it.j1) continue;
      const AttnTileRange rg = attn_tile_range(P, it, w);
      for (int j = it.j0 - 1; j < it.j1; ++j, ++round) {
        // P V of tile j, Q K of tile j + 1; everything they need before the turn is taken
        const uint32_t kp = pos + 2 * (j + 1 - it.j0), vp = kp - 1;
        const bool pv = j >= rg.a && j < rg.b, qk = j + 1 >= rg.a && j + 1 < rg.b;
        if (j >= it.j0 && !wait(full(vp), (vp / L::kStages) & 1)) return;
        if (j + 1 < it.j1 && !wait(full(kp), (kp / L::kStages) & 1)) return;
        if (qk && j + 1 == rg.a) {
          if (!wait(smem + L::kQFull + 8 * w, qph)) return;
          qph ^= 1;
        }
        if (pv && j == rg.a && oany && !wait(smem + L::kOFree + 8 * w, oph ^ 1)) return;
        if (pv && !wait(smem + L::kPMost + 8 * w, pph)) return;
        if ((round > 0 || w == 1) && !wait(my_turn, w == 0 ? (round - 1) & 1 : round & 1)) return;
        tc::fence_after();
        if (pv) {
          if (!issue_pv(tmem, w, vp, j > rg.a, pph)) return;
          pph ^= 1;
        }
        if (qk) issue_qk(tmem, w, w, kp);
        tc::arrive(your_turn);
        if (pv && j == rg.b - 1) {
          tc::commit(smem + L::kOFull + 8 * w);
          oph ^= 1;
          oany = 1;
        }
        if (qk && j + 1 == rg.b - 1) tc::commit(smem + L::kQEmpty + 8 * w);
        if (j >= it.j0) tc::commit(empty(vp));
        if (j + 1 < it.j1) tc::commit(empty(kp));
      }
      pos += 2 * (it.j1 - it.j0);
    }
  }

  // c of this row's scores: an FP8 cache's Q rows had an exponent taken out
  __device__ __forceinline__ float row_c(int set, int row) const {
    const int e = reinterpret_cast<const volatile unsigned char*>(smem_ptr + L::kQScale)[set * 128 + row];
    return e == 0 ? P.c : fmaxf(ldexpf(P.c, e - 135), kAttnLeastC);
  }

  // ---- softmax --------------------------------------------------------------------------------------
  // O columns of this lane's row times f
  __device__ __forceinline__ void rescale(uint32_t o, float f) const {
#pragma unroll
    for (int k = 0; k < DP; k += 16) {
      uint32_t r[16];
      tc::ld16(o + k, r);
      tc::wait_ld();
#pragma unroll
      for (int e = 0; e < 16; ++e) r[e] = __float_as_uint(__uint_as_float(r[e]) * f);
      tc::st16(o + k, r);
    }
  }
  // Where a row's result goes: its place in out, or in the parts (place >= 0).
  struct Dest {
    long long row, place;
    int head;
  };
  __device__ __forceinline__ Dest dest(const AttnItem& it, int w, int in_tile) const {
    Dest d;
    d.row = it.s.row0 + (long long)(it.tok0 + w * P.tok_per_tile + in_tile / P.group);
    d.head = it.kvh * P.group + in_tile % P.group;
    d.place = it.whole ? -1 : ((long long)blockIdx.x * 2 + it.slot) * P.part_rows + w * kAttnTile + in_tile;
    return d;
  }
  // 32 columns of the result of a row
  __device__ __forceinline__ void store32(const float* x, const Dest& to, int col) const {
    if (to.place >= 0) {
      float* o = P.part_o + to.place * P.head_dim + col;
#pragma unroll
      for (int e = 0; e < 32; e += 4)
        if (col + e < P.head_dim) *reinterpret_cast<float4*>(o + e) = make_float4(x[e], x[e + 1], x[e + 2], x[e + 3]);
    } else {
      uint16_t* o = P.out + to.row * P.ld_out + (long long)to.head * P.head_dim + col;
#pragma unroll
      for (int e = 0; e < 32; e += 8)
        if (col + e < P.head_dim)
          *reinterpret_cast<uint4*>(o + e) = make_uint4(bf_pack(x[e], x[e + 1]), bf_pack(x[e + 2], x[e + 3]),
                                                        bf_pack(x[e + 4], x[e + 5]), bf_pack(x[e + 6], x[e + 7]));
    }
  }
  // N (4 or 8) columns of the result of a row
  template <int N>
  __device__ __forceinline__ void store_few(const float* x, const Dest& to, int col) const {
    if (col >= P.head_dim) return;  // head_dim is a multiple of 8, col of N
    if (to.place >= 0) {
      float* o = P.part_o + to.place * P.head_dim + col;
#pragma unroll
      for (int e = 0; e < N; e += 4) *reinterpret_cast<float4*>(o + e) = make_float4(x[e], x[e + 1], x[e + 2], x[e + 3]);
    } else {
      uint16_t* o = P.out + to.row * P.ld_out + (long long)to.head * P.head_dim + col;
#pragma unroll
      for (int e = 0; e < N; e += 4) *reinterpret_cast<uint2*>(o + e) = make_uint2(bf_pack(x[e], x[e + 1]), bf_pack(x[e + 2], x[e + 3]));
    }
  }
  __device__ __forceinline__ void store_z(float z, const Dest& to) const {
    if (to.place >= 0) P.part_z[to.place] = z;
    else if (P.lse != nullptr) P.lse[to.row * P.heads_q + to.head] = z * kLn2;
  }
  // Rows first, first + step, .. below end of query tile w again, one by one, each from the keys it sees and no others.
  __device__ __forceinline__ void redo(const AttnItem& it, int w, int first, int end, int step) const {
    const int lane = threadIdx.x & 31;
    const int tok0 = it.tok0 + w * P.tok_per_tile, rows = attn_tile_range(P, it, w).rows;
    for (int r = first; r < end && r < rows; r += step) {
      const int i = tok0 + r / P.group;
      const Dest to = dest(it, w, r);
      int lo = attn_lo(P, it.s, i), hi = attn_hi(P, it.s, i);
      lo = lo > it.j0 * kAttnTile ? lo : it.j0 * kAttnTile;
      hi = hi < it.j1 * kAttnTile ? hi : it.j1 * kAttnTile;
      float o[DP / 32], z;
      if (F8) attn_row<IoE4m3, DP / 32>(P, it.b, to.row, to.head, lo, hi, o, z, smem + L::kDeadline);
      else attn_row<IoBf16, DP / 32>(P, it.b, to.row, to.head, lo, hi, o, z, smem + L::kDeadline);
#pragma unroll
      for (int e = 0; e < DP / 32; ++e) {
        const int d = lane + 32 * e;
        if (d < P.head_dim) {
          if (to.place >= 0) P.part_o[to.place * P.head_dim + d] = o[e];
          else IoBf16::store(P.out, to.row * P.ld_out + (long long)to.head * P.head_dim + d, o[e] * P.v_scale);
        }
      }
      if (lane == 0) store_z(z, to);
    }
  }

  // One score tile: S -> P, running m and l of this lane's row.  QUAD: the 32 columns of this warp's quarter.
  // Columns [from, to) of the tile are keys that the row sees.
  // Not QUAD: the first 96 keys' weights are announced while the last 32 are computed, which takes about as long as the products
  // of the 96.  (8192 tokens: 726 us; announced after 64, when the products wait in their turn, 755.)
  __device__ __forceinline__ void tile(uint32_t s_addr, uint32_t o_addr, int from, int to, bool masked, bool first, float c, float& m,
                                       float& l, uint32_t p_most) const {
    // The first half stays in registers from the maximum to the exponentials; the second is read again when the first is half
    // done, so that a thread never holds more than 128 scores and nothing else.
    constexpr int N = QUAD ? kAttnTile / 4 : kAttnTile / 2;
    const int first_col = QUAD ? (int)((threadIdx.x >> 5) & 3) * N : 0;
    float s[N], t[QUAD ? 1 : N];
    auto mask = [&](float* x, int col) {
#pragma unroll
      for (int k = 0; k < N; ++k) x[k] = col + k >= from && col + k < to ? x[k] : kNegInf;
    };
#pragma unroll
    for (int k = 0; k < N; k += 32) tc::ld32(s_addr + first_col + k, reinterpret_cast<uint32_t*>(s) + k);
    if constexpr (!QUAD) {
#pragma unroll
      for (int k = 0; k < N; k += 32) tc::ld32(s_addr + N + k, reinterpret_cast<uint32_t*>(t) + k);
    }
    tc::wait_ld();
    if (masked) {
      mask(s, first_col);
      if constexpr (!QUAD) mask(t, N);
    }
    float mx[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) mx[e] = QUAD ? s[e] : fmaxf(s[e], t[e]);
#pragma unroll
    for (int k = 8; k < N; k += 8) {
#pragma unroll
      for (int e = 0; e < 8; ++e) mx[e] = QUAD ? fmaxf(mx[e], s[k + e]) : tc::max3(mx[e], s[k + e], t[QUAD ? 0 : k + e]);
    }
    const float mn = tc::max3(tc::max3(mx[0], mx[1], mx[2]), tc::max3(mx[3], mx[4], mx[5]), fmaxf(mx[6], mx[7]));
    // m is the maximum that the exponents are taken against; it follows the true one when that is 2^8 ahead
    const bool grow = mn > m && (m == kNegInf || (mn - m) * c > 8.f);
    if (__any_sync(0xffffffffu, grow)) {
      const float f = !grow ? 1.f : m == kNegInf ? 0.f : tc::ex2((m - mn) * c);
      if (grow) {
        l = m == kNegInf ? l : l * f;
        m = mn;
      }
      if (!first) rescale(o_addr, f);
    }
    const float mc = m == kNegInf ? 0.f : m * c - kUp;
    const float2 c2 = make_float2(c, c), mc2 = make_float2(-mc, -mc);
    float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
    auto weights = [&](const float* x, int col) {  // 32 columns from `col`
      uint32_t p[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        float2 y = __ffma2_rn(make_float2(x[2 * e], x[2 * e + 1]), c2, mc2);
        y.x = tc::ex2(y.x);
        y.y = tc::ex2(y.y);
        sum[e & 1] = __fadd2_rn(sum[e & 1], y);
        p[e] = F8 ? tc::pack_f16_sat(y.x, y.y) : bf_pack(y.x, y.y);
      }
      tc::st16(s_addr + col / 2, p);
    };
    weights(s, first_col);
    if constexpr (!QUAD) {
#pragma unroll
      for (int k = 0; k < N; k += 32) tc::ld32(s_addr + N + k, reinterpret_cast<uint32_t*>(t) + k);
      weights(s + 32, 32);
      tc::wait_ld();
      if (masked) mask(t, N);
      weights(t, 64);
      tc::wait_st();
      tc::fence_before();
      __syncwarp();
      if ((threadIdx.x & 31) == 0) tc::arrive(p_most);
      weights(t + 32, 96);
    }
    if (QUAD) {  // the other quarters' keys are not this warp's: zeros in their place
      uint32_t none[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) none[e] = 0u;
#pragma unroll
      for (int h = 1; h < 4; ++h) tc::st16(s_addr + ((first_col / 2 + h * 16) & 63), none);
    }
    l += (sum[0].x + sum[0].y) + (sum[1].x + sum[1].y);
    tc::wait_st();
    tc::fence_before();
  }

  __device__ __forceinline__ void run_softmax(uint32_t tmem, int w) const {
    const int lane = threadIdx.x & 31;
    const int wtid = QUAD ? lane : threadIdx.x & 127, first_row = wtid & ~31;  // this thread's row, its warp's first
    const uint32_t lanes = (threadIdx.x & 96) << 16;  // a warp reaches the 32 TMEM lanes of its place in the warpgroup
    uint32_t sph = 0, oph = 0, mlph = 0, ml_any = 0, pass = 0;
    int count = 0;
    const uint32_t all = 0xffffffffu;
    // The item stays in shared memory and is read again at its end: registers are for the scores.
    for (uint32_t n_item = 0;; ++n_item) {
      if (!__all_sync(all, item_wait(n_item))) return;
      float m = kNegInf, l = 0.f, c = P.c;
      {
        AttnItem it;
        get_item(n_item, it);
        if (it.b < 0) return;
        const AttnTileRange rg = attn_tile_range(P, it, ONE ? 0 : w);
        const int tok0 = it.tok0 + (ONE ? 0 : w * P.tok_per_tile);
        if (it.j0 < it.j1) {
          const int i = tok0 + wtid / P.group;
          const bool valid = wtid < rg.rows, busy = first_row < rg.rows;  // busy: some row of this warp is in use
          const int lo = valid ? attn_lo(P, it.s, i) : 0, hi = valid ? attn_hi(P, it.s, i) : 0;
          const int j_first = ONE ? it.j0 + w : rg.a, j_end = ONE ? it.j1 : rg.b;
          const int plain_from = rg.lo_max, plain_to = rg.hi_min;  // tiles inside [plain_from, plain_to) need no mask
#pragma unroll 1
          for (int j = j_first; j < j_end; j += ONE ? 2 : 1) {
            if (!__all_sync(all, wait(smem + L::kSFull + 8 * w, sph))) return;
            sph ^= 1;
            if (busy) {
              tc::fence_after();
              if (F8) c = row_c(ONE ? count & 3 : w + 2 * oph, wtid);
              const int k0 = j * kAttnTile;
              tile(tmem + lanes + w * kAttnTile, tmem + lanes + 2 * kAttnTile + w * DP, lo - k0, hi - k0,
                   k0 < plain_from || k0 + kAttnTile > plain_to, j == j_first, c, m, l, smem + L::kPMost + 8 * w);
            }
            __syncwarp();
            if (lane == 0) {
              if (!QUAD && !busy) tc::arrive(smem + L::kPMost + 8 * w);
              if ((j & 62) == 62) moving();
              tc::arrive(smem + L::kPFull + 8 * w);
            }
          }
        }
      }
      AttnItem it;
      get_item(n_item, it);
      const AttnTileRange rg = attn_tile_range(P, it, ONE ? 0 : w);
      const int tiles = it.j1 - it.j0;
      const bool valid = wtid < rg.rows, busy = first_row < rg.rows;
      const Dest to = dest(it, ONE ? 0 : w, wtid);
      const bool cut = to.place >= 0;
      if (!ONE) {
        const bool own = rg.a < rg.b;  // some tile of the item was this warpgroup's
        if (own) {
          if (!__all_sync(all, wait(smem + L::kOFull + 8 * w, oph))) return;
          oph ^= 1;
          tc::fence_after();
        }
        const bool again = tiles > 0 && poison()[count & 3] == count + 1;
        if (busy && !again) {
          const float inv = l == 0.f ? 0.f : (cut ? 1.f : P.v_scale) / l;
#pragma unroll
          for (int k = 0; k < DP; k += 32) {
            uint32_t o[32];
            float x[32];
            if (own) {
              tc::ld32(tmem + lanes + 2 * kAttnTile + w * DP + k, o);
              tc::wait_ld();
            }
#pragma unroll
            for (int e = 0; e < 32; ++e) x[e] = l == 0.f ? 0.f : __uint_as_float(o[e]) * inv;
            if (valid && !(cut && l == 0.f)) store32(x, to, k);
          }
          if (valid) store_z(l == 0.f ? kNegInf : m == kNegInf ? l : fmaf(m, c, log2f(l) - kUp), to);
        }
        if (again && busy) redo(it, w, first_row, first_row + 32, 1);
        if (own) {
          tc::fence_before();
          __syncwarp();
          if (lane == 0) tc::arrive(smem + L::kOFree + 8 * w);
        }
      } else if (tiles <= 0) {
        if (w == 0 && valid && (!QUAD || threadIdx.x < 32)) {
          float x[32];
#pragma unroll
          for (int e = 0; e < 32; ++e) x[e] = 0.f;
          for (int k = 0; k < DP; k += 32) store32(x, to, k);
          store_z(kNegInf, to);
        }
      } else {
        // the parts of the same rows: one per warpgroup, QUAD one per warp
        float2* ml = reinterpret_cast<float2*>(smem_ptr + L::kMlRows);
        const bool two = tiles > 1;
        if (ml_any && !__all_sync(all, wait(smem + L::kMlFree, mlph ^ 1))) return;
        ml[threadIdx.x] = make_float2(m, l);
        __syncwarp();
        if (lane == 0) tc::arrive(smem + L::kMl);
        if (!__all_sync(all, wait(smem + L::kMl, mlph))) return;
        constexpr int kParts = QUAD ? 8 : 2;
        float f[kParts], lp[kParts], mm = kNegInf;
#pragma unroll
        for (int p = 0; p < kParts; ++p) {
          const float2 v = ml[(QUAD ? 32 * p : 128 * p) + wtid];
          f[p] = v.x;
          lp[p] = v.y;
          mm = fmaxf(mm, v.x);
        }
        __syncwarp();
        if (lane == 0) tc::arrive(smem + L::kMlFree);
        mlph ^= 1;
        ml_any = 1;
        if (!__all_sync(all, wait(smem + L::kOFull, oph & 1))) return;
        oph ^= 1;
        if (two) {
          if (!__all_sync(all, wait(smem + L::kOFull + 8, oph >> 1))) return;
          oph ^= 2;
        }
        tc::fence_after();
        const bool again = poison()[count & 3] == count + 1;
        if (F8) c = row_c(count & 3, wtid);
        // a part without keys counts nothing; one that met only NaN scores makes the row NaN
        float lt = 0.f;
#pragma unroll
        for (int p = 0; p < kParts; ++p) {
          f[p] = f[p] == kNegInf ? (lp[p] != 0.f ? 1.f : 0.f) : tc::ex2((f[p] - mm) * c);
          lt = fmaf(f[p], lp[p], lt);
        }
        const float z = lt == 0.f ? kNegInf : mm == kNegInf ? lt : fmaf(mm, c, log2f(lt) - kUp);
        const float inv = lt == 0.f ? 0.f : (cut ? 1.f : P.v_scale) / lt;
        const bool put = valid && !(cut && lt == 0.f);
        const uint32_t o0 = tmem + lanes + 2 * kAttnTile, o1 = o0 + DP;
        if constexpr (QUAD) {
          // Two warps reach the same rows' quarter: each adds up both warpgroups' parts for half the columns.  The four quarters'
          // sums meet in the item's Q buffer, which is done with: kCols columns of each half at a time.
          constexpr int kCols = DP / 4, kMine = kCols / 4;  // kMine: columns this warp puts together, its lane's row
          static_assert(4 * 2 * kCols * 32 * 4 == L::kTile, "");
          const int part = threadIdx.x >> 5, quarter = part & 3;
          float* scratch = reinterpret_cast<float*>(smem_ptr + L::kQ0 + (count & 1) * L::kTile);
          float f0 = 0.f, f1 = 0.f;  // f[quarter], f[4 + quarter], without indexing registers
#pragma unroll
          for (int p = 0; p < 4; ++p) {
            f0 = p == quarter ? f[p] : f0;
            f1 = p == quarter && two ? f[4 + p] : f1;
          }
#pragma unroll 1
          for (int k = 0; k < 2; ++k) {
            const int col = w * (DP / 2) + k * kCols;
#pragma unroll 1  // small code: unrolled, the FP8 kernel's main loop lost 9 % to instruction fetches (214 us against 195)
            for (int q = 0; q < kCols; q += 16) {
              uint32_t a[16], b[16];
              tc::ld16(o0 + col + q, a);
              if (two) tc::ld16(o1 + col + q, b);
              tc::wait_ld();
#pragma unroll
              for (int e = 0; e < 16; ++e) {
                float x = f0 == 0.f ? 0.f : f0 * __uint_as_float(a[e]);
                if (f1 != 0.f) x = fmaf(f1, __uint_as_float(b[e]), x);
                scratch[((quarter * 2 + w) * kCols + q + e) * 32 + lane] = x;
              }
            }
            __syncwarp();
            if (lane == 0) tc::arrive(smem + L::kPass);
            if (!__all_sync(all, wait(smem + L::kPass, pass))) return;
            pass ^= 1;
            float x[kMine];
#pragma unroll
            for (int e = 0; e < kMine; ++e) {
              x[e] = 0.f;
#pragma unroll
              for (int p = 0; p < 4; ++p) x[e] += scratch[(p * 2 * kCols + part * kMine + e) * 32 + lane];
              x[e] *= inv;
            }
            if (put && !again) store_few<kMine>(x, to, col + quarter * kMine);
            if (k == 0) {  // the second round's sums go where these were
              __syncwarp();
              if (lane == 0) tc::arrive(smem + L::kPass);
              if (!__all_sync(all, wait(smem + L::kPass, pass))) return;
              pass ^= 1;
            }
          }
          ptx::fence_proxy_async();  // the buffer's next writer is a copy
          __syncwarp();
          if (lane == 0) tc::arrive(smem + L::kQEmpty + 8 * (count & 1));
          if (valid && part == 0 && !again) store_z(z, to);
          if (again) redo(it, 0, part, 32, 8);  // all eight warps have these rows
        } else {
          if (busy && !again) {
#pragma unroll
            for (int kk = 0; kk < DP / 2; kk += 32) {
              const int k = w * (DP / 2) + kk;
              uint32_t a[32], b[32];
              tc::ld32(o0 + k, a);
              if (two) tc::ld32(o1 + k, b);
              tc::wait_ld();
              float x[32];
#pragma unroll
              for (int e = 0; e < 32; ++e) {
                float v = f[0] == 0.f ? 0.f : f[0] * __uint_as_float(a[e]);
                if (two && f[1] != 0.f) v = fmaf(f[1], __uint_as_float(b[e]), v);
                x[e] = lt == 0.f ? 0.f : v * inv;
              }
              if (put) store32(x, to, k);
            }
            if (valid && w == 0) store_z(z, to);
          }
          if (again && busy) redo(it, 0, first_row + w, first_row + 32, 2);  // both warpgroups have them
        }
        tc::fence_before();
        __syncwarp();
        if (lane == 0) {
          tc::arrive(smem + L::kOFree);
          if (two) tc::arrive(smem + L::kOFree + 8);
        }
      }
      if (tiles > 0) ++count;
      __syncwarp();
      if (lane == 0) item_done(n_item);
    }
  }
};

template <int DP, bool F8, int FORM, bool TMA>
__global__ void __launch_bounds__(kAttnTcThreads, 1) attn_tc_kernel(const __grid_constant__ AttnParams P,
                                                                    const __grid_constant__ AttnMaps maps) {
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  using K = AttnTc<DP, F8, FORM, TMA>;
  using L = AttnSmem<DP, F8>;
  const uint32_t smem = ptx::smem_u32(smem_raw);
  const int warp = threadIdx.x >> 5;
  if (smem & 1023u) {  // the swizzle counts on it; no other shared memory is declared, so this does not happen
    if (threadIdx.x == 0) *P.error = 8;
    return;
  }
  if (threadIdx.x == 0) {
    for (int i = 0; i < L::kStages; ++i) {
      ptx::mbar_init(smem + L::kFull + 8 * i, 4);
      ptx::mbar_init(smem + L::kEmpty + 8 * i, K::ONE ? 1 : 2);
      ptx::mbar_init(smem + L::kRawFull + 8 * i, 1);
    }
    for (int i = 0; i < 2; ++i) {
      ptx::mbar_init(smem + L::kQFull + 8 * i, 1);
      ptx::mbar_init(smem + L::kQRaw + 8 * i, 1);
      ptx::mbar_init(smem + L::kTurn + 8 * i, 1);
      ptx::mbar_init(smem + L::kQEmpty + 8 * i, K::QUAD ? 9 : 1);
      ptx::mbar_init(smem + L::kSFull + 8 * i, 1);
      ptx::mbar_init(smem + L::kPFull + 8 * i, 4);
      ptx::mbar_init(smem + L::kPMost + 8 * i, 4);
      ptx::mbar_init(smem + L::kOFull + 8 * i, 1);
      ptx::mbar_init(smem + L::kOFree + 8 * i, K::ONE ? 8 : 4);
    }
    ptx::mbar_init(smem + L::kMl, 8);
    ptx::mbar_init(smem + L::kMlFree, 8);
    for (int i = 0; i < L::kItemSlots; ++i) {
      ptx::mbar_init(smem + L::kItemFull + 8 * i, 1);
      ptx::mbar_init(smem + L::kItemEmpty + 8 * i, K::kReaders);
    }
    ptx::mbar_init(smem + L::kDrain, K::ONE ? 1 : 2);
    ptx::mbar_init(smem + L::kPass, 8);
    *reinterpret_cast<volatile int*>(smem_raw + L::kAbort) = 0;
    for (int i = 0; i < 4; ++i) reinterpret_cast<volatile int*>(smem_raw + L::kPoison)[i] = 0;
    ptx::fence_barrier_init();
    ptx::fence_proxy_async();
  }
  if (warp == 12) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem + L::kTmem) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    tc::fence_before();
  }
  __syncthreads();
  tc::fence_after();
  const uint32_t tmem = *reinterpret_cast<const volatile uint32_t*>(smem_raw + L::kTmem);
  asm volatile("griddepcontrol.wait;" ::: "memory");

  AttnWalk walk(blockIdx.x, gridDim.x);
  // Whole units, one per sequence and key head: nothing to work out beforehand, which takes two microseconds.
  if (!K::ONE || P.starts != nullptr) {
    long long* scratch = reinterpret_cast<long long*>(smem_raw + L::kMlRows);  // nobody's yet
    AttnStart* start = reinterpret_cast<AttnStart*>(smem_raw + L::kMlRows + 512);
    attn_find_start(P, scratch, start);
    walk = AttnWalk(*start);
    __syncthreads();
  }
  walk.deadline = smem + L::kDeadline;
  const K k{P, maps, smem, smem_raw};
  // Every warp for itself: none of its lanes may look at the word before it holds a time.  (By every thread: 8 x 1000 keys 17.6 us
  // instead of 17.2, 64 x 8192 keys 236 instead of 233.)
  if ((threadIdx.x & 31) == 0) k.moving();
  __syncwarp();
  // 512 threads start with 128 registers each; 2 x 184 + 64 + 80 = 4 x 128
  if (warp < 8) {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 184;");
    k.run_softmax(tmem, warp >> 2);
  } else if (warp < 12) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
    if (TMA) k.run_workers(threadIdx.x - 256);
    else k.run_loader(threadIdx.x - 256);
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 80;");
    if (warp == 12 || (!K::ONE && warp == 15)) {
      if ((threadIdx.x & 31) == 0) {
        if (K::ONE) k.run_mma_one(tmem);
        else k.run_mma_two(tmem, warp == 12 ? 0 : 1);
        // every matrix product has ended before the tiles and TMEM go away, whichever way the loop ended
        tc::commit(smem + L::kDrain);
        k.wait_drain(smem + L::kDrain, 0);
      }
      __syncwarp();
    } else if (warp == 13) {
      if (TMA) k.run_producer(threadIdx.x & 31);
    } else if (warp == 14) {
      k.run_q(threadIdx.x & 31, walk);
    } else if (threadIdx.x == 480) {
      for (uint32_t i = 0; k.put_item(walk, i); ++i) {
      }
    }
  }
  tc::fence_before();
  __syncthreads();
  if (warp == 12) {
    tc::fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem));
  }
}

}  // namespace qknorm
