/*
 * libqknorm -- from the normalised Q and K to the attention output: rotary positions, the write of K
 * and V into a paged cache (fused with the norm and the rotation), attention over that cache.
 *
 * QK-Norm sits between the projection and attention (Section II-A of the paper); these are the
 * steps that follow it in every layer.  Conventions are those of qknorm.h: device pointers, the
 * caller owns every buffer, work is enqueued on `stream` without synchronising, a qknorm_status
 * comes back, nothing is launched on an error, calls may be captured into CUDA graphs and may run
 * at the same time on different streams (each attention call with a workspace of its own).
 * Arithmetic is fp32 (angles: fp64), every result is rounded once to its storage format, to nearest even
 * (FP8-E4M3: saturating at +-448); the matrix products of attention take rounded softmax weights, see
 * qknorm_attn_paged.  Results are bitwise reproducible run to run, except where two
 * tokens of one call name the same cache slot (each value there is then one of theirs).
 *
 * Rows are tokens: q is [tokens, dq] with dq = heads * head_dim, row t starts ld_q ELEMENTS after
 * row t-1 (0 = contiguous), so q, k and v may be column blocks of one fused projection output.
 *
 * Device-side integers (positions, slots, tables, lengths) are read by the kernels and cannot be
 * checked on the host; each entry point says what an out-of-range value does.  None of them makes
 * a kernel read or write outside the buffers of the call.
 */
#ifndef QKNORM_ATTN_H_
#define QKNORM_ATTN_H_

#include "qknorm.h"

#ifdef __cplusplus
extern "C" {
#endif

#define QKNORM_MAX_HEAD_DIM 512      /* largest head_dim of the entry points below */
#define QKNORM_MAX_KEYS 0x7fffff00   /* largest max_kv of qknorm_attn_paged */
#define QKNORM_MAX_HEAD_DIM_E2M1 256 /* largest head_dim of a 4-bit cache */
#define QKNORM_MAX_AXES 8            /* largest num_axes of a rotation with several axes */

/* How the frequencies of qknorm_rope_frequencies are scaled for contexts longer than trained on. */
typedef enum {
  QKNORM_ROPE_PLAIN = 0,  /* theta^(-2i/rot_dim) */
  QKNORM_ROPE_LINEAR = 1, /* every frequency / factor */
  QKNORM_ROPE_BASE = 2,   /* theta * factor^(rot_dim/(rot_dim-2)): the slowest pair slows by `factor`, the fastest stays */
  QKNORM_ROPE_RAMP = 3,   /* by turns within original_len: >= high keeps, <= low is divided by factor, a ramp linear in the
                             pair's index between; mscale = 0.1 ln(factor) + 1 (YaRN) */
  QKNORM_ROPE_BANDS = 4   /* by turns within original_len: >= high keeps, <= low is divided by factor, interpolated
                             linearly in the number of turns between */
} qknorm_rope_scaling;

/*
 * qknorm_rope_frequencies -- HOST helper: radians per position of the rot_dim/2 pairs.
 *   inv_freq [rot_dim/2] doubles, HOST, written; copy it to the device for the calls below
 *   mscale   HOST, written: the factor that goes with the scaling (1 unless QKNORM_ROPE_RAMP)
 *   factor >= 1, original_len > 0 and 0 < low < high are looked at only by the scalings that use them.
 * rot_dim odd, < 2 or > QKNORM_MAX_HEAD_DIM, theta <= 1 (or NaN), an unknown scaling or a bad parameter is QKNORM_ERR_SHAPE.
 */
int qknorm_rope_frequencies(int32_t rot_dim, double theta, int32_t scaling, double factor, double original_len,
                            double low, double high, double* inv_freq, float* mscale);

/* A rotation: pair i of every head turns by positions[t] * inv_freq[i] and is multiplied by mscale.
 * The first rot_dim columns of a head rotate, the others pass through unchanged. */
typedef struct {
  const int64_t* positions; /* [tokens], device; any value, negative too */
  const double* inv_freq;   /* [rot_dim/2], device: radians per position */
  int32_t rot_dim;          /* even, 0 .. head_dim; 0 = no rotation (the pointers are ignored) */
  int32_t interleaved;      /* 0: pairs (i, i + rot_dim/2); 1: pairs (2i, 2i+1) */
  float mscale;             /* 1 unless the frequencies are scaled in a way that asks for it */
} qknorm_rotation;

/*
 * qknorm_rope -- rotary positions on Q and K.
 *   out[a] = (x[a] cos - x[b] sin) * mscale,  out[b] = (x[b] cos + x[a] sin) * mscale  for every pair (a, b)
 *   inverse = 1 turns the other way.  The rotation is orthogonal, so that is its backward pass: given
 *   dL/dout it returns dL/dx (mscale included), with the same positions.
 *   q [tokens, dq], k [tokens, dk] bf16 (qknorm_rope_e4m3: FP8-E4M3); out_* may be exactly its own input.
 *   dq == 0 or dk == 0 skips that tensor.
 * The angle is formed in fp64 and reduced to one turn before cos and sin are taken, so it is as exact at
 * position 10^6 as at 1.  Vectorised for 16-byte aligned rows (E4M3: 8-byte) with head_dim and rot_dim multiples of
 * 16; anything else takes a general kernel.
 */
int qknorm_rope(const void* q, const void* k, const qknorm_rotation* rot, int64_t tokens, int32_t dq, int32_t dk,
                int32_t head_dim, int64_t ld_q, int64_t ld_k, int32_t inverse, void* out_q, void* out_k,
                int64_t ld_out_q, int64_t ld_out_k, void* stream);
int qknorm_rope_e4m3(const void* q, const void* k, const qknorm_rotation* rot, int64_t tokens, int32_t dq, int32_t dk,
                     int32_t head_dim, int64_t ld_q, int64_t ld_k, int32_t inverse, void* out_q, void* out_k,
                     int64_t ld_out_q, int64_t ld_out_k, void* stream);

/*
 * A paged cache: pools of num_pages pages, a page holds page_size tokens, a token heads * head_dim
 * values.  Element (page, token, head, d) of K is at k[page*k_page + token*k_token + head*k_head + d], likewise V, in
 * ELEMENTS: any order of the axes, K and V in one buffer or in two, with gaps or between one another (if one lies in the other's
 * gaps, qknorm_fwd_append asks for the same strides of both; unlike ones are QKNORM_ERR_ALIAS).
 * e4m3 = 0: bf16.  e4m3 = 1: FP8-E4M3 that stands for stored * k_scale (v_scale); the scales are ignored for bf16.
 */
typedef struct {
  void* k;
  void* v;
  int64_t k_page, k_token, k_head;
  int64_t v_page, v_token, v_head;
  int64_t num_pages;
  int32_t page_size;
  int32_t heads;
  int32_t head_dim;
  int32_t e4m3;
  float k_scale, v_scale;
} qknorm_paged_cache;

typedef enum {
  QKNORM_NORM_NONE = 0,      /* gammas and eps ignored */
  QKNORM_NORM_LAYERWISE = 1, /* one factor per token and tensor, as qknorm_fwd */
  QKNORM_NORM_HEADWISE = 2   /* one factor per head, as qknorm_fwd_headwise */
} qknorm_norm;

/*
 * qknorm_fwd_append -- norm, rotation and cache write in one pass over the projection's output:
 *   q: normalised, rotated, written to out_q;  k: normalised, rotated, written to its cache slot;
 *   v: written to its cache slot as it is.
 *   q [tokens, dq], k and v [tokens, cache->heads * head_dim] bf16, row strides ld_* elements (0 = contiguous)
 *   gamma_q [dq], gamma_k [heads * head_dim] bf16     rot may be NULL (no rotation)
 *   slots [tokens] int64, device: page * page_size + token inside the page.  A slot outside
 *   [0, num_pages * page_size), -1 for instance, writes nothing to the cache (a padded token); its q row is written.
 *   out_q [tokens, dq] bf16; may be exactly q.  dq == 0: no q.
 * Nothing is rounded between the steps: norm, rotation and division by the cache's scale (as a
 * product with its fp32 reciprocal, which has to be finite) are fp32.
 */
int qknorm_fwd_append(const void* q, const void* k, const void* v, const void* gamma_q, const void* gamma_k,
                      int32_t norm, float eps, const qknorm_rotation* rot, const int64_t* slots,
                      const qknorm_paged_cache* cache, int64_t tokens, int32_t dq, int64_t ld_q, int64_t ld_k,
                      int64_t ld_v, void* out_q, int64_t ld_out_q, void* stream);

/*
 * qknorm_attn_paged -- attention of the batch's new tokens over the paged cache.
 *   Sequence b has its new tokens in rows q_starts[b] .. q_starts[b+1]-1 of q (n of them) and kv_lens[b] keys in
 *   the cache, the new tokens' own among them (append first).  Row i of the sequence stands at position
 *   kv_lens[b] - n + i.  It sees key j (0 <= j < kv_lens[b]) if
 *       causal == 0 or j <= position,   and   window == 0 or j > position - window.
 *   out[row, h] = sum_j p_j v_j,  p = softmax over the keys it sees of scale * q[row, h] . k_j,
 *   with key head h / (heads_q / cache->heads).  A row that sees no key gets zeros and lse = -inf.
 *
 *   q, out       [tokens, heads_q * head_dim] bf16, row strides ld_q, ld_out elements (0 = contiguous)
 *   block_table  [num_seqs, table_cols] int32, device, rows ld_table elements apart (0 = table_cols): page of keys
 *                j*page_size .. of the sequence.  Only entries up to the last visible key are read.  An entry outside
 *                [0, num_pages) stands for a page of zeros.
 *   kv_lens [num_seqs], q_starts [num_seqs+1]: int32, device.  q_starts ascends within 0..tokens.
 *   max_q, max_kv: upper bounds of a sequence's new tokens and keys.  They choose the launch shape; new
 *                tokens past max_q are left out, keys past min(max_kv, table_cols * page_size) are not seen.
 *   lse          [tokens, heads_q] fp32 or NULL: log(sum_j exp(scale q.k_j))
 *   workspace    device, 16-byte aligned, at least qknorm_attn_paged_workspace(...) bytes; its contents mean nothing
 *                between calls.  Two calls that may run at the same time need one each.
 *   out and lse may not overlap any other buffer of the call.  scale > 0; scale (times k_scale) times log2(e) has to fit
 *   fp32 (QKNORM_ERR_SHAPE), and so have the scores times it, which is not checked.
 *   Rows of out and lse outside every sequence are not written, and such rows of q do not matter.
 *   Keys, values that a row does not see have no influence on it, whatever they hold (NaN and infinities too);
 *   a row whose every visible score is -inf gets zeros.  An infinite value that a row does see makes that element infinite or NaN.
 *
 * Kernels: "attn_tc" (tcgen05 tensor cores) for head_dim a multiple of 8 up to 128, 16-byte aligned rows and at most 128 query
 * heads per key head; "attn_general" otherwise.  The batch's key tiles are shared out evenly over the SMs; where that can cut
 * the keys of a row in two or more, the parts lie in the workspace and a second launch joins them (otherwise no workspace
 * is asked for).  A wait inside "attn_tc" that runs out -- two seconds in which nothing else in its CTA moved -- sets the device's error
 * word (qknorm_device_error_word): 7 a tile or a product did not come, 9 a copy did not land before the CTA ended; 8: shared memory is not
 * aligned.  Rows that are done again because a tile holds a value that they must not see take about 1.2 us a key, up to 32 rows in turn.
 *
 * Rounding in "attn_tc": scores, maxima, sums and the accumulated output are fp32.  The weights are rounded for the product with V: to
 * bf16 (half a step: 2^-8 relative) over a bf16 cache, to fp16 over an FP8 one (2^-11 relative, and at least 2^-32 of the row's largest weight).
 * Over an FP8 cache the queries are brought to fp16, a power of two taken out of each row first: exact but for parts below 2^-30 of
 * the row's largest element.  "attn_general" rounds neither.  In "attn_tc" a row whose scores (times log2(e)) pass 2^22 tells those apart that differ by more
 * than a few fp32 steps; closer ones share the weight.
 */
int qknorm_attn_paged(const void* q, int64_t ld_q, const qknorm_paged_cache* cache, const int32_t* block_table,
                      int32_t table_cols, int64_t ld_table, const int32_t* kv_lens, const int32_t* q_starts,
                      int32_t num_seqs, int64_t tokens, int32_t max_q, int32_t max_kv, int32_t heads_q, float scale,
                      int32_t causal, int32_t window, void* out, int64_t ld_out, float* lse, void* workspace,
                      int64_t workspace_bytes, void* stream);

/* Bytes of workspace that a call of these sizes needs on the current device, causal or not (0 is possible); HOST, written. */
int qknorm_attn_paged_workspace(int32_t num_seqs, int64_t tokens, int32_t max_q, int32_t max_kv, int32_t heads_q,
                                int32_t heads_kv, int32_t head_dim, int32_t window, int64_t* bytes);

/*
 * Rotary positions with several axes: images and video place a token by time, height and width at once, and every
 * pair of a head turns by one of them.  Pair i turns by positions[axis[i]][t] * inv_freq[i]; all else is as in qknorm_rotation.
 */
typedef struct {
  const int64_t* positions; /* [num_axes][tokens], device, an axis' positions ld_positions elements after the last's */
  int64_t ld_positions;     /* 0 = tokens */
  const double* inv_freq;   /* [rot_dim/2], device */
  const uint8_t* axis;      /* [rot_dim/2], device; a pair whose axis is num_axes or more stands at position 0.  NULL: axis 0 for all */
  int32_t num_axes;         /* 1 .. QKNORM_MAX_AXES */
  int32_t rot_dim;          /* even, 0 .. head_dim; 0 = no rotation (the pointers are ignored) */
  int32_t interleaved;
  float mscale;
} qknorm_rotation_axes;

/* qknorm_rope, qknorm_rope_e4m3 and qknorm_fwd_append with such a rotation (inverse = 1 is the backward pass here too). */
int qknorm_rope_axes(const void* q, const void* k, const qknorm_rotation_axes* rot, int64_t tokens, int32_t dq, int32_t dk,
                     int32_t head_dim, int64_t ld_q, int64_t ld_k, int32_t inverse, void* out_q, void* out_k,
                     int64_t ld_out_q, int64_t ld_out_k, void* stream);
int qknorm_rope_axes_e4m3(const void* q, const void* k, const qknorm_rotation_axes* rot, int64_t tokens, int32_t dq,
                          int32_t dk, int32_t head_dim, int64_t ld_q, int64_t ld_k, int32_t inverse, void* out_q,
                          void* out_k, int64_t ld_out_q, int64_t ld_out_k, void* stream);
int qknorm_fwd_append_axes(const void* q, const void* k, const void* v, const void* gamma_q, const void* gamma_k,
                           int32_t norm, float eps, const qknorm_rotation_axes* rot, const int64_t* slots,
                           const qknorm_paged_cache* cache, int64_t tokens, int32_t dq, int64_t ld_q, int64_t ld_k,
                           int64_t ld_v, void* out_q, int64_t ld_out_q, void* stream);

/*
 * A paged cache in 4 bits.  16 consecutive elements of a head are a block: sixteen E2M1 codes (sign, two exponent bits,
 * one of mantissa: 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives) and one E4M3 scale; an element of K stands for
 * code * scale * k_scale.  k and v hold head_dim/2 bytes per token and head, element 2i in the low four bits of byte i;
 * k_scales and v_scales head_dim/16 bytes.  All strides are in BYTES; any order of the axes, with gaps, as in qknorm_paged_cache.
 *   head_dim: a multiple of 16 up to QKNORM_MAX_HEAD_DIM_E2M1.
 *   k and v with their strides: multiples of 8 bytes (of 16 for the faster copies, head_dim a multiple of 32 then).
 *   k_scales and v_scales with theirs: multiples of the largest power of two up to 8 that divides head_dim/16.
 * Fastest to read: a head's tokens one after the other in a page (k_token = head_dim/2, ks_token = head_dim/16), head_dim 64 or 128,
 * pages of a multiple of 8 tokens, addresses and the other strides multiples of 16 bytes.
 */
typedef struct {
  void* k;
  void* v;
  void* k_scales;
  void* v_scales;
  int64_t k_page, k_token, k_head;
  int64_t v_page, v_token, v_head;
  int64_t ks_page, ks_token, ks_head;
  int64_t vs_page, vs_token, vs_head;
  int64_t num_pages;
  int32_t page_size;
  int32_t heads;
  int32_t head_dim;
  float k_scale, v_scale;
} qknorm_paged_cache_e2m1;

/*
 * qknorm_fwd_append_e2m1 -- qknorm_fwd_append into a 4-bit cache; rot may be NULL.
 * With y = x / k_scale (as a product with the fp32 reciprocal, which has to be finite) a block's scale is
 * f = max |y| / 6 (the correctly rounded quotient) rounded to E4M3, nearest even, saturating at 448; a code is y / f (the correctly rounded quotient) rounded to
 * E2M1, nearest even, saturating at +-6.  f = 0 (a block of zeros, or too small for E4M3) gives codes of zero.  A block with a NaN gets
 * the scale NaN and reads back as NaN; infinities saturate.  Two tokens of a call that name the same slot leave codes and scales of either.
 */
int qknorm_fwd_append_e2m1(const void* q, const void* k, const void* v, const void* gamma_q, const void* gamma_k,
                           int32_t norm, float eps, const qknorm_rotation_axes* rot, const int64_t* slots,
                           const qknorm_paged_cache_e2m1* cache, int64_t tokens, int32_t dq, int64_t ld_q, int64_t ld_k,
                           int64_t ld_v, void* out_q, int64_t ld_out_q, void* stream);

/*
 * qknorm_attn_paged_e2m1 -- qknorm_attn_paged over a 4-bit cache: the same arguments, the same rows, keys, masks and refusals.
 * k_scale and v_scale are taken as they stand.  K and V widen exactly; scores, maxima, sums and the output are fp32; the
 * weights are rounded to fp16 (2^-11 relative, at least 2^-32 of the row's largest weight), whichever kernel runs.  "attn_e2m1" brings queries to fp16
 * with a power of two taken out of each row (exact but for parts below 2^-30 of the row's largest element).
 *
 * Kernels: "attn_e2m1" (mma.sync out of registers) for up to 96 rows (max_q times the query heads of a key head) per sequence; for more the
 * visible part of the cache is widened once into the workspace, K to bf16 and V to fp16, and "attn_tc" reads that -- where rows of q and out
 * are 16-byte aligned, head_dim is at most 128 and the widened cache, 4 bytes an element of max_kv keys of every sequence (with a window, too),
 * at most 2 GB.  A wait
 * inside "attn_e2m1" that runs out after a second sets the device's error word to 10.
 */
int qknorm_attn_paged_e2m1(const void* q, int64_t ld_q, const qknorm_paged_cache_e2m1* cache, const int32_t* block_table,
                           int32_t table_cols, int64_t ld_table, const int32_t* kv_lens, const int32_t* q_starts,
                           int32_t num_seqs, int64_t tokens, int32_t max_q, int32_t max_kv, int32_t heads_q, float scale,
                           int32_t causal, int32_t window, void* out, int64_t ld_out, float* lse, void* workspace,
                           int64_t workspace_bytes, void* stream);

/* Bytes of workspace that a call of these sizes needs on the current device (0 is possible); HOST, written. */
int qknorm_attn_paged_e2m1_workspace(int32_t num_seqs, int64_t tokens, int32_t max_q, int32_t max_kv, int32_t heads_q,
                                     int32_t heads_kv, int32_t head_dim, int32_t window, int64_t* bytes);

#ifdef __cplusplus
}
#endif
#endif /* QKNORM_ATTN_H_ */
