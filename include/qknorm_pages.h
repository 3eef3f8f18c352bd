/*
 * libqknorm -- the life of a paged cache's pages: copying, forking a sequence, freeing, compacting.
 *
 * Conventions are those of qknorm.h and qknorm_attn.h: device pointers, the caller owns every buffer, work is enqueued on
 * `stream` without synchronising, a qknorm_status comes back, nothing is launched on an error, calls may be captured into
 * CUDA graphs.  Results do not depend on the order in which threads run.
 *
 * A cache is described by what attention reads, and one array more:
 *   table [rows, table_cols] int32, rows ld_table elements apart (0 = table_cols): the pages of each row's sequence
 *   lens  [rows] int32: its tokens.  Row r holds the first ceil(lens[r] / page_size) entries of its table row (table_cols at most)
 *   refs  [num_pages] int32: how many rows hold the page; a page with none (0 or less) is free.  A page that a row is given by other
 *         means has to be counted there.
 * Calls that change these arrays, or pages, and calls that read them have to be ordered, on one stream or by events.
 *
 * Device-side integers cannot be checked on the host: rows and pages outside their ranges are passed over, as each entry point
 * says.  None of them makes a kernel read or write outside the buffers of the call.
 */
#ifndef QKNORM_PAGES_H_
#define QKNORM_PAGES_H_

#include "qknorm.h"

#ifdef __cplusplus
extern "C" {
#endif

#define QKNORM_MAX_POOLS 1024  /* largest num_pools */

/*
 * Where pages lie: page p is count[0] x count[1] pieces of `bytes` bytes, piece (i, j) at base + p*page + i*stride[0] + j*stride[1].
 * One pool can be K or V of one layer, or all layers of a cache in one buffer.  Strides are in BYTES and not negative; the pieces of a
 * call's pools must not share bytes.  Fastest where everything is a multiple of 16.
 */
typedef struct {
  void* base;
  int64_t page;
  int64_t count[2], stride[2];
  int64_t bytes;
} qknorm_page_pool;

/*
 * qknorm_pages_copy -- page src[i] to page dst[i] in every pool, i < n.
 *   pools  HOST array of num_pools, read during the call
 *   src, dst [n] int32, device.  A pair with a page outside [0, num_pages), or of a page with itself, copies nothing.
 *   A page named in dst twice, or in dst and in src of another pair, ends up with bytes of either.
 */
int qknorm_pages_copy(const qknorm_page_pool* pools, int32_t num_pools, int64_t num_pages, const int32_t* src,
                      const int32_t* dst, int32_t n, void* stream);

/*
 * qknorm_pages_fork -- row children[i] becomes a copy of row parents[i] that can grow by itself: it shares the parent's full
 * pages (their refs go up by one) and gets a copy of its last page if that is not full, in the free page with the lowest number that
 * no fork before it in the call has taken.  Table entries behind the last page become -1.
 *   parents, children [n] int32, device.  A fork is left out, changing nothing, if one of its rows is outside [0, rows), if the child
 *   holds anything (lens[child] != 0; free it first), is its own parent or was named by an earlier fork of the call, if the
 *   parent's tokens need more than table_cols entries, or if it needs a page and none is left.  Parents are taken as they were before the call.
 *   ok [n] int32, device or NULL: 1 for a fork that was made, 0 for one left out
 *   workspace: device, 16-byte aligned, qknorm_pages_workspace(num_pages, rows, n) bytes; its contents mean nothing between calls.
 */
int qknorm_pages_fork(const qknorm_page_pool* pools, int32_t num_pools, int64_t num_pages, int32_t* refs, int32_t* table,
                      int32_t table_cols, int64_t ld_table, int32_t* lens, int32_t rows, int32_t page_size,
                      const int32_t* parents, const int32_t* children, int32_t n, int32_t* ok, void* workspace,
                      int64_t workspace_bytes, void* stream);

/*
 * qknorm_pages_free -- rows list[i] give up their pages (refs go down by one) and their length becomes 0; the table stays as it is.
 *   list [n] int32, device; rows outside [0, rows) are passed over, a row named twice is freed once.
 */
int qknorm_pages_free(int32_t* refs, int64_t num_pages, const int32_t* table, int32_t table_cols, int64_t ld_table,
                      int32_t* lens, int32_t rows, int32_t page_size, const int32_t* list, int32_t n, void* stream);

/*
 * qknorm_pages_compact -- the held pages move together at the pool's start: with `live` pages held, the k-th held page at or behind
 * number `live` goes to the k-th free one before it.  Its contents are copied in every pool, its refs move along, and every entry that a
 * row holds follows.  What the freed pages behind contain does not change.
 *   live [1] int32, device, written: the number of pages held, all below it now
 *   workspace as above, with n = 0.
 */
int qknorm_pages_compact(const qknorm_page_pool* pools, int32_t num_pools, int64_t num_pages, int32_t* refs, int32_t* table,
                         int32_t table_cols, int64_t ld_table, const int32_t* lens, int32_t rows, int32_t page_size,
                         int32_t* live, void* workspace, int64_t workspace_bytes, void* stream);

/* Bytes of workspace of qknorm_pages_fork (n forks) and qknorm_pages_compact (n = 0); HOST, written. */
int qknorm_pages_workspace(int64_t num_pages, int32_t rows, int32_t n, int64_t* bytes);

#ifdef __cplusplus
}
#endif
#endif /* QKNORM_PAGES_H_ */
