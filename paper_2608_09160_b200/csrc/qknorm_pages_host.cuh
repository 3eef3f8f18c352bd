// Host side of the entry points of include/qknorm_pages.h: validation and launch.
// Included by qknorm_api.cu INSIDE its unnamed namespace, after qknorm_attn_host.cuh.
#pragma once

// What every call says of the cache's books.
struct PageBooks {
  Region regions[8];
  bool written[8];
  int n = 0;
  void add(const void* p, int64_t bytes, bool writes) {
    if (!p || bytes <= 0) return;
    written[n] = writes;
    regions[n++] = flat(p, (uintptr_t)bytes);
  }
};

int check_pools(const qknorm_page_pool* pools, int32_t num_pools, int64_t num_pages) {
  if (num_pools < 0 || num_pools > QKNORM_MAX_POOLS || num_pages < 1 || num_pages > 0x7fffffff) return QKNORM_ERR_SHAPE;
  if (num_pools > 0 && !pools) return QKNORM_ERR_NULL;
  for (int i = 0; i < num_pools; ++i) {
    const qknorm_page_pool& p = pools[i];
    if (!p.base) return QKNORM_ERR_NULL;
    if (p.page < 0 || p.count[0] < 1 || p.count[1] < 1 || p.count[0] > 0x7fffffff || p.count[1] > 0x7fffffff || p.stride[0] < 0 || p.stride[1] < 0 ||
        p.bytes < 1)
      return QKNORM_ERR_SHAPE;
    // the three axes, from the shortest stride to the longest: nothing in the place of anything else
    int64_t n[3] = {num_pages, p.count[0], p.count[1]}, stride[3] = {p.page, p.stride[0], p.stride[1]};
    for (int a = 0; a < 3; ++a)
      for (int b = a + 1; b < 3; ++b)
        if (stride[b] < stride[a]) {
          const int64_t s = stride[a], m = n[a];
          stride[a] = stride[b], n[a] = n[b];
          stride[b] = s, n[b] = m;
        }
    __int128 inside = p.bytes;
    for (int a = 0; a < 3; ++a) {
      if (n[a] == 1) continue;
      if (stride[a] < inside) return QKNORM_ERR_SHAPE;
      inside += (__int128)(n[a] - 1) * stride[a];
    }
    if (inside > ((__int128)1 << 60)) return QKNORM_ERR_SHAPE;
  }
  return QKNORM_OK;
}

uintptr_t pool_extent(const qknorm_page_pool& p, int64_t num_pages) {
  return (uintptr_t)((num_pages - 1) * p.page + (p.count[0] - 1) * p.stride[0] + (p.count[1] - 1) * p.stride[1] + p.bytes);
}

// The small arrays may overlap neither one another, unless both are only read, nor a pool's pages.
int check_books(const PageBooks& b, const qknorm_page_pool* pools, int num_pools, int64_t num_pages) {
  for (int i = 0; i < b.n; ++i) {
    for (int j = 0; j < i; ++j)
      if ((b.written[i] || b.written[j]) && may_overlap(b.regions[i], b.regions[j])) return QKNORM_ERR_ALIAS;
    for (int k = 0; k < num_pools; ++k)
      if (may_overlap(b.regions[i], flat(pools[k].base, pool_extent(pools[k], num_pages)))) return QKNORM_ERR_ALIAS;
  }
  return QKNORM_OK;
}

// Sizes and pointers of table, lens and refs.
int check_tables(const void* refs, const void* table, int32_t cols, int64_t ld, const void* lens, int32_t rows, int32_t page_size, PageParams& P) {
  if (cols < 0 || ld < 0 || (ld != 0 && ld < cols) || rows < 0 || page_size < 1) return QKNORM_ERR_SHAPE;
  P.cols = cols;
  P.ld = ld ? ld : cols;
  P.rows = rows;
  P.page_size = page_size;
  if (!refs || (rows > 0 && (!lens || (cols > 0 && !table)))) return QKNORM_ERR_NULL;
  if (((uintptr_t)refs | (uintptr_t)table | (uintptr_t)lens) & 3u) return QKNORM_ERR_ALIGN;
  P.refs = (int*)const_cast<void*>(refs);
  P.table = (int*)const_cast<void*>(table);
  P.lens = (int*)const_cast<void*>(lens);
  return QKNORM_OK;
}

void book_tables(const PageParams& P, PageBooks& b, bool writes_table, bool writes_lens) {
  b.add(P.refs, 4 * P.num_pages, true);
  if (P.rows > 0 && P.cols > 0) b.add(P.table, 4 * ((int64_t)(P.rows - 1) * P.ld + P.cols), writes_table);
  b.add(P.lens, 4 * (int64_t)P.rows, writes_lens);
}

int64_t pages_workspace_ints(int64_t num_pages, int64_t rows, int64_t n) {
  const int64_t fork = rows + 4 * n, compact = 2 * (num_pages / 2 + 1) + num_pages + 4;
  return (fork > compact ? fork : compact) + 3;
}

int run_pages_workspace(int64_t num_pages, int32_t rows, int32_t n, int64_t* bytes) {
  if (!bytes) return QKNORM_ERR_NULL;
  if (num_pages < 1 || num_pages > 0x7fffffff || rows < 0 || n < 0) return QKNORM_ERR_SHAPE;
  *bytes = (4 * pages_workspace_ints(num_pages, rows, n) + 15) / 16 * 16;
  return QKNORM_OK;
}

int check_pages_workspace(const PageParams& P, int n, void* ws, int64_t ws_bytes, const qknorm_page_pool* pools, int num_pools, const PageBooks& b) {
  int64_t need = 0;
  const int rc = run_pages_workspace(P.num_pages, P.rows, n, &need);
  if (rc != QKNORM_OK) return rc;
  if (!ws || ws_bytes < need || !aligned16(ws)) return QKNORM_ERR_SCRATCH;
  const Region w = flat(ws, (uintptr_t)need);
  for (int i = 0; i < b.n; ++i)
    if (may_overlap(w, b.regions[i])) return QKNORM_ERR_SCRATCH;
  for (int k = 0; k < num_pools; ++k)
    if (may_overlap(w, flat(pools[k].base, pool_extent(pools[k], P.num_pages)))) return QKNORM_ERR_SCRATCH;
  return QKNORM_OK;
}

// Moves the pairs' pages, pairs: their number, or at most; the first launch keeps the books.
int launch_moves(const PageParams& P, const qknorm_page_pool* pools, int num_pools, int64_t pairs, cudaStream_t stream) {
  const DeviceInfo* dev = nullptr;
  int rc = current_device(&dev);
  if (rc != QKNORM_OK) return rc;
  MoveParams M;
  M.P = P;
  for (int k0 = 0; k0 == 0 || k0 < num_pools; k0 += kPagePools) {
    M.pools = num_pools - k0 < kPagePools ? num_pools - k0 : kPagePools;
    int64_t most = 1;  // items of a pool
    for (int k = 0; k < M.pools; ++k) {
      const qknorm_page_pool& p = pools[k0 + k];
      PagePool& q = M.pool[k];
      q.base = (char*)p.base;
      q.page = p.page;
      q.stride0 = p.stride[0];
      q.stride1 = p.stride[1];
      q.bytes = p.bytes;
      q.pieces = p.count[0] * p.count[1];
      q.count1 = (int)p.count[1];
      const uintptr_t all = (uintptr_t)p.base | (uintptr_t)p.page | (uintptr_t)(p.count[0] > 1 ? p.stride[0] : 0) |
                            (uintptr_t)(p.count[1] > 1 ? p.stride[1] : 0) | (uintptr_t)p.bytes;
      q.unit = all % 16 == 0 ? 16 : all % 4 == 0 ? 4 : 1;
      const __int128 items = (__int128)q.pieces * ((p.bytes + kPageChunk - 1) / kPageChunk) * pairs;
      most = items > most ? (items < 0x7fffffff ? (int64_t)items : 0x7fffffff) : most;
    }
    // eight CTAs for every SM, shared between the pools
    int64_t x = (8 * (int64_t)dev->sm_count + M.pools - 1) / (M.pools > 0 ? M.pools : 1);
    const int64_t books = M.P.books == 1 ? P.n : M.P.books == 2 ? P.rows : 0;
    if (most < books) most = books;
    if (x > most) x = most;
    const cudaError_t e = launch_overlapped(pages_move_kernel_for(), dim3((unsigned)x, (unsigned)(M.pools + (M.P.books ? 1 : 0))),
                                            (unsigned)kPageThreads, 0, stream, M);
    if (e != cudaSuccess) return set_cuda_error(e);
    if ((rc = finish_launch("pages")) != QKNORM_OK) return rc;
    M.P.books = 0;
  }
  return QKNORM_OK;
}

int run_pages_copy(const qknorm_page_pool* pools, int32_t num_pools, int64_t num_pages, const int32_t* src, const int32_t* dst, int32_t n,
                   cudaStream_t stream) {
  int rc = check_pools(pools, num_pools, num_pages);
  if (rc != QKNORM_OK) return rc;
  if (n < 0) return QKNORM_ERR_SHAPE;
  if (n == 0 || num_pools == 0) return QKNORM_OK;
  if (!src || !dst) return QKNORM_ERR_NULL;
  if (((uintptr_t)src | (uintptr_t)dst) & 3u) return QKNORM_ERR_ALIGN;
  for (int k = 0; k < num_pools; ++k) {
    const Region p = flat(pools[k].base, pool_extent(pools[k], num_pages));
    if (may_overlap(p, flat(src, 4 * (uintptr_t)n)) || may_overlap(p, flat(dst, 4 * (uintptr_t)n))) return QKNORM_ERR_ALIAS;
  }
  PageParams P;
  memset(&P, 0, sizeof(P));
  P.num_pages = num_pages;
  P.from = src;
  P.to = dst;
  P.n = n;
  return launch_moves(P, pools, num_pools, n, stream);
}

int run_pages_fork(const qknorm_page_pool* pools, int32_t num_pools, int64_t num_pages, int32_t* refs, int32_t* table, int32_t cols, int64_t ld,
                   int32_t* lens, int32_t rows, int32_t page_size, const int32_t* parents, const int32_t* children, int32_t n, int32_t* ok,
                   void* ws, int64_t ws_bytes, cudaStream_t stream) {
  int rc = check_pools(pools, num_pools, num_pages);
  if (rc != QKNORM_OK) return rc;
  PageParams P;
  memset(&P, 0, sizeof(P));
  P.num_pages = num_pages;
  if ((rc = check_tables(refs, table, cols, ld, lens, rows, page_size, P)) != QKNORM_OK) return rc;
  if (n < 0) return QKNORM_ERR_SHAPE;
  if (n == 0) return QKNORM_OK;
  if (!parents || !children) return QKNORM_ERR_NULL;
  if (((uintptr_t)parents | (uintptr_t)children | (uintptr_t)ok) & 3u) return QKNORM_ERR_ALIGN;
  PageBooks b;
  book_tables(P, b, true, true);
  b.add(parents, 4 * (int64_t)n, false);
  b.add(children, 4 * (int64_t)n, false);
  b.add(ok, 4 * (int64_t)n, true);
  if ((rc = check_books(b, pools, num_pools, num_pages)) != QKNORM_OK) return rc;
  if ((rc = check_pages_workspace(P, n, ws, ws_bytes, pools, num_pools, b)) != QKNORM_OK) return rc;
  P.parents = parents;
  P.children = children;
  P.n = n;
  P.ok = ok;
  P.src = (int*)ws;
  P.dst = P.src + n;
  P.len = P.dst + n;
  P.free_page = P.len + n;
  P.claim = P.free_page + n;
  const cudaError_t e = launch_overlapped(pages_kernel_for(kPagesForkPlan), 1, (unsigned)kPlanThreads, 0, stream, P);
  if (e != cudaSuccess) return set_cuda_error(e);
  if ((rc = finish_launch("pages")) != QKNORM_OK) return rc;
  P.from = P.src;
  P.to = P.dst;
  P.books = 1;
  return launch_moves(P, pools, num_pools, n, stream);
}

int run_pages_free(int32_t* refs, int64_t num_pages, const int32_t* table, int32_t cols, int64_t ld, int32_t* lens, int32_t rows,
                   int32_t page_size, const int32_t* list, int32_t n, cudaStream_t stream) {
  if (num_pages < 1 || num_pages > 0x7fffffff) return QKNORM_ERR_SHAPE;
  PageParams P;
  memset(&P, 0, sizeof(P));
  P.num_pages = num_pages;
  int rc = check_tables(refs, table, cols, ld, lens, rows, page_size, P);
  if (rc != QKNORM_OK) return rc;
  if (n < 0) return QKNORM_ERR_SHAPE;
  if (n == 0) return QKNORM_OK;
  if (!list) return QKNORM_ERR_NULL;
  if ((uintptr_t)list & 3u) return QKNORM_ERR_ALIGN;
  PageBooks b;
  book_tables(P, b, false, true);
  b.add(list, 4 * (int64_t)n, false);
  if ((rc = check_books(b, nullptr, 0, num_pages)) != QKNORM_OK) return rc;
  P.children = list;
  P.n = n;
  const cudaError_t e = launch_overlapped(pages_kernel_for(kPagesFree), (unsigned)n, (unsigned)kPageThreads, 0, stream, P);
  if (e != cudaSuccess) return set_cuda_error(e);
  return finish_launch("pages");
}

int run_pages_compact(const qknorm_page_pool* pools, int32_t num_pools, int64_t num_pages, int32_t* refs, int32_t* table, int32_t cols, int64_t ld,
                      const int32_t* lens, int32_t rows, int32_t page_size, int32_t* live, void* ws, int64_t ws_bytes, cudaStream_t stream) {
  int rc = check_pools(pools, num_pools, num_pages);
  if (rc != QKNORM_OK) return rc;
  PageParams P;
  memset(&P, 0, sizeof(P));
  P.num_pages = num_pages;
  if ((rc = check_tables(refs, table, cols, ld, lens, rows, page_size, P)) != QKNORM_OK) return rc;
  if (!live) return QKNORM_ERR_NULL;
  if ((uintptr_t)live & 3u) return QKNORM_ERR_ALIGN;
  PageBooks b;
  book_tables(P, b, true, false);
  b.add(live, 4, true);
  if ((rc = check_books(b, pools, num_pools, num_pages)) != QKNORM_OK) return rc;
  if ((rc = check_pages_workspace(P, 0, ws, ws_bytes, pools, num_pools, b)) != QKNORM_OK) return rc;
  const int64_t half = num_pages / 2 + 1;
  P.live = live;
  P.src = (int*)ws;
  P.dst = P.src + half;
  P.map = P.dst + half;
  P.count = P.map + num_pages;
  const cudaError_t e = launch_overlapped(pages_kernel_for(kPagesCompactPlan), (unsigned)kPlanCluster, (unsigned)kPlanThreads, 0, stream, P);
  if (e != cudaSuccess) return set_cuda_error(e);
  if ((rc = finish_launch("pages")) != QKNORM_OK) return rc;
  P.from = P.src;
  P.to = P.dst;
  P.n_device = P.count;
  P.books = 2;
  return launch_moves(P, pools, num_pools, num_pages / 2, stream);
}
