// The extern "C" entry points of include/qknorm_pages.h.  Included by qknorm_api.cu at file scope.
#pragma once

extern "C" {

int qknorm_pages_copy(const qknorm_page_pool* pools, int32_t num_pools, int64_t num_pages, const int32_t* src,
                      const int32_t* dst, int32_t n, void* stream) {
  return qknorm::run_pages_copy(pools, num_pools, num_pages, src, dst, n, (cudaStream_t)stream);
}

int qknorm_pages_fork(const qknorm_page_pool* pools, int32_t num_pools, int64_t num_pages, int32_t* refs, int32_t* table,
                      int32_t table_cols, int64_t ld_table, int32_t* lens, int32_t rows, int32_t page_size,
                      const int32_t* parents, const int32_t* children, int32_t n, int32_t* ok, void* workspace,
                      int64_t workspace_bytes, void* stream) {
  return qknorm::run_pages_fork(pools, num_pools, num_pages, refs, table, table_cols, ld_table, lens, rows, page_size, parents,
                                children, n, ok, workspace, workspace_bytes, (cudaStream_t)stream);
}

int qknorm_pages_free(int32_t* refs, int64_t num_pages, const int32_t* table, int32_t table_cols, int64_t ld_table,
                      int32_t* lens, int32_t rows, int32_t page_size, const int32_t* list, int32_t n, void* stream) {
  return qknorm::run_pages_free(refs, num_pages, table, table_cols, ld_table, lens, rows, page_size, list, n,
                                (cudaStream_t)stream);
}

int qknorm_pages_compact(const qknorm_page_pool* pools, int32_t num_pools, int64_t num_pages, int32_t* refs, int32_t* table,
                         int32_t table_cols, int64_t ld_table, const int32_t* lens, int32_t rows, int32_t page_size,
                         int32_t* live, void* workspace, int64_t workspace_bytes, void* stream) {
  return qknorm::run_pages_compact(pools, num_pools, num_pages, refs, table, table_cols, ld_table, lens, rows, page_size, live,
                                   workspace, workspace_bytes, (cudaStream_t)stream);
}

int qknorm_pages_workspace(int64_t num_pages, int32_t rows, int32_t n, int64_t* bytes) {
  return qknorm::run_pages_workspace(num_pages, rows, n, bytes);
}

}  // extern "C"
