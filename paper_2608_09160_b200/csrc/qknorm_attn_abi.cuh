// The extern "C" entry points of include/qknorm_attn.h.  Included by qknorm_api.cu at file scope.
#pragma once

extern "C" {

int qknorm_rope_frequencies(int32_t rot_dim, double theta, int32_t scaling, double factor, double original_len,
                            double low, double high, double* inv_freq, float* mscale) {
  return qknorm::rope_frequencies(rot_dim, theta, scaling, factor, original_len, low, high, inv_freq, mscale);
}

int qknorm_rope(const void* q, const void* k, const qknorm_rotation* rot, int64_t tokens, int32_t dq, int32_t dk,
                int32_t head_dim, int64_t ld_q, int64_t ld_k, int32_t inverse, void* out_q, void* out_k,
                int64_t ld_out_q, int64_t ld_out_k, void* stream) {
  return qknorm::run_rope(2, q, k, rot, tokens, dq, dk, head_dim, ld_q, ld_k, inverse, out_q, out_k, ld_out_q, ld_out_k,
                          (cudaStream_t)stream);
}

int qknorm_rope_e4m3(const void* q, const void* k, const qknorm_rotation* rot, int64_t tokens, int32_t dq, int32_t dk,
                     int32_t head_dim, int64_t ld_q, int64_t ld_k, int32_t inverse, void* out_q, void* out_k,
                     int64_t ld_out_q, int64_t ld_out_k, void* stream) {
  return qknorm::run_rope(1, q, k, rot, tokens, dq, dk, head_dim, ld_q, ld_k, inverse, out_q, out_k, ld_out_q, ld_out_k,
                          (cudaStream_t)stream);
}

int qknorm_rope_axes(const void* q, const void* k, const qknorm_rotation_axes* rot, int64_t tokens, int32_t dq, int32_t dk,
                     int32_t head_dim, int64_t ld_q, int64_t ld_k, int32_t inverse, void* out_q, void* out_k,
                     int64_t ld_out_q, int64_t ld_out_k, void* stream) {
  return qknorm::run_rope(2, q, k, rot, tokens, dq, dk, head_dim, ld_q, ld_k, inverse, out_q, out_k, ld_out_q, ld_out_k,
                          (cudaStream_t)stream);
}

int qknorm_rope_axes_e4m3(const void* q, const void* k, const qknorm_rotation_axes* rot, int64_t tokens, int32_t dq,
                          int32_t dk, int32_t head_dim, int64_t ld_q, int64_t ld_k, int32_t inverse, void* out_q,
                          void* out_k, int64_t ld_out_q, int64_t ld_out_k, void* stream) {
  return qknorm::run_rope(1, q, k, rot, tokens, dq, dk, head_dim, ld_q, ld_k, inverse, out_q, out_k, ld_out_q, ld_out_k,
                          (cudaStream_t)stream);
}

int qknorm_fwd_append_axes(const void* q, const void* k, const void* v, const void* gamma_q, const void* gamma_k,
                           int32_t norm, float eps, const qknorm_rotation_axes* rot, const int64_t* slots,
                           const qknorm_paged_cache* cache, int64_t tokens, int32_t dq, int64_t ld_q, int64_t ld_k,
                           int64_t ld_v, void* out_q, int64_t ld_out_q, void* stream) {
  return qknorm::run_append(q, k, v, gamma_q, gamma_k, norm, eps, rot, slots, cache, tokens, dq, ld_q, ld_k, ld_v, out_q,
                            ld_out_q, (cudaStream_t)stream);
}

int qknorm_fwd_append_e2m1(const void* q, const void* k, const void* v, const void* gamma_q, const void* gamma_k,
                           int32_t norm, float eps, const qknorm_rotation_axes* rot, const int64_t* slots,
                           const qknorm_paged_cache_e2m1* cache, int64_t tokens, int32_t dq, int64_t ld_q, int64_t ld_k,
                           int64_t ld_v, void* out_q, int64_t ld_out_q, void* stream) {
  return qknorm::run_append(q, k, v, gamma_q, gamma_k, norm, eps, rot, slots, cache, tokens, dq, ld_q, ld_k, ld_v, out_q,
                            ld_out_q, (cudaStream_t)stream);
}

int qknorm_attn_paged_e2m1(const void* q, int64_t ld_q, const qknorm_paged_cache_e2m1* cache, const int32_t* block_table,
                           int32_t table_cols, int64_t ld_table, const int32_t* kv_lens, const int32_t* q_starts,
                           int32_t num_seqs, int64_t tokens, int32_t max_q, int32_t max_kv, int32_t heads_q, float scale,
                           int32_t causal, int32_t window, void* out, int64_t ld_out, float* lse, void* workspace,
                           int64_t workspace_bytes, void* stream) {
  return qknorm::run_attn_e2m1(q, ld_q, cache, block_table, table_cols, ld_table, kv_lens, q_starts, num_seqs, tokens, max_q,
                               max_kv, heads_q, scale, causal, window, out, ld_out, lse, workspace, workspace_bytes,
                               (cudaStream_t)stream);
}

int qknorm_attn_paged_e2m1_workspace(int32_t num_seqs, int64_t tokens, int32_t max_q, int32_t max_kv, int32_t heads_q,
                                     int32_t heads_kv, int32_t head_dim, int32_t window, int64_t* bytes) {
  return qknorm::run_attn_e2m1_workspace(num_seqs, tokens, max_q, max_kv, heads_q, heads_kv, head_dim, window, bytes);
}

int qknorm_fwd_append(const void* q, const void* k, const void* v, const void* gamma_q, const void* gamma_k,
                      int32_t norm, float eps, const qknorm_rotation* rot, const int64_t* slots,
                      const qknorm_paged_cache* cache, int64_t tokens, int32_t dq, int64_t ld_q, int64_t ld_k,
                      int64_t ld_v, void* out_q, int64_t ld_out_q, void* stream) {
  return qknorm::run_append(q, k, v, gamma_q, gamma_k, norm, eps, rot, slots, cache, tokens, dq, ld_q, ld_k, ld_v, out_q,
                            ld_out_q, (cudaStream_t)stream);
}

int qknorm_attn_paged(const void* q, int64_t ld_q, const qknorm_paged_cache* cache, const int32_t* block_table,
                      int32_t table_cols, int64_t ld_table, const int32_t* kv_lens, const int32_t* q_starts,
                      int32_t num_seqs, int64_t tokens, int32_t max_q, int32_t max_kv, int32_t heads_q, float scale,
                      int32_t causal, int32_t window, void* out, int64_t ld_out, float* lse, void* workspace,
                      int64_t workspace_bytes, void* stream) {
  return qknorm::run_attn(q, ld_q, cache, block_table, table_cols, ld_table, kv_lens, q_starts, num_seqs, tokens, max_q,
                          max_kv, heads_q, scale, causal, window, out, ld_out, lse, workspace, workspace_bytes,
                          (cudaStream_t)stream);
}

int qknorm_attn_paged_workspace(int32_t num_seqs, int64_t tokens, int32_t max_q, int32_t max_kv, int32_t heads_q,
                                int32_t heads_kv, int32_t head_dim, int32_t window, int64_t* bytes) {
  return qknorm::run_attn_workspace(num_seqs, tokens, max_q, max_kv, heads_q, heads_kv, head_dim, window, bytes);
}

}  // extern "C"
