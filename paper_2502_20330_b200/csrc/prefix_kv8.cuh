// Launchers of the prefix attention (attention_prefix.cu) and of the FP8 cache (kv_fp8.cu), called by the entry points.
#pragma once

#include "common.cuh"

namespace rapid {

size_t prefix_attention_workspace_bytes(const rapid_attn_shape* s, int gamma);
// paged == nullptr: prefix K/V apart from the own caches; else both in the pools k_cache / v_cache
int launch_verify_attention_prefix(const void* q, const void* k_prefix, const void* v_prefix,
                                   const rapid_prefix_kv* prefix, const int32_t* prefix_len, const void* k_cache,
                                   const void* v_cache, const rapid_paged_kv* paged, const int32_t* block_table,
                                   const int32_t* ctx_lens, int gamma, void* out, const rapid_attn_shape* shape,
                                   const rapid_attn_params* params, void* workspace, size_t workspace_bytes,
                                   cudaStream_t stream);
size_t kv_fill_workspace_bytes(int B, int Hkv);
int launch_kv_fill_fp8(const void* k_new, const void* v_new, const rapid_kv_rows* rows, int T, const int32_t* n_tokens,
                       void* k_cache, void* v_cache, float* k_scale, float* v_scale, int32_t* ctx_lens_out, int headroom,
                       const rapid_attn_shape* shape, void* workspace, size_t workspace_bytes, cudaStream_t stream);
int launch_kv_append_fp8(const void* k_new, const void* v_new, const rapid_kv_rows* rows, void* k_cache, void* v_cache,
                         const float* k_scale, const float* v_scale, const int32_t* ctx_lens, int32_t* ctx_lens_out,
                         int gamma, const rapid_attn_shape* shape, int32_t* status_word, cudaStream_t stream);
int launch_kv_read_fp8(const void* k_cache, const void* v_cache, const float* k_scale, const float* v_scale,
                       const int32_t* ctx_lens, const rapid_attn_shape* shape, const int32_t* chunk_idx, int n_chunks,
                       int chunk_tokens, void* k_out, void* v_out, const rapid_attn_shape* out_shape, int32_t* out_lens,
                       int32_t* status_word, cudaStream_t stream);

}  // namespace rapid
