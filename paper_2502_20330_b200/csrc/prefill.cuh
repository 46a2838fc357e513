// Launchers of the position rotation (rope.cu) and of the attention of many new rows (attention_prefill.cu), called by the entry points.
#pragma once

#include "common.cuh"

namespace rapid {

int launch_rope_apply(const void* q, const rapid_kv_rows* q_rows, void* q_out, const rapid_kv_rows* q_out_rows, const void* k,
                      const rapid_kv_rows* k_rows, void* k_out, const rapid_kv_rows* k_out_rows, int B, int T, int Hq, int Hkv,
                      int D, const int32_t* positions, const rapid_rope* rope, int inverse, cudaStream_t stream);
// paged == nullptr: a contiguous cache
int launch_kv_append_rope(const void* q, const rapid_kv_rows* q_rows, const void* k_new, const void* v_new,
                          const rapid_kv_rows* rows, int T, const int32_t* n_tokens, void* q_out, void* k_cache, void* v_cache,
                          const rapid_paged_kv* paged, const int32_t* block_table, const int32_t* ctx_lens,
                          int32_t* ctx_lens_out, const rapid_rope* rope, const int32_t* positions,
                          const rapid_attn_shape* shape, int32_t* status_word, cudaStream_t stream);
size_t prefill_attention_workspace_bytes(const rapid_attn_shape* s, int T);
int launch_prefill_attention(const void* q, const rapid_kv_rows* q_rows, int T, const int32_t* n_tokens, const void* k_cache,
                             const void* v_cache, const rapid_paged_kv* paged, const int32_t* block_table,
                             const int32_t* ctx_lens, void* out, const rapid_attn_shape* shape,
                             const rapid_attn_params* params, void* workspace, size_t workspace_bytes, cudaStream_t stream);

}  // namespace rapid
