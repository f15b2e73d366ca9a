// Launchers of the 8-bit cache's kernels (no validation, the entry points have done it).
#pragma once
#include "flexco_internal.h"
#include "flexco_kv8.h"

namespace flexco {

// LDS of the block that takes a single token, all kv heads of it: angles, largest magnitudes and old scales, codes of the values
constexpr size_t KV8_APPEND_LDS = 48 * 1024;
inline size_t kv8_append_token_lds(const flexco_layer_cfg& c) {
  return sizeof(double) * c.head_dim + (size_t)c.n_kv_heads * (4 * sizeof(uint32_t) + c.head_dim);
}

// q_cache: NULL, or where the finetune window's rotated queries go as well (its first row's)
int32_t launch_kv8_append(const flexco_layer_cfg& c, const flexco_maps& m, const int32_t* runs, int n_runs, const void* qkv,
                          const flexco_kv8_pool& pool, void* q_out, size_t ld_q, void* q_cache, hipStream_t s);
int32_t launch_kv8_expand(const flexco_layer_cfg& c, const flexco_kv8_pool& pool, const int32_t* src, int n_tokens,
                          const flexco_kv_pool& wide, const int32_t* dst, hipStream_t s);
// partial rows as the 16-bit kernels leave them (attn_generic.hip), for launch_kv8_merge
int32_t launch_kv8_attention_generic(const flexco_layer_cfg& c, const flexco_maps& m, const void* q, size_t ldq,
                                     const flexco_kv8_pool& pool, float* part_ml, float* part_acc, void* out, size_t ldo, float* lse,
                                     hipStream_t s, const AttnKeep* keep);

// joins partial rows where a request was cut (fold: splits taken as one, of requests of one token)
int32_t launch_kv8_merge(const flexco_layer_cfg& c, const flexco_maps& m, const float* part_ml, const float* part_acc, void* out, size_t ldo,
                         float* lse, hipStream_t s, int fold, const AttnKeep* keep);

// (with the joining of partial rows) bf16, head_dim 128, page_size 16, at most 16 query heads per kv head; otherwise FLEXCO_EUNSUPPORTED without launching
int32_t launch_kv8_attention_mfma(const flexco_layer_cfg& c, const flexco_maps& m, const void* q, size_t ldq, const flexco_kv8_pool& pool,
                                  float* part_ml, float* part_acc, void* out, size_t ldo, float* lse, hipStream_t s,
                                  const AttnKeep* keep);

}  // namespace flexco
