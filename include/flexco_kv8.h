/*
 * flexco, 8-bit paged KV cache.  C ABI, beside flexco.h and with its conventions: status codes and
 * flexco_last_error, the caller owns all memory, nothing is allocated and nothing synchronised, every argument is checked on
 * the host before anything is launched.
 *
 * The cache of Sec. 7 (pages of page_size positions, a sequence's pages in any order) with one byte per element instead of
 * the activations' two or four: decode attention reads little else, and a pool holds twice the sequences beside the
 * finetuning job.  An element is code x scale: the code an 8-bit float with 4 exponent and 3 mantissa bits (e4m3: largest 448,
 * no infinities, NaN = 0x7f and 0xff), the scale a power of two for each (page, kv head), of K and of V each, held as a float
 * (other positive numbers in its place give results without meaning).
 *
 * What flexco_kv8_append writes: the scale of a page is 2^e with e >= -117 the least that keeps its elements within 448 (code x scale
 * is then exact in bf16, and a scale that grows later costs codes no second rounding but below the type's smallest normal
 * number).  Elements that are no finite number are stored as NaN and take no part in a scale.  Finite ones beyond 1.875 x 2^127 are stored as
 * that, off by less than 2^-4: under the largest scale, 2^120, the next number is an infinity in the activations' types.
 */
#ifndef FLEXCO_KV8_H
#define FLEXCO_KV8_H

#include "flexco.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Version of this header's ABI (increases when a struct below changes or an entry point is added).  flexco_abi_version is that
 * of flexco.h, which this header leaves as it is. */
int32_t flexco_kv8_abi_version(void);

/* One layer's 8-bit cache (device).  head_dim d is a multiple of 16.
 *   k_codes [num_pages, nkv, d / 16, page_size, 16]   keys after RoPE: pieces of 16 channels, those of all positions together
 *   v_codes [num_pages, nkv, d, page_size]            values, position-minor inside a page
 *   k_scale, v_scale [num_pages, nkv]
 * codes 16-byte aligned, scales 4-byte aligned.  The scale of a page no position has been written to is never read. */
typedef struct flexco_kv8_pool {
  uint8_t* k_codes;
  uint8_t* v_codes;
  float*   k_scale;
  float*   v_scale;
  int32_t  num_pages;
  int32_t  page_size;
} flexco_kv8_pool;

/* The runs of a batch: its tokens by the page they are written to (one scale is chosen per run and head).  host_maps: as filled by
 * flexco_build_maps, arrays in host memory.  runs (host): pairs (first token, number of tokens), batch order, room for
 * `capacity` pairs (host_maps->T always suffices); *n_runs = pairs written.  Host only.
 * Errors: EINVAL, EPAGE (two runs write into one page: its scale would be chosen twice), EWORKSPACE (capacity, or no host memory). */
int32_t flexco_kv8_runs(const flexco_maps* host_maps, int32_t* runs, int32_t capacity, int32_t* n_runs);

/* Append of the batch's tokens (Alg. 2: Append): queries and keys are rotated to their positions, keys and values written to
 * their slots.
 *   maps  : device-rebased maps of the batch;  runs: device, the n_runs pairs of flexco_kv8_runs for these maps (a run
 *           outside the batch, e.g. (-1, 0) in a place left free, or reaching past its page is left out)
 *   qkv   : device [T, (nq + 2 nkv) d], rows of query, key and value heads before rotation, dtype of cfg
 *   q_out : device, T rows of nq d elements, ld_q elements apart: the rotated queries.  q_out may be qkv with ld_q its row length
 *           (rotation in place; keys and values are left as they are); else the two may not overlap.
 * A run that begins its page begins the page's scale, and what the page's other slots held is lost; any other run keeps the scale
 * or raises it, and then rounds the codes of all the page's other slots to the new one.
 * Reads of cfg: n_q_heads, n_kv_heads, head_dim, dtype, page_size, rope_theta.
 * Errors: EINVAL, ESHAPE (head_dim no multiple of 16), EPAGE (maps of a larger pool), EUNSUPPORTED (a token's kv heads take more LDS
 * than a block has, 8 head_dim + n_kv_heads (head_dim + 16) > 49152; more than 2^24 runs x kv heads), EHIP. */
int32_t flexco_kv8_append(const flexco_layer_cfg* cfg, const flexco_maps* maps, const int32_t* runs, int32_t n_runs,
                          const void* qkv, const flexco_kv8_pool* pool, void* q_out, size_t ld_q, void* stream);

/* flexco_attention_mixed over an 8-bit pool: every token attends to positions 0 .. own position of its sequence; q, out, lse and
 * ws as there (flexco_workspace_bytes covers it).  Key positions behind a token's own never reach its row, whatever
 * they hold.  lse may be NULL.
 * Gradients: flexco_kv8_expand the sequence's pages, then flexco_attention_window_bwd (flexco_lora_bwd) on that pool: the keys and
 * values are bit for bit those this call read (the rounding into the cache counts as the identity).
 * Errors: EINVAL, ESHAPE, EPAGE, EWORKSPACE, EHIP. */
int32_t flexco_kv8_attention(const flexco_layer_cfg* cfg, const flexco_maps* maps, const void* q, const flexco_kv8_pool* pool,
                             void* out, float* lse, void* ws, size_t ws_bytes, void* stream);

/* A sequence's pages written out in the dtype of cfg: positions [0, n_tokens) of the sequence that holds src_pages in pool go to the
 * pages dst_pages of wide (layout of flexco.h); the slots behind them in the last page are written as zeros.  src_pages,
 * dst_pages: device int32 [ceil(n_tokens / page_size)]; a pair with an id outside its pool is left out, no page may be
 * written twice in a call.  The two pools may differ in their number of pages, not in page_size.
 * Errors: EINVAL, ESHAPE, EUNSUPPORTED (more than 2^24 pages x kv heads), EHIP. */
int32_t flexco_kv8_expand(const flexco_layer_cfg* cfg, const flexco_kv8_pool* pool, const int32_t* src_pages, int32_t n_tokens,
                          const flexco_kv_pool* wide, const int32_t* dst_pages, void* stream);

/* flexco_layer_forward over an 8-bit pool: flexco_kv8_append (of all the batch's runs) and flexco_kv8_attention in place of the 16-bit
 * steps, everything else - arguments, the finetune window's saved rows, workspace - as there.  What flexco_kv8_append refuses is
 * refused here, before anything is launched.  A later flexco_lora_bwd of the window takes a pool that
 * flexco_kv8_expand has filled with the sequence's pages. */
int32_t flexco_kv8_layer_forward(const flexco_layer_cfg* cfg, const flexco_base_weights* w, const flexco_lora* lora,
                                 const flexco_maps* maps, const int32_t* runs, int32_t n_runs, const void* x_in, void* x_out,
                                 const flexco_kv8_pool* pool, const flexco_ft_state* ft, void* ws, size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* FLEXCO_KV8_H */
