// Attention over the 8-bit cache for any type, head size, page size and grouping (fp32 activations, and bf16 shapes that the
// matrix-core kernels of kv8_attn_mfma.hip do not take).  Work list, partial rows and merge are those of attn_generic.hip.
//
// One wavefront per column (token, query head) of a work item: runs of 64 keys, one per lane for the scores - a key's channels
// lie in pieces of 16 beside the other keys' pieces, so a wavefront's loads are whole lines - then one channel per lane for
// the output, sixteen keys' codes of a channel to a load, with the running maximum and sum of a softmax in fp32 (scores and sums are
// never rounded below it).  A key's scale goes to its score, a value's scale to its probability: codes are multiplied as they
// are.  Only keys up to the column's own position are read.  Bound by the latency of a run's loads, sums and exchanges: about 3 us
// per 64 keys of a wavefront, 8.1 us for 4 requests and two chunks of up to 64 keys (fp32, 4 heads of 64).
#include <algorithm>
#include <cfloat>
#include "flexco_internal.h"
#include "kv8_codes.h"
#include "kv8_internal.h"

namespace flexco {

namespace {

struct Kv8Args {
  const int32_t *tok_pos, *block_table, *tile_req, *tile_tok0, *tile_ntok, *tile_nsplit, *tile_part0, *item_tile,
      *item_split, *item_ntiles;
  int max_pages, nq, nkv, d, ps, split_keys, cols_per_tile, col_blocks;
  float scale;
  void* out;
  size_t ldo;
  float* lse;         // or NULL
  AttnKeep keep;
};

constexpr int NW = 4;      // wavefronts = columns of a block
constexpr int MAX_D = 256;

template <typename T, int DU>
__global__ __launch_bounds__(64 * NW) void kv8_attn_generic_kernel(Kv8Args a, const T* __restrict__ q, size_t ldq,
                                                                   const uint8_t* __restrict__ k_codes, const uint8_t* __restrict__ v_codes,
                                                                   const float* __restrict__ k_scale, const float* __restrict__ v_scale,
                                                                   float* __restrict__ part_ml, float* __restrict__ part_acc) {
  __shared__ float q_sh[NW][MAX_D], p_sh[NW][64];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  float* qs = q_sh[wave];
  float* ps_w = p_sh[wave];
  const int item = blockIdx.x, kvh = blockIdx.y, tile_in = blockIdx.z / a.col_blocks, run = blockIdx.z % a.col_blocks;
  const int ntl = a.item_ntiles[item], tile0 = a.item_tile[item], split = a.item_split[item];
  if (tile_in >= ntl) return;
  const int tile = tile0 + tile_in;
  const int r = a.tile_req[tile], t0 = a.tile_tok0[tile], ntok = a.tile_ntok[tile], nsplit = a.tile_nsplit[tile];
  if (split >= nsplit) return;
  const int group = a.nq / a.nkv, d = a.d, ps = a.ps, pieces = d / 16;
  const int k0 = split * a.split_keys;                        // the first key of a page
  const int32_t* bt = a.block_table + (size_t)r * a.max_pages + k0 / ps;
  const bool whole = nsplit == 1;
  for (int c = run * NW + wave; c < ntok * group; c += NW * a.col_blocks) {
    const int t = t0 + c / group, h = kvh * group + c % group;
    const int nk = max(0, min(k0 + a.split_keys, a.tok_pos[t] + 1) - k0);
    for (int dd = lane; dd < d; dd += 64) qs[dd] = ld(q + (size_t)t * ldq + (size_t)h * d + dd);
    __builtin_amdgcn_wave_barrier();
    float m = -INFINITY, l = 0.f, acc[DU];
#pragma unroll
    for (int u = 0; u < DU; ++u) acc[u] = 0.f;
    for (int j0 = 0; j0 < nk; j0 += 64) {
      const int j = min(j0 + lane, nk - 1);                   // (past the last key: it again, not counted)
      const bool ok = j0 + lane < nk;
      const size_t ph = (size_t)bt[j / ps] * a.nkv + kvh;
      const uint8_t* kr = k_codes + ph * ps * d + (size_t)(j % ps) * 16;
      const int n = min(64, nk - j0);
      // sixteen keys of a channel: one page, one load (a run's are asked for before its scores, past the last key the last ones again)
      u32x4 vw[4][DU];
      if (ps % 16 == 0) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int k = j0 + min(16 * i, (n - 1) & ~15);
          const uint8_t* vr = v_codes + ((size_t)bt[k / ps] * a.nkv + kvh) * ps * d + k % ps;
#pragma unroll
          for (int u = 0; u < DU; ++u) vw[i][u] = *reinterpret_cast<const u32x4*>(vr + (size_t)min(lane + 64 * u, d - 1) * ps);   // (channels past head_dim: not stored)
        }
      }
      float s = 0.f;
#pragma unroll 4
      for (int p = 0; p < pieces; ++p) {
        float kv[16];
        kv8_decode16(*reinterpret_cast<const u32x4*>(kr + (size_t)p * ps * 16), kv);
#pragma unroll
        for (int e = 0; e < 16; ++e) s += qs[p * 16 + e] * kv[e];
      }
      s = ok ? s * (k_scale[ph] * a.scale) : -INFINITY;
      float mx = s;
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor(mx, o, 64));
      const float m_new = fmaxf(m, mx), m_use = m_new == -INFINITY ? 0.f : m_new;
      const float alpha = __expf(m - m_use), p = ok ? __expf(s - m_use) : 0.f;
      float sum = p;
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
      l = l * alpha + sum;
      m = m_new;
      ps_w[lane] = p * v_scale[ph];
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int u = 0; u < DU; ++u) acc[u] *= alpha;
      if (ps % 16 == 0) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int gn = n - 16 * i;
          if (gn <= 0) break;
#pragma unroll
          for (int u = 0; u < DU; ++u) {
            float v[16];
            kv8_decode16(vw[i][u], v);
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[u] += e < gn ? ps_w[16 * i + e] * v[e] : 0.f;   // (slots past the last key may hold anything)
          }
        }
      } else {
        for (int e = 0; e < n; ++e) {
          const uint8_t* vr = v_codes + ((size_t)bt[(j0 + e) / ps] * a.nkv + kvh) * ps * d + (j0 + e) % ps;
          const float w = ps_w[e];
#pragma unroll
          for (int u = 0; u < DU; ++u) acc[u] += w * __builtin_amdgcn_cvt_f32_fp8((int)vr[(size_t)min(lane + 64 * u, d - 1) * ps], 0);
        }
      }
      __builtin_amdgcn_wave_barrier();
    }
    const size_t idx = ((size_t)(a.tile_part0[tile] + split) * a.nkv + kvh) * a.cols_per_tile + c;
    const bool kept = whole && a.keep.lse2 && t >= a.keep.tok0 && t < a.keep.tok0 + a.keep.n;
    const float inv = 1.0f / l;
#pragma unroll
    for (int u = 0; u < DU; ++u) {
      const int dd = lane + 64 * u;
      if (dd >= d) break;
      if (!whole) {
        part_acc[idx * d + dd] = acc[u];
        continue;
      }
      st((T*)a.out + (size_t)t * a.ldo + (size_t)h * d + dd, acc[u] * inv);
      if (kept) st((T*)a.keep.out2 + ((size_t)(t - a.keep.tok0) * a.nq + h) * d + dd, acc[u] * inv);
    }
    if (lane == 0) {
      // (-infinity: no visible key, left out by the join.  Keys of NaN scores alone leave m there too, and their NaN has to get past it.)
      if (!whole) { part_ml[idx * 2] = l == l ? m : fmaxf(m, -FLT_MAX); part_ml[idx * 2 + 1] = l; }
      else if (a.lse) a.lse[(size_t)t * a.nq + h] = m + __logf(l);
      if (kept) a.keep.lse2[(size_t)(t - a.keep.tok0) * a.nq + h] = m + __logf(l);
    }
    __builtin_amdgcn_wave_barrier();
  }
}

}  // namespace

int32_t launch_kv8_attention_generic(const flexco_layer_cfg& c, const flexco_maps& m, const void* q, size_t ldq,
                                     const flexco_kv8_pool& pool, float* part_ml, float* part_acc, void* out, size_t ldo, float* lse,
                                     hipStream_t s, const AttnKeep* keep) {
  const int group = c.n_q_heads / c.n_kv_heads;
  Kv8Args a;
  a.tok_pos = m.tok_pos; a.block_table = m.block_table; a.tile_req = m.tile_req; a.tile_tok0 = m.tile_tok0;
  a.tile_ntok = m.tile_ntok; a.tile_nsplit = m.tile_nsplit; a.tile_part0 = m.tile_part0; a.item_tile = m.item_tile;
  a.item_split = m.item_split; a.item_ntiles = m.item_ntiles;
  a.max_pages = m.max_pages; a.nq = c.n_q_heads; a.nkv = c.n_kv_heads; a.d = c.head_dim; a.ps = c.page_size;
  a.split_keys = m.kv_split_pages * c.page_size;
  a.cols_per_tile = m.tile_tokens * group;
  a.scale = 1.0f / sqrtf((float)c.head_dim);
  a.out = out; a.ldo = ldo; a.lse = lse;
  a.keep = keep ? *keep : AttnKeep{nullptr, nullptr, 0, 0};
  const bool singles = m.n_single == m.n_items;               // (one tile of one token per item)
  a.col_blocks = singles ? (group + NW - 1) / NW : 4;
  const dim3 grid(m.n_items, c.n_kv_heads, (singles ? 1 : FLEXCO_ATTN_ITEM_TILES) * a.col_blocks);
#define FLEXCO_KV8_GENERIC(T_, DU_)                                                                                              \
  hipLaunchKernelGGL((kv8_attn_generic_kernel<T_, DU_>), grid, dim3(64 * NW), 0, s, a, (const T_*)q, ldq, pool.k_codes, pool.v_codes, \
                     pool.k_scale, pool.v_scale, part_ml, part_acc)
  const int du = (c.head_dim + 63) / 64;
  if (c.dtype == FLEXCO_BF16) {
    if (du == 1) FLEXCO_KV8_GENERIC(bf16_t, 1); else if (du == 2) FLEXCO_KV8_GENERIC(bf16_t, 2); else FLEXCO_KV8_GENERIC(bf16_t, 4);
  } else {
    if (du == 1) FLEXCO_KV8_GENERIC(float, 1); else if (du == 2) FLEXCO_KV8_GENERIC(float, 2); else FLEXCO_KV8_GENERIC(float, 4);
  }
#undef FLEXCO_KV8_GENERIC
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return fail(FLEXCO_EHIP, "launch of kv8_attn_generic failed: %s", hipGetErrorString(e));
  return FLEXCO_OK;
}

}  // namespace flexco
