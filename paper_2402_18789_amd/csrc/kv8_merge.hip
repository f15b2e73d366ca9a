// Joining the partial rows of the 8-bit attention: a row's pieces are (m_i, l_i, o_i), sums of exp(s - m_i) and of exp(s - m_i) v over the keys
// of a piece; with M = max m_i the row is sum o_i exp(m_i - M) / sum l_i exp(m_i - M), its log-sum-exp M plus the log of that sum.
// A piece without a visible key has m_i = -infinity and is left out; one whose keys' scores are all NaN has the lowest finite m_i.
#include "device_types.h"
#include "flexco_internal.h"
#include "kv8_internal.h"

namespace flexco {

namespace {

struct MergeArgs {
  const int32_t *tok_tile, *tok_req, *req_tok_off, *tile_nsplit, *tile_part0, *tile_tok0;
  int nq, nkv, d, cpt, fold;
  const float *part_ml, *part_acc;
  void* out;
  size_t ldo;
  float* lse;         // or NULL
  AttnKeep keep;
};

// A block per (token, query head, 128 channels), for lists in which a request is cut into many pieces: eight groups of 32 lanes take the
// pieces in turn, four loads at a time, and add up in LDS in group order.  Bound by the latency of two rounds of loads: up to 32 pieces of three
// long contexts over 40 heads 4.9 us.  (The merge that lists of few pieces take walks them one group per row: 118 pieces of these 50 us.)
constexpr int MG = 8, MD = 128;
template <typename T>
__global__ __launch_bounds__(32 * MG) void kv8_merge_long_kernel(MergeArgs a) {
  __shared__ float red_m[32 * MG / 64], part[MG][MD], part_l[MG];
  const int t = blockIdx.x, h = blockIdx.y, tid = threadIdx.x, grp = tid >> 5, dd = blockIdx.z * MD + 4 * (tid & 31);
  const int group = a.nq / a.nkv, kvh = h / group, tile = a.tok_tile[t], r = a.tok_req[t];
  const int fold = a.fold > 1 && a.req_tok_off[r + 1] - a.req_tok_off[r] == 1 ? a.fold : 1;
  const int n = (a.tile_nsplit[tile] + fold - 1) / fold;       // partial rows
  if (n == 1) return;                                          // the attention kernel has written these rows itself (whole block)
  const size_t idx0 = ((size_t)a.tile_part0[tile] * a.nkv + kvh) * a.cpt + (t - a.tile_tok0[tile]) * group + h % group;
  const size_t step = (size_t)fold * a.nkv * a.cpt;
  float m = -INFINITY;
  for (int i = tid; i < n; i += 32 * MG) m = fmaxf(m, a.part_ml[(idx0 + i * step) * 2]);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
  if ((tid & 63) == 0) red_m[tid >> 6] = m;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < 32 * MG / 64; ++w) m = fmaxf(m, red_m[w]);
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  float l = 0.f;
  const bool mine = dd < a.d;                                  // (head_dim is a multiple of 16)
  constexpr int U = 4;
  for (int i0 = grp; i0 < n; i0 += MG * U) {
    float2 ml[U];
    f32x4 v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const size_t idx = idx0 + min(i0 + u * MG, n - 1) * step;
      ml[u] = *reinterpret_cast<const float2*>(a.part_ml + idx * 2);
      v[u] = *reinterpret_cast<const f32x4*>(a.part_acc + idx * a.d + (mine ? dd : 0));
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (i0 + u * MG < n && !(ml[u].x == -INFINITY)) {       // (the sums of a piece without a visible key are not written)
        const float w = __expf(ml[u].x - m);
        l += ml[u].y * w;
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[j] += v[u][j] * w;
      }
  }
  *reinterpret_cast<f32x4*>(&part[grp][4 * (tid & 31)]) = acc;
  if ((tid & 31) == 0) part_l[grp] = l;
  __syncthreads();
  if (grp != 0) return;
  f32x4 row = {0.f, 0.f, 0.f, 0.f};
  float L = 0.f;
#pragma unroll
  for (int w = 0; w < MG; ++w) {
    const f32x4 v = *reinterpret_cast<const f32x4*>(&part[w][4 * (tid & 31)]);
#pragma unroll
    for (int j = 0; j < 4; ++j) row[j] += v[j];
    L += part_l[w];
  }
  const float inv = 1.0f / L;
  const bool kept = a.keep.lse2 && t >= a.keep.tok0 && t < a.keep.tok0 + a.keep.n;
  if (mine) {
    typedef T T4 __attribute__((ext_vector_type(4)));
    T4 o;
#pragma unroll
    for (int j = 0; j < 4; ++j) o[j] = (T)(row[j] * inv);
    *reinterpret_cast<T4*>((T*)a.out + (size_t)t * a.ldo + (size_t)h * a.d + dd) = o;
    if (kept) *reinterpret_cast<T4*>((T*)a.keep.out2 + ((size_t)(t - a.keep.tok0) * a.nq + h) * a.d + dd) = o;
  }
  if (dd == 0) {
    const float z = m + __logf(L);
    if (a.lse) a.lse[(size_t)t * a.nq + h] = z;
    if (kept) a.keep.lse2[(size_t)(t - a.keep.tok0) * a.nq + h] = z;
  }
}

}  // namespace

int32_t launch_kv8_merge(const flexco_layer_cfg& c, const flexco_maps& m, const float* part_ml, const float* part_acc, void* out, size_t ldo,
                         float* lse, hipStream_t s, int fold, const AttnKeep* keep) {
  KernelTimerScope ts(FLEXCO_K_ATTN_MERGE, s);
  // The long form from nine pieces on where there are few rows (4 tokens of 4000 keys in eights 18.4 -> 15.1 us, 8 of 8000 in 32s 36.0 -> 32.5;
  // with 256 x 16 rows of up to five pieces it cost 4 more), from seventeen on in any case.
  const int most = (m.max_pages + fold * m.kv_split_pages - 1) / (fold * m.kv_split_pages);
  const bool long_axis = most > 16 || (most > 8 && (int64_t)m.T * c.n_q_heads <= 2048);
  if (!long_axis || ldo % 4 != 0 || ((uintptr_t)out & 15)) return launch_attention_merge(c, m, part_ml, part_acc, out, ldo, lse, s, fold, keep);
  MergeArgs a;
  a.tok_tile = m.tok_tile; a.tok_req = m.tok_req; a.req_tok_off = m.req_tok_off;
  a.tile_nsplit = m.tile_nsplit; a.tile_part0 = m.tile_part0; a.tile_tok0 = m.tile_tok0;
  a.nq = c.n_q_heads; a.nkv = c.n_kv_heads; a.d = c.head_dim; a.cpt = m.tile_tokens * (c.n_q_heads / c.n_kv_heads); a.fold = fold;
  a.part_ml = part_ml; a.part_acc = part_acc;
  a.out = out; a.ldo = ldo; a.lse = lse;
  a.keep = keep ? *keep : AttnKeep{nullptr, nullptr, 0, 0};
  const dim3 grid(m.T, c.n_q_heads, (c.head_dim + MD - 1) / MD);
  if (c.dtype == FLEXCO_BF16) hipLaunchKernelGGL(kv8_merge_long_kernel<bf16_t>, grid, dim3(32 * MG), 0, s, a);
  else hipLaunchKernelGGL(kv8_merge_long_kernel<float>, grid, dim3(32 * MG), 0, s, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return fail(FLEXCO_EHIP, "launch of kv8_merge_long failed: %s", hipGetErrorString(e));
  return FLEXCO_OK;
}

}  // namespace flexco
