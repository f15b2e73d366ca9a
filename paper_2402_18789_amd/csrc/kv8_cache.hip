// The 8-bit paged cache: append of a batch's tokens and pages written out again (format and rules: flexco_kv8.h).
//
// Append.  One block per (run, kv head): the run's tokens of the head's query group, its keys and its values.  A page's scale
// is chosen from all of its new rows, so the block first takes the largest magnitude of the rotated keys and of the values
// and then rounds them; it owns the page's codes of the head, so a scale that has grown is applied to the codes already there by the
// same block.  Bound by HBM: (2 nq + 2 nkv) d activations and 2 nkv d bytes per token.
#include "flexco_internal.h"
#include "flexco_kv8.h"
#include "kv8_codes.h"
#include "kv8_internal.h"
#include "rope.h"

namespace flexco {

namespace {

constexpr int THREADS = 256;
constexpr int GROUP = 16;          // tokens whose angles are in LDS at a time

__device__ inline void load8(const float* p, float* v) { Vec<float>::load(p, v); Vec<float>::load(p + 4, v + 4); }
__device__ inline void load8(const bf16_t* p, float* v) { Vec<bf16_t>::load(p, v); }
__device__ inline void store8(float* p, const float* v) { Vec<float>::store(p, v); Vec<float>::store(p + 4, v + 4); }
__device__ inline void store8(bf16_t* p, const float* v) { Vec<bf16_t>::store(p, v); }

struct AppendArgs {
  const int32_t *runs, *tok_pos, *slot;
  uint8_t *k_codes, *v_codes;
  float *k_scale, *v_scale;
  int n_runs, T, num_pages, ps, nq, nkv, d;
  size_t ld_q;
  // the finetune window's rotated queries, written a second time (row i of the window at q_cache + i nq d); n_ft = 0: none
  int ft_tok0, n_ft;
  void* q_cache;
};

// largest of a block's values, in every thread
__device__ inline float block_max(float v, float* red) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) v = fmaxf(v, red[w]);
  return v;
}

template <typename T>
__global__ __launch_bounds__(THREADS) void kv8_append_kernel(AppendArgs a, RopeFreq freq, const T* qkv, T* q_out) {
  extern __shared__ float cs[];               // [GROUP][d]: cosines, then sines, of a token's d / 2 angles
  __shared__ float red_k[THREADS / 64], red_v[THREADS / 64];
  const int run = blockIdx.x / a.nkv, kvh = blockIdx.x % a.nkv, tid = threadIdx.x;
  const int t0 = a.runs[2 * run], n = a.runs[2 * run + 1];
  const int d = a.d, half = d >> 1, ps = a.ps, group = a.nq / a.nkv;
  if (t0 < 0 || n < 1 || n > ps || t0 > a.T - n) return;                // (whole block, as below)
  const int sl = a.slot[t0], page = sl / ps, at = sl % ps;
  if (sl < 0 || page >= a.num_pages || at + n > ps) return;
  const size_t row_el = (size_t)(a.nq + 2 * a.nkv) * d;
  const T* rows = qkv + (size_t)t0 * row_el;
  const int k_col = (a.nq + kvh) * d, v_col = (a.nq + a.nkv + kvh) * d;
  const int pieces8 = d / 8;

  auto angles = [&](int g0, int gn) {
    for (int i = tid; i < gn * half; i += THREADS) {
      const int tl = i / half, j = i % half;
      rope_cos_sin(freq, j, a.tok_pos[t0 + g0 + tl], &cs[tl * d + j], &cs[tl * d + half + j]);
    }
  };
  // eight rotated channels ch .. ch + 7 of a row of keys
  auto key8 = [&](int g0, int tl, int ch, float* v) {
    const T* kr = rows + (size_t)(g0 + tl) * row_el + k_col;
    const bool low = ch < half;
    float x[8], y[8];
    load8(kr + ch, x);
    load8(kr + (low ? ch + half : ch - half), y);
    const float* c = cs + tl * d + (low ? ch : ch - half);
    const float sg = low ? -1.f : 1.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = x[e] * c[e] + sg * y[e] * c[half + e];
  };

  // queries out, and the largest magnitudes
  float mk = 0.f, mv = 0.f;
  for (int g0 = 0; g0 < n; g0 += GROUP) {
    const int gn = min(GROUP, n - g0);
    if (g0) __syncthreads();
    angles(g0, gn);
    __syncthreads();
    for (int u = tid; u < gn * group * (pieces8 / 2); u += THREADS) {
      const int ch = u % (pieces8 / 2) * 8, hh = u / (pieces8 / 2) % group, tl = u / (pieces8 / 2) / group;
      const int h = kvh * group + hh, t = t0 + g0 + tl;
      const T* qr = rows + (size_t)(g0 + tl) * row_el + (size_t)h * d;
      float x[8], y[8], lo[8], hi[8];
      load8(qr + ch, x);
      load8(qr + ch + half, y);
      const float* c = cs + tl * d + ch;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        lo[e] = x[e] * c[e] - y[e] * c[half + e];
        hi[e] = y[e] * c[e] + x[e] * c[half + e];
      }
      T* o = q_out + (size_t)t * a.ld_q + (size_t)h * d + ch;
      store8(o, lo);
      store8(o + half, hi);
      if (t >= a.ft_tok0 && t < a.ft_tok0 + a.n_ft) {
        T* o2 = (T*)a.q_cache + ((size_t)(t - a.ft_tok0) * a.nq + h) * d + ch;
        store8(o2, lo);
        store8(o2 + half, hi);
      }
    }
    for (int u = tid; u < gn * pieces8; u += THREADS) {
      const int tl = u / pieces8, ch = u % pieces8 * 8;
      float v[8];
      key8(g0, tl, ch, v);
#pragma unroll
      for (int e = 0; e < 8; ++e) mk = fmaxf(mk, kv8_finite(v[e]) ? fabsf(v[e]) : 0.f);
      load8(rows + (size_t)(g0 + tl) * row_el + v_col + ch, v);
#pragma unroll
      for (int e = 0; e < 8; ++e) mv = fmaxf(mv, kv8_finite(v[e]) ? fabsf(v[e]) : 0.f);
    }
  }
  const size_t ph = (size_t)page * a.nkv + kvh;
  const float old_k = at ? a.k_scale[ph] : 0.f, old_v = at ? a.v_scale[ph] : 0.f;
  const float s_k = fmaxf(old_k, kv8_scale_for(block_max(mk, red_k))), s_v = fmaxf(old_v, kv8_scale_for(block_max(mv, red_v)));
  __syncthreads();                       // (every thread has read the old scales)
  if (tid == 0) { a.k_scale[ph] = s_k; a.v_scale[ph] = s_v; }
  const float inv_k = 1.f / s_k, inv_v = 1.f / s_v;      // (powers of two)
  uint8_t* kc = a.k_codes + ph * ps * d;
  uint8_t* vc = a.v_codes + ph * ps * d;
  // codes that were there, at the new scale
  if (at && s_k > old_k)
    for (int u = tid; u < (d / 16) * ps; u += THREADS) {
      const int p = u % ps;
      if (p >= at && p < at + n) continue;
      u32x4 w = *reinterpret_cast<u32x4*>(kc + (size_t)u * 16);
      float v[16];
      kv8_decode16(w, v);
#pragma unroll
      for (int e = 0; e < 16; ++e) v[e] *= old_k * inv_k;
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = kv8_encode4(v + 4 * i);
      *reinterpret_cast<u32x4*>(kc + (size_t)u * 16) = w;
    }
  if (at && s_v > old_v)
    for (int u = tid; u < d * ps; u += THREADS) {
      const int p = u % ps;
      if (p >= at && p < at + n) continue;
      const float v[4] = {__builtin_amdgcn_cvt_f32_fp8((int)vc[u], 0) * old_v * inv_v, 0.f, 0.f, 0.f};
      vc[u] = (uint8_t)kv8_encode4(v);
    }
  for (int g0 = 0; g0 < n; g0 += GROUP) {
    const int gn = min(GROUP, n - g0);
    if (n > GROUP) {
      __syncthreads();
      angles(g0, gn);
      __syncthreads();
    }
    for (int u = tid; u < gn * pieces8; u += THREADS) {
      const int tl = u / pieces8, ch = u % pieces8 * 8;
      float v[8];
      key8(g0, tl, ch, v);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = kv8_storable(v[e]) * inv_k;
      const u32x2 w = {kv8_encode4(v), kv8_encode4(v + 4)};
      *reinterpret_cast<u32x2*>(kc + ((size_t)(ch / 16) * ps + at + g0 + tl) * 16 + ch % 16) = w;
    }
    for (int u = tid; u < gn * d; u += THREADS) {
      const int tl = u / d, ch = u % d;
      const float v[4] = {kv8_storable(ld(rows + (size_t)(g0 + tl) * row_el + v_col + ch)) * inv_v, 0.f, 0.f, 0.f};
      vc[(size_t)ch * ps + at + g0 + tl] = (uint8_t)kv8_encode4(v);
    }
  }
}

// Expand.  One block per (page, kv head): 2 d ps codes in, as many elements out.
template <typename T>
__global__ __launch_bounds__(THREADS) void kv8_expand_kernel(const uint8_t* __restrict__ k_codes, const uint8_t* __restrict__ v_codes,
                                                             const float* __restrict__ k_scale, const float* __restrict__ v_scale,
                                                             const int32_t* __restrict__ src, const int32_t* __restrict__ dst,
                                                             T* __restrict__ kp, T* __restrict__ vp, int src_pages, int dst_pages,
                                                             int n_tokens, int nkv, int d, int ps) {
  const int i = blockIdx.x / nkv, kvh = blockIdx.x % nkv;
  const int from = src[i], to = dst[i];
  if (from < 0 || from >= src_pages || to < 0 || to >= dst_pages) return;
  const size_t ph = (size_t)from * nkv + kvh, oh = (size_t)to * nkv + kvh;
  const float sk = k_scale[ph], sv = v_scale[ph];
  const uint8_t* kc = k_codes + ph * ps * d;
  const uint8_t* vc = v_codes + ph * ps * d;
  T* ko = kp + oh * ps * d;
  T* vo = vp + oh * ps * d;
  const int pieces = d / 16, n = n_tokens - i * ps;              // the sequence's tokens from this page on
  for (int u = threadIdx.x; u < pieces * ps; u += THREADS) {
    // neighbouring threads write a key's row; it lies in pieces among the other keys'
    const int key = u / pieces, c = u % pieces;
    float v[16];
    kv8_decode16(*reinterpret_cast<const u32x4*>(kc + ((size_t)c * ps + key) * 16), v);
#pragma unroll
    for (int e = 0; e < 16; ++e) v[e] = key < n ? v[e] * sk : 0.f;
    store8(ko + (size_t)u * 16, v);
    store8(ko + (size_t)u * 16 + 8, v + 8);
    kv8_decode16(*reinterpret_cast<const u32x4*>(vc + (size_t)u * 16), v);
#pragma unroll
    for (int e = 0; e < 16; ++e) v[e] = (u * 16 + e) % ps < n ? v[e] * sv : 0.f;
    store8(vo + (size_t)u * 16, v);
    store8(vo + (size_t)u * 16 + 8, v + 8);
  }
}

int32_t post(const char* what) {
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return fail(FLEXCO_EHIP, "launch of %s failed: %s", what, hipGetErrorString(e));
  return FLEXCO_OK;
}

}  // namespace

int32_t launch_kv8_append(const flexco_layer_cfg& c, const flexco_maps& m, const int32_t* runs, int n_runs, const void* qkv,
                          const flexco_kv8_pool& pool, void* q_out, size_t ld_q, void* q_cache, hipStream_t s) {
  if (n_runs == 0) return FLEXCO_OK;
  RopeFreq freq;
  FLEXCO_TRY(rope_freq(c, &freq));
  const AppendArgs a{runs, m.tok_pos, m.slot, pool.k_codes, pool.v_codes, pool.k_scale, pool.v_scale, n_runs, m.T, pool.num_pages,
                     pool.page_size, c.n_q_heads, c.n_kv_heads, c.head_dim, ld_q, m.ft_tok0, q_cache ? m.n_ft : 0, q_cache};
  const dim3 grid((unsigned)n_runs * c.n_kv_heads);
  const size_t shm = sizeof(float) * GROUP * c.head_dim;
  if (c.dtype == FLEXCO_BF16)
    hipLaunchKernelGGL((kv8_append_kernel<bf16_t>), grid, dim3(THREADS), shm, s, a, freq, (const bf16_t*)qkv, (bf16_t*)q_out);
  else
    hipLaunchKernelGGL((kv8_append_kernel<float>), grid, dim3(THREADS), shm, s, a, freq, (const float*)qkv, (float*)q_out);
  return post("kv8_append");
}

int32_t launch_kv8_expand(const flexco_layer_cfg& c, const flexco_kv8_pool& pool, const int32_t* src, int n_tokens,
                          const flexco_kv_pool& wide, const int32_t* dst, hipStream_t s) {
  const int n_pages = (n_tokens + c.page_size - 1) / c.page_size;
  if (n_pages == 0) return FLEXCO_OK;
  const dim3 grid((unsigned)n_pages * c.n_kv_heads);
  if (c.dtype == FLEXCO_BF16)
    hipLaunchKernelGGL((kv8_expand_kernel<bf16_t>), grid, dim3(THREADS), 0, s, pool.k_codes, pool.v_codes, pool.k_scale, pool.v_scale, src,
                       dst, (bf16_t*)wide.k_pages, (bf16_t*)wide.v_pages, pool.num_pages, wide.num_pages, n_tokens, c.n_kv_heads, c.head_dim,
                       c.page_size);
  else
    hipLaunchKernelGGL((kv8_expand_kernel<float>), grid, dim3(THREADS), 0, s, pool.k_codes, pool.v_codes, pool.k_scale, pool.v_scale, src,
                       dst, (float*)wide.k_pages, (float*)wide.v_pages, pool.num_pages, wide.num_pages, n_tokens, c.n_kv_heads, c.head_dim,
                       c.page_size);
  return post("kv8_expand");
}

}  // namespace flexco
