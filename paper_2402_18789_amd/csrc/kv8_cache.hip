// The 8-bit paged cache: append of a batch's tokens and pages written out again (format and rules: flexco_kv8.h).
//
// Append.  A page's scale is chosen from all of its new rows, so the rotated keys and the values of a (run, kv head) are held until
// their largest magnitude is known; whoever does that owns the page's codes of the head, so a scale that has grown is applied to the
// codes already there on the spot.  Bound by HBM: (2 nq + 2 nkv) d activations and 2 nkv d bytes per token.
// Keys are rotated in double precision and rounded once, into the cache (an angle's fp32 error of 5e-7 moved one code in 10^5).
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

// Cosine and sine of pair i's angle at position pos: the turn's distance to the nearest quarter, at most an eighth, and the Taylor series of
// both there (x <= pi / 4: what is left out is below 5e-14).
__device__ inline void cos_sin_64(const RopeFreq& f, int i, int pos, double* c, double* s) {
  const double r = (double)pos * f.rev[i], turn = r - floor(r), quarter = rint(4.0 * turn);
  const double x = (turn - 0.25 * quarter) * 6.283185307179586476925, y = x * x;
  const double sn = x * (1.0 + y * (-1.0 / 6 + y * (1.0 / 120 + y * (-1.0 / 5040 + y * (1.0 / 362880 + y * (-1.0 / 39916800 + y * (1.0 / 6227020800.0)))))));
  const double cs = 1.0 + y * (-0.5 + y * (1.0 / 24 + y * (-1.0 / 720 + y * (1.0 / 40320 + y * (-1.0 / 3628800 + y * (1.0 / 479001600.0 + y * (-1.0 / 87178291200.0)))))));
  const int k = (int)quarter & 3;
  const double a = k & 1 ? sn : cs, b = k & 1 ? cs : sn;
  *c = k == 1 || k == 2 ? -a : a;
  *s = k >= 2 ? -b : b;
}

// cs: d / 2 cosines, then sines, of a token.  Eight pairs from channel ch < d / 2 on: x, y -> x c - y s, y c + x s
template <typename F>
__device__ inline void rotate8(const double* cs, int half, int ch, const float* x, const float* y, F* lo, F* hi) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const F c = (F)cs[ch + e], s = (F)cs[half + ch + e];
    lo[e] = (F)x[e] * c - (F)y[e] * s;
    hi[e] = (F)y[e] * c + (F)x[e] * s;
  }
}
__device__ inline float finite_abs(float v) { return kv8_finite(v) ? fabsf(v) : 0.f; }

template <typename T>
__device__ inline void query8(const AppendArgs& a, const double* cs, const T* row, T* q_out, int t, int h, int ch) {
  const int half = a.d >> 1;
  float x[8], y[8], lo[8], hi[8];
  load8(row + (size_t)h * a.d + ch, x);
  load8(row + (size_t)h * a.d + ch + half, y);
  rotate8<float>(cs, half, ch, x, y, lo, hi);
  T* o = q_out + (size_t)t * a.ld_q + (size_t)h * a.d + ch;
  store8(o, lo);
  store8(o + half, hi);
  if (t >= a.ft_tok0 && t < a.ft_tok0 + a.n_ft) {
    T* o2 = (T*)a.q_cache + ((size_t)(t - a.ft_tok0) * a.nq + h) * a.d + ch;
    store8(o2, lo);
    store8(o2 + half, hi);
  }
}
__device__ inline u32x2 encode8(const float* v, float inv) {
  float w[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) w[e] = kv8_storable(v[e]) * inv;
  return u32x2{kv8_encode4(w), kv8_encode4(w + 4)};
}
template <typename T>
__device__ inline void key8(const AppendArgs& a, const double* cs, const T* row, int kvh, int ch, float* lo, float* hi) {
  const int half = a.d >> 1;
  const T* kr = row + (size_t)(a.nq + kvh) * a.d;
  float x[8], y[8];
  double l[8], h[8];
  load8(kr + ch, x);
  load8(kr + ch + half, y);
  rotate8<double>(cs, half, ch, x, y, l, h);
#pragma unroll
  for (int e = 0; e < 8; ++e) { lo[e] = (float)l[e]; hi[e] = (float)h[e]; }
}

// Sixteen bytes of a page's codes (unit u of d ps / 16) times `by`, but for those of positions [at, at + n)
__device__ inline void rescale_unit(uint8_t* codes, int u, int ps, int at, int n, float by, bool keys) {
  u32x4* p = reinterpret_cast<u32x4*>(codes + (size_t)u * 16);
  const u32x4 was = *p;
  u32x4 now;
  float v[16];
  kv8_decode16(was, v);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t mask = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int pos = keys ? u % ps : (16 * u + 4 * i + e) % ps;
      v[4 * i + e] *= by;
      mask |= (pos >= at && pos < at + n ? 0xffu : 0u) << (8 * e);
    }
    now[i] = (was[i] & mask) | (kv8_encode4(v + 4 * i) & ~mask);
  }
  *p = now;
}

// The scales of a run's page and head: of K and of V.  amax: bits of the largest magnitudes (LDS, order of positive floats is that of
// their bits).
struct Scales { float old_k, old_v, k, v; };
__device__ inline Scales page_scales(const AppendArgs& a, size_t ph, int at, uint32_t amax_k, uint32_t amax_v) {
  Scales s;
  s.old_k = at ? a.k_scale[ph] : 0.f;
  s.old_v = at ? a.v_scale[ph] : 0.f;
  s.k = fmaxf(s.old_k, kv8_scale_for(__builtin_bit_cast(float, amax_k)));
  s.v = fmaxf(s.old_v, kv8_scale_for(__builtin_bit_cast(float, amax_v)));
  return s;
}

// A run of one token: one block for all heads (a block per head had an eighth of its threads at work).
template <typename T>
__device__ inline void append_token(const AppendArgs& a, const RopeFreq& freq, const T* qkv, T* q_out, int t, int page, int at, double* cs,
                                    uint32_t* amax) {
  const int tid = threadIdx.x, d = a.d, half = d >> 1, pc = d / 16;
  const T* row = qkv + (size_t)t * (a.nq + 2 * a.nkv) * d;
  for (int h = tid; h < 2 * a.nkv; h += THREADS) amax[h] = 0;
  for (int i = tid; i < half; i += THREADS) cos_sin_64(freq, i, a.tok_pos[t], &cs[i], &cs[half + i]);
  __syncthreads();
  const T* vrow = row + (size_t)(a.nq + a.nkv) * d;
  for (int u = tid; u < 2 * a.nkv * pc; u += THREADS) {
    const int h = u / pc % a.nkv, ch = u % pc * 8;
    float v[16], m = 0.f;
    if (u < a.nkv * pc) {
      key8(a, cs, row, h, ch, v, v + 8);
    } else {
      load8(vrow + (size_t)h * d + 2 * ch, v);
      load8(vrow + (size_t)h * d + 2 * ch + 8, v + 8);
    }
#pragma unroll
    for (int e = 0; e < 16; ++e) m = fmaxf(m, finite_abs(v[e]));
    atomicMax(&amax[u < a.nkv * pc ? h : a.nkv + h], __builtin_bit_cast(uint32_t, m));
  }
  __syncthreads();
  // (old scales are read here by every thread of a head and written behind the next barrier)
  for (int u = tid; u < 2 * a.nkv * pc; u += THREADS) {
    const int h = u / pc % a.nkv, ch = u % pc * 8;
    const size_t ph = (size_t)page * a.nkv + h;
    const Scales s = page_scales(a, ph, at, amax[h], amax[a.nkv + h]);
    float v[16];
    if (u < a.nkv * pc) {
      key8(a, cs, row, h, ch, v, v + 8);
      uint8_t* kc = a.k_codes + ph * a.ps * d;
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int c = ch + x * half;
        *reinterpret_cast<u32x2*>(kc + ((size_t)(c / 16) * a.ps + at) * 16 + c % 16) = encode8(v + 8 * x, 1.f / s.k);
      }
    } else {
      load8(vrow + (size_t)h * d + 2 * ch, v);
      load8(vrow + (size_t)h * d + 2 * ch + 8, v + 8);
      uint8_t* vc = a.v_codes + ph * a.ps * d + at;
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const u32x2 w = encode8(v + 8 * x, 1.f / s.v);
#pragma unroll
        for (int e = 0; e < 8; ++e) vc[(size_t)(2 * ch + 8 * x + e) * a.ps] = (uint8_t)(w[e / 4] >> (8 * (e % 4)));
      }
    }
  }
  for (int u = tid; u < a.nq * pc; u += THREADS) query8(a, cs, row, q_out, t, u / pc, u % pc * 8);
  __syncthreads();
  if (at) {
    const int units = d * a.ps / 16;
    for (int i = tid; i < 2 * a.nkv * units; i += THREADS) {
      const int h = i / units % a.nkv;
      const bool keys = i < a.nkv * units;
      const size_t ph = (size_t)page * a.nkv + h;
      const Scales s = page_scales(a, ph, at, amax[h], amax[a.nkv + h]);
      if (keys ? s.k > s.old_k : s.v > s.old_v)
        rescale_unit((keys ? a.k_codes : a.v_codes) + ph * a.ps * d, i % units, a.ps, at, 1, keys ? s.old_k / s.k : s.old_v / s.v, keys);
    }
  }
  __syncthreads();
  for (int h = tid; h < a.nkv; h += THREADS) {
    const size_t ph = (size_t)page * a.nkv + h;
    const Scales s = page_scales(a, ph, at, amax[h], amax[a.nkv + h]);
    a.k_scale[ph] = s.k;
    a.v_scale[ph] = s.v;
  }
}

// A run's page of sixteen positions, head_dim up to 128: half the block's threads hold the keys, half the values, sixteen elements
// each, from their load to their codes, which go to memory through an image of the page in LDS: 16 bytes at a time.
template <typename T>
__device__ inline void append_page16(const AppendArgs& a, const RopeFreq& freq, const T* qkv, T* q_out, int t0, int n, int kvh, int page,
                                     int at, double* cs, uint32_t* amax) {
  __shared__ __attribute__((aligned(16))) uint8_t image[2][16 * 128];
  const int tid = threadIdx.x, d = a.d, half = d >> 1, pc = d / 16, group = a.nq / a.nkv;
  const size_t row_el = (size_t)(a.nq + 2 * a.nkv) * d, ph = (size_t)page * a.nkv + kvh;
  const T* rows = qkv + (size_t)t0 * row_el;
  const bool keys = tid < THREADS / 2;
  const int u = tid % (THREADS / 2), tl = u / pc, ch = u % pc * 8;
  const bool mine = u < n * pc;
  // (everything that needs nothing but the run is asked for before the angles)
  float x[16];
  const T* src = rows + (size_t)tl * row_el + (size_t)(keys ? a.nq + kvh : a.nq + a.nkv + kvh) * d;
  if (mine) {
    load8(src + (keys ? ch : 2 * ch), x);
    load8(src + (keys ? ch + half : 2 * ch + 8), x + 8);
  }
  const float old_k = at ? a.k_scale[ph] : 0.f, old_v = at ? a.v_scale[ph] : 0.f;
  if (tid < 2) amax[tid] = 0;
  for (int i = tid; i < n * half; i += THREADS) cos_sin_64(freq, i % half, a.tok_pos[t0 + i / half], &cs[i / half * d + i % half], &cs[i / half * d + half + i % half]);
  __syncthreads();
  float m = 0.f;
  if (mine) {
    if (keys) {
      double l[8], h[8];
      rotate8<double>(cs + tl * d, half, ch, x, x + 8, l, h);
#pragma unroll
      for (int e = 0; e < 8; ++e) { x[e] = (float)l[e]; x[8 + e] = (float)h[e]; }
    }
#pragma unroll
    for (int e = 0; e < 16; ++e) m = fmaxf(m, finite_abs(x[e]));
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
  if ((tid & 63) == 0) atomicMax(&amax[keys ? 0 : 1], __builtin_bit_cast(uint32_t, m));
  __syncthreads();
  const float s_k = fmaxf(old_k, kv8_scale_for(__builtin_bit_cast(float, amax[0]))), s_v = fmaxf(old_v, kv8_scale_for(__builtin_bit_cast(float, amax[1])));
  if (tid == 0) { a.k_scale[ph] = s_k; a.v_scale[ph] = s_v; }
  if (mine) {
    const float inv = 1.f / (keys ? s_k : s_v);
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      const u32x2 w = encode8(x + 8 * y, inv);
      if (keys) {
        const int c = ch + y * half;
        *reinterpret_cast<u32x2*>(&image[0][(c / 16 * 16 + at + tl) * 16 + c % 16]) = w;
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) image[1][(2 * ch + 8 * y + e) * 16 + at + tl] = (uint8_t)(w[e / 4] >> (8 * (e % 4)));
      }
    }
  }
  for (int i = tid; i < n * group * pc; i += THREADS) {
    const int qt = i / (group * pc), h = kvh * group + i / pc % group;
    query8(a, cs + qt * d, rows + (size_t)qt * row_el, q_out, t0 + qt, h, i % pc * 8);
  }
  __syncthreads();
  // a unit: sixteen channels of a position (keys), sixteen positions of a channel (values)
  if (u >= pc * 16) return;
  uint8_t* to = (keys ? a.k_codes : a.v_codes) + ph * 16 * d + (size_t)u * 16;
  u32x4 w = *reinterpret_cast<const u32x4*>(&image[keys ? 0 : 1][u * 16]);
  const bool grew = at && (keys ? s_k > old_k : s_v > old_v);
  if (n < 16) {
    // what other positions' codes are, at a scale that has grown
    if (keys && !grew && !(u % 16 >= at && u % 16 < at + n)) return;
    const u32x4 there = *reinterpret_cast<const u32x4*>(to);
    const float by = keys ? old_k / s_k : old_v / s_v;
    float v[16];
    kv8_decode16(there, v);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t kept = there[i], mask = 0;
      if (grew) {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[4 * i + e] *= by;
        kept = kv8_encode4(v + 4 * i);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int pos = keys ? u % 16 : 4 * i + e;
        mask |= (pos >= at && pos < at + n ? 0xffu : 0u) << (8 * e);
      }
      w[i] = (w[i] & mask) | (kept & ~mask);
    }
  }
  *reinterpret_cast<u32x4*>(to) = w;
}

// Any page size and head_dim: one block per (run, kv head), the rows read again for their codes.
template <typename T>
__device__ inline void append_any(const AppendArgs& a, const RopeFreq& freq, const T* qkv, T* q_out, int t0, int n, int kvh, int page, int at,
                                  double* cs, uint32_t* amax) {
  const int tid = threadIdx.x, d = a.d, half = d >> 1, ps = a.ps, pc = d / 16, group = a.nq / a.nkv;
  const size_t row_el = (size_t)(a.nq + 2 * a.nkv) * d, ph = (size_t)page * a.nkv + kvh;
  const T* rows = qkv + (size_t)t0 * row_el;
  const size_t v_col = (size_t)(a.nq + a.nkv + kvh) * d;
  if (tid < 2) amax[tid] = 0;
  float mk = 0.f, mv = 0.f;
  auto angles = [&](int g0, int gn) {
    __syncthreads();
    for (int i = tid; i < gn * half; i += THREADS)
      cos_sin_64(freq, i % half, a.tok_pos[t0 + g0 + i / half], &cs[i / half * d + i % half], &cs[i / half * d + half + i % half]);
    __syncthreads();
  };
  for (int g0 = 0; g0 < n; g0 += GROUP) {
    const int gn = min(GROUP, n - g0);
    angles(g0, gn);
    for (int u = tid; u < gn * group * pc; u += THREADS) {
      const int tl = u / (group * pc);
      query8(a, cs + tl * d, rows + (size_t)(g0 + tl) * row_el, q_out, t0 + g0 + tl, kvh * group + u / pc % group, u % pc * 8);
    }
    for (int u = tid; u < gn * pc; u += THREADS) {
      const int tl = u / pc, ch = u % pc * 8;
      const T* row = rows + (size_t)(g0 + tl) * row_el;
      float v[16];
      key8(a, cs + tl * d, row, kvh, ch, v, v + 8);
#pragma unroll
      for (int e = 0; e < 16; ++e) mk = fmaxf(mk, finite_abs(v[e]));
      load8(row + v_col + 2 * ch, v);
      load8(row + v_col + 2 * ch + 8, v + 8);
#pragma unroll
      for (int e = 0; e < 16; ++e) mv = fmaxf(mv, finite_abs(v[e]));
    }
  }
  atomicMax(&amax[0], __builtin_bit_cast(uint32_t, mk));
  atomicMax(&amax[1], __builtin_bit_cast(uint32_t, mv));
  __syncthreads();
  const Scales s = page_scales(a, ph, at, amax[0], amax[1]);
  __syncthreads();                       // (every thread has read the old scales)
  if (tid == 0) { a.k_scale[ph] = s.k; a.v_scale[ph] = s.v; }
  uint8_t* kc = a.k_codes + ph * ps * d;
  uint8_t* vc = a.v_codes + ph * ps * d;
  if (at)
    for (int u = tid; u < d * ps / 16; u += THREADS) {
      if (s.k > s.old_k) rescale_unit(kc, u, ps, at, n, s.old_k / s.k, true);
      if (s.v > s.old_v) rescale_unit(vc, u, ps, at, n, s.old_v / s.v, false);
    }
  __syncthreads();                       // (a unit of values may hold new positions as well)
  for (int g0 = 0; g0 < n; g0 += GROUP) {
    const int gn = min(GROUP, n - g0);
    if (n > GROUP) angles(g0, gn);
    for (int u = tid; u < gn * pc; u += THREADS) {
      const int tl = u / pc, ch = u % pc * 8;
      float v[16];
      key8(a, cs + tl * d, rows + (size_t)(g0 + tl) * row_el, kvh, ch, v, v + 8);
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int c = ch + x * half;
        *reinterpret_cast<u32x2*>(kc + ((size_t)(c / 16) * ps + at + g0 + tl) * 16 + c % 16) = encode8(v + 8 * x, 1.f / s.k);
      }
    }
    for (int u = tid; u < gn * d; u += THREADS) {
      const int tl = u / d, ch = u % d;
      const float v[4] = {kv8_storable(ld(rows + (size_t)(g0 + tl) * row_el + v_col + ch)) * (1.f / s.v), 0.f, 0.f, 0.f};
      vc[(size_t)ch * ps + at + g0 + tl] = (uint8_t)kv8_encode4(v);
    }
  }
}

// FORM 0: every run is one token, a block each.  1: pages of sixteen, head_dim up to 128; 2: any; a block per (run, kv head), runs of one
// token to the first head's.
template <typename T, int FORM>
__global__ __launch_bounds__(THREADS) void kv8_append_kernel(AppendArgs a, RopeFreq freq, const T* qkv, T* q_out) {
  extern __shared__ double cs[];              // [tokens][d] angles, then 2 nkv largest magnitudes
  const int run = FORM == 0 ? blockIdx.x : blockIdx.x / a.nkv, kvh = FORM == 0 ? 0 : blockIdx.x % a.nkv;
  const int t0 = a.runs[2 * run], n = a.runs[2 * run + 1];
  if (t0 < 0 || n < 1 || n > a.ps || t0 > a.T - n) return;              // (whole block, as below)
  const int sl = a.slot[t0], page = sl / a.ps, at = sl % a.ps;
  if (sl < 0 || page >= a.num_pages || at + n > a.ps) return;
  uint32_t* amax = reinterpret_cast<uint32_t*>(cs + (FORM == 0 ? 1 : GROUP) * a.d);
  if (n == 1) {
    if (kvh == 0) append_token(a, freq, qkv, q_out, t0, page, at, cs, amax);
  } else if constexpr (FORM == 1) {
    append_page16(a, freq, qkv, q_out, t0, n, kvh, page, at, cs, amax);
  } else if constexpr (FORM == 2) {
    append_any(a, freq, qkv, q_out, t0, n, kvh, page, at, cs, amax);
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
  const int pieces = d / 16, units = pieces * ps, n = n_tokens - i * ps;      // n: the sequence's tokens from this page on
  for (int w = threadIdx.x; w < 2 * units; w += THREADS) {
    float v[16];
    if (w < units) {
      // neighbouring threads write a key's row; it lies in pieces among the other keys'
      const int key = w / pieces, c = w % pieces;
      kv8_decode16(*reinterpret_cast<const u32x4*>(kc + ((size_t)c * ps + key) * 16), v);
#pragma unroll
      for (int e = 0; e < 16; ++e) v[e] = key < n ? v[e] * sk : 0.f;
      store8(ko + (size_t)w * 16, v);
      store8(ko + (size_t)w * 16 + 8, v + 8);
    } else {
      const int u = w - units;
      kv8_decode16(*reinterpret_cast<const u32x4*>(vc + (size_t)u * 16), v);
#pragma unroll
      for (int e = 0; e < 16; ++e) v[e] = (u * 16 + e) % ps < n ? v[e] * sv : 0.f;
      store8(vo + (size_t)u * 16, v);
      store8(vo + (size_t)u * 16 + 8, v + 8);
    }
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
  const int form = n_runs == m.T ? 0 : c.page_size == 16 && c.head_dim <= 128 ? 1 : 2;
  const dim3 grid(form == 0 ? (unsigned)n_runs : (unsigned)n_runs * c.n_kv_heads);
  const size_t shm = sizeof(double) * (form == 0 ? 1 : GROUP) * c.head_dim + sizeof(uint32_t) * 2 * c.n_kv_heads;
  if (shm > 48 * 1024) return fail(FLEXCO_EUNSUPPORTED, "8-bit append: %d kv heads of %d are too many", c.n_kv_heads, c.head_dim);
#define FLEXCO_KV8_APPEND(T_, FORM_) \
  hipLaunchKernelGGL((kv8_append_kernel<T_, FORM_>), grid, dim3(THREADS), shm, s, a, freq, (const T_*)qkv, (T_*)q_out)
  if (c.dtype == FLEXCO_BF16) {
    if (form == 0) FLEXCO_KV8_APPEND(bf16_t, 0); else if (form == 1) FLEXCO_KV8_APPEND(bf16_t, 1); else FLEXCO_KV8_APPEND(bf16_t, 2);
  } else {
    if (form == 0) FLEXCO_KV8_APPEND(float, 0); else if (form == 1) FLEXCO_KV8_APPEND(float, 1); else FLEXCO_KV8_APPEND(float, 2);
  }
#undef FLEXCO_KV8_APPEND
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
