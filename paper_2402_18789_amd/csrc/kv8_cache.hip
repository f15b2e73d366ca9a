// The 8-bit paged cache: append of a batch's tokens and pages written out again (format and rules: flexco_kv8.h).
//
// Append.  A page's scale is chosen from all of its new rows, so the rotated keys and the values of a (run, kv head) are held until
// their largest magnitude is known; whoever does that owns the page's codes of the head, so a scale that has grown is applied to the
// codes already there on the spot.  Bound by HBM for many tokens: (2 nq + 2 nkv) d activations and 2 nkv d bytes per token (4000 tokens of chunks over
// 32/8 heads 22.5 us, 4.0 TB/s), by latency for few (one 5.8 us, 512 single ones over 40/8 heads 9.1, where all of them raise their pages'
// scales about 15).
// Keys are rotated in double precision and rounded once, into the cache (an angle's fp32 error of 5e-7 moved one code in 10^5).
#include <algorithm>
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

// eight elements as they lie in memory
template <typename T> struct Raw8;
template <> struct Raw8<bf16_t> {
  bf16x8 v;
  __device__ void load(const bf16_t* p) { v = *reinterpret_cast<const bf16x8*>(p); }
  __device__ void get(float* x) const {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = (float)v[e];
  }
};
template <> struct Raw8<float> {
  f32x4 v[2];
  __device__ void load(const float* p) { v[0] = *reinterpret_cast<const f32x4*>(p); v[1] = *reinterpret_cast<const f32x4*>(p + 4); }
  __device__ void get(float* x) const {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = v[e / 4][e % 4];
  }
};

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

// Cosine and sine of an angle of pos * rev turns: the turn's distance to the nearest quarter, at most an eighth, and the Taylor series of
// both there (x <= pi / 4: what is left out is below 2e-9, and the fp32 value of a key is off by 6e-8 anyway).
__device__ inline void cos_sin_64(double rev, int pos, double* c, double* s) {
  const double r = (double)pos * rev, turn = r - floor(r), quarter = rint(4.0 * turn);
  const double x = (turn - 0.25 * quarter) * 6.283185307179586476925, y = x * x;
  const double sn = x * (1.0 + y * (-1.0 / 6 + y * (1.0 / 120 + y * (-1.0 / 5040 + y * (1.0 / 362880)))));
  const double cs = 1.0 + y * (-0.5 + y * (1.0 / 24 + y * (-1.0 / 720 + y * (1.0 / 40320 + y * (-1.0 / 3628800)))));
  const int k = (int)quarter & 3;
  const double a = k & 1 ? sn : cs, b = k & 1 ? cs : sn;
  *c = k == 1 || k == 2 ? -a : a;
  *s = k >= 2 ? -b : b;
}

// Eight pairs x, y (channels ch .. + 7 and d / 2 + ch .. + 7 of a head) turned: x c - y s, y c + x s
template <typename F>
struct Angles8 {
  F c[8], s[8];
  template <typename A>
  __device__ Angles8(const A* cs, int half, int ch) {          // cs: d / 2 cosines, then sines, of a token
#pragma unroll
    for (int e = 0; e < 8; ++e) { c[e] = (F)cs[ch + e]; s[e] = (F)cs[half + ch + e]; }
  }
  __device__ void turn(const float* x, const float* y, float* lo, float* hi) const {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const F l = (F)x[e] * c[e] - (F)y[e] * s[e], h = (F)y[e] * c[e] + (F)x[e] * s[e];
      lo[e] = (float)l;
      hi[e] = (float)h;
    }
  }
};
// Largest magnitude of sixteen elements, those that are no finite number left out; all: every one is stored as it is (kv8_storable).  (x 0
// summed is NaN where one is infinite or NaN: a multiply-add per element instead of two comparisons in the two places that ask.)
__device__ inline float largest16(const float* v, bool* all) {
  float odd = 0.f, m = 0.f;
#pragma unroll
  for (int e = 0; e < 16; ++e) odd = __builtin_fmaf(v[e], 0.f, odd);
  *all = odd == odd;
  if (*all) {
#pragma unroll
    for (int e = 0; e < 16; ++e) m = fmaxf(m, fabsf(v[e]));
  } else {
#pragma unroll
    for (int e = 0; e < 16; ++e) m = fmaxf(m, kv8_finite(v[e]) ? fabsf(v[e]) : 0.f);
  }
  *all = *all && m <= KV8_MOST;
  return m;
}

// turned queries of token t, head h, channels ch .. + 7 and d / 2 + ch .. + 7
template <typename T>
__device__ inline void put_query(const AppendArgs& a, const Angles8<float>& an, const float* x, const float* y, T* q_out, int t, int h, int ch) {
  const int half = a.d >> 1;
  float lo[8], hi[8];
  an.turn(x, y, lo, hi);
  T* o = q_out + (size_t)t * a.ld_q + (size_t)h * a.d + ch;
  store8(o, lo);
  store8(o + half, hi);
  if (t >= a.ft_tok0 && t < a.ft_tok0 + a.n_ft) {
    T* o2 = (T*)a.q_cache + ((size_t)(t - a.ft_tok0) * a.nq + h) * a.d + ch;
    store8(o2, lo);
    store8(o2 + half, hi);
  }
}
template <typename T>
__device__ inline void query8(const AppendArgs& a, const double* cs, const T* row, T* q_out, int t, int h, int ch) {
  const int half = a.d >> 1;
  float x[8], y[8];
  load8(row + (size_t)h * a.d + ch, x);
  load8(row + (size_t)h * a.d + ch + half, y);
  put_query(a, Angles8<float>(cs, half, ch), x, y, q_out, t, h, ch);
}
__device__ inline u32x2 encode8(const float* v, float inv, bool all) {
  float w[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) w[e] = v[e] * inv;
  if (!all)
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = kv8_storable(v[e]) * inv;
  return u32x2{kv8_encode4(w), kv8_encode4(w + 4)};
}
template <typename T>
__device__ inline void key8(const AppendArgs& a, const double* cs, const T* row, int kvh, int ch, float* lo, float* hi) {
  const int half = a.d >> 1;
  const T* kr = row + (size_t)(a.nq + kvh) * a.d;
  float x[8], y[8];
  load8(kr + ch, x);
  load8(kr + ch + half, y);
  Angles8<double>(cs, half, ch).turn(x, y, lo, hi);
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

// A page's scale for a run whose largest magnitude has the bits amax (LDS: the order of positive floats is that of their bits); old: the
// page's own, 0 where the run begins it
__device__ inline float new_scale(float old, uint32_t amax) { return fmaxf(old, kv8_scale_for(__builtin_bit_cast(float, amax))); }

// A run of one token: one block for all heads (a block per head had an eighth of its threads at work).  Elements are asked for before
// the angles are computed: a thread holds a piece of a key or value head and QP of query heads; what is beyond that is read later.
template <typename T, int QP>
struct TokenRow {
  float kv[16];
  Raw8<T> q[QP ? QP : 1][2];

  // piece u: sixteen channels of a value head, or of a key head before it is turned (ch .. + 7, d / 2 + ch .. + 7)
  __device__ static void load_kv(const AppendArgs& a, const T* row, int u, float* v) {
    const int pc = a.d / 16, ch = u % pc * 8;
    const T* p = row + (size_t)(a.nq + u / pc) * a.d;                // (key heads, then value heads)
    load8(p + (u < a.nkv * pc ? ch : 2 * ch), v);
    load8(p + (u < a.nkv * pc ? ch + (a.d >> 1) : 2 * ch + 8), v + 8);
  }
  __device__ void load(const AppendArgs& a, const T* row) {
    const int tid = threadIdx.x, pc = a.d / 16;
    if (tid < 2 * a.nkv * pc) load_kv(a, row, tid, kv);
#pragma unroll
    for (int i = 0; i < QP; ++i)
      if (tid + i * THREADS < a.nq * pc) {
        const T* p = row + (size_t)((tid + i * THREADS) / pc) * a.d + (tid + i * THREADS) % pc * 8;
        q[i][0].load(p);
        q[i][1].load(p + (a.d >> 1));
      }
  }
};
template <typename T>
__device__ inline const T* row_of(const AppendArgs& a, const T* qkv, int t) { return qkv + (size_t)t * (a.nq + 2 * a.nkv) * a.d; }

template <typename T, int QP>
__device__ inline void append_token(const AppendArgs& a, const RopeFreq& freq, const T* row, TokenRow<T, QP>& held, T* q_out, int t, int pos, int page,
                                    int at, double* cs, uint32_t* amax) {
  const int tid = threadIdx.x, d = a.d, half = d >> 1, pc = d / 16, nkv = a.nkv;
  float* old = reinterpret_cast<float*>(amax + 2 * nkv);             // [2 nkv]
  uint8_t* v_row = reinterpret_cast<uint8_t*>(old + 2 * nkv);        // [nkv][d] codes of the values
  const int n_kv = 2 * nkv * pc, n_q = a.nq * pc;                    // pieces: keys, then values; queries
  const size_t ph0 = (size_t)page * nkv;
  float (&kv)[16] = held.kv;
  bool all = true;
  for (int h = tid; h < 2 * nkv; h += THREADS) {
    old[h] = !at ? 0.f : h < nkv ? a.k_scale[ph0 + h] : a.v_scale[ph0 + h - nkv];
    amax[h] = 0;
  }
  for (int i = tid; i < half; i += THREADS) cos_sin_64(freq.rev[i], pos, &cs[i], &cs[half + i]);
  __syncthreads();
  auto turned_kv = [&](int u, float* v) {                           // (a key piece in its place, the rest as it is)
    if (u >= nkv * pc) return;
    float lo[8], hi[8];
    Angles8<double>(cs, half, u % pc * 8).turn(v, v + 8, lo, hi);
#pragma unroll
    for (int e = 0; e < 8; ++e) { v[e] = lo[e]; v[8 + e] = hi[e]; }
  };
  for (int u = tid; u < n_kv; u += THREADS) {
    float v[16], m;
    if (u == tid) {
      turned_kv(u, kv);
      m = largest16(kv, &all);
    } else {
      bool there;
      held.load_kv(a, row, u, v);
      turned_kv(u, v);
      m = largest16(v, &there);
    }
    atomicMax(&amax[u / pc], __builtin_bit_cast(uint32_t, m));
  }
#pragma unroll
  for (int i = 0; i < QP; ++i) {
    const int u = tid + i * THREADS, ch = u % pc * 8;
    if (u < n_q) {
      float y[16];
      held.q[i][0].get(y);
      held.q[i][1].get(y + 8);
      put_query(a, Angles8<float>(cs, half, ch), y, y + 8, q_out, t, u / pc, ch);
    }
  }
  for (int u = tid + QP * THREADS; u < n_q; u += THREADS) query8(a, cs, row, q_out, t, u / pc, u % pc * 8);
  __syncthreads();
  auto put_kv = [&](int u, const float* p, bool finite) {
    const int h = u / pc, ch = u % pc * 8;
    const size_t ph = ph0 + h % nkv;
    const float inv = 1.f / new_scale(old[h], amax[h]);
    const u32x2 w[2] = {encode8(p, inv, finite), encode8(p + 8, inv, finite)};
    if (h < nkv) {
      uint8_t* kc = a.k_codes + ph * a.ps * d;
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int c = ch + x * half;
        *reinterpret_cast<u32x2*>(kc + ((size_t)(c / 16) * a.ps + at) * 16 + c % 16) = w[x];
      }
    } else {
      u32x2* vc = reinterpret_cast<u32x2*>(v_row + (size_t)(h - nkv) * d + 2 * ch);
      vc[0] = w[0];
      vc[1] = w[1];
    }
  };
  if (tid < n_kv) put_kv(tid, kv, all);
  for (int u = tid + THREADS; u < n_kv; u += THREADS) {
    float v[16];
    held.load_kv(a, row, u, v);
    turned_kv(u, v);
    put_kv(u, v, false);
  }
  for (int h = tid; h < 2 * nkv; h += THREADS) (h < nkv ? a.k_scale : a.v_scale)[ph0 + h % nkv] = new_scale(old[h], amax[h]);
  __syncthreads();
  // A value's codes lie page_size bytes apart: neighbouring threads store neighbours, eight to a line (stored by the piece, a line to a byte,
  // 512 tokens took 11.0 us, this 9.2).
  for (int c = tid; c < nkv * d; c += THREADS) a.v_codes[(ph0 * d + c) * a.ps + at] = v_row[c];
  if (!at) return;
  __syncthreads();                       // (a unit of values holds the new position as well)
  const int units = d * a.ps / 16;
  for (int h = tid >> 6; h < 2 * nkv; h += THREADS / 64) {           // a wavefront per head
    const float s = new_scale(old[h], amax[h]);
    if (!(s > old[h])) continue;
    for (int u = tid & 63; u < units; u += 64)
      rescale_unit((h < nkv ? a.k_codes : a.v_codes) + (ph0 + h % nkv) * a.ps * d, u, a.ps, at, 1, old[h] / s, h < nkv);
  }
}

// A run's page of sixteen positions, head_dim 16 PC up to 128: half the block's threads hold the keys, half the values, sixteen elements
// each, from their load to their codes, which go to memory through an image of the page in LDS: 16 bytes at a time.  A thread's queries
// are those of its position and channels, so that it reads their angles once.
template <typename T, int PC>
__device__ inline void append_page16(const AppendArgs& a, const RopeFreq& freq, const T* qkv, T* q_out, int t0, int n, int kvh, int page,
                                     int at, float* cs, uint32_t* amax) {
  __shared__ __attribute__((aligned(16))) uint8_t image[2][16 * 16 * PC];
  constexpr int d = 16 * PC, half = d / 2;
  const int tid = threadIdx.x, group = a.nq / a.nkv;
  const size_t row_el = (size_t)(a.nq + 2 * a.nkv) * d, ph = (size_t)page * a.nkv + kvh;
  const bool keys = tid < THREADS / 2;
  const int u = tid % (THREADS / 2), tl = u / PC, ch = u % PC * 8;
  const bool mine = u < n * PC;
  const T* row = qkv + (size_t)(t0 + (mine ? tl : 0)) * row_el;
  // (everything that needs nothing but the run is asked for before the angles)
  float x[16];
  Raw8<T> q0, q1;
  const T* src = row + (size_t)(keys ? a.nq + kvh : a.nq + a.nkv + kvh) * d;
  load8(src + (keys ? ch : 2 * ch), x);
  load8(src + (keys ? ch + half : 2 * ch + 8), x + 8);
  const T* qrow = row + (size_t)(kvh * group) * d + ch;
  const int h0 = keys ? 1 : 0;                 // every other query head, the value half's share the larger
  if (h0 < group) {
    q0.load(qrow + h0 * d);
    q1.load(qrow + h0 * d + half);
  }
  const float old_k = at ? a.k_scale[ph] : 0.f, old_v = at ? a.v_scale[ph] : 0.f;
  if (tid < 2) amax[tid] = 0;
  // a key's thread computes the angles of its position and channels, in double precision for the key, and leaves them for the queries
  float m = 0.f;
  bool all = true;
  if (mine) {
    if (keys) {
      const int pos = a.tok_pos[t0] + tl;                            // (a run's positions follow one another)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        double c, sn;
        cos_sin_64(freq.rev[ch + e], pos, &c, &sn);
        const double lo = x[e] * c - x[8 + e] * sn, hi = x[8 + e] * c + x[e] * sn;
        x[e] = (float)lo;
        x[8 + e] = (float)hi;
        cs[tl * d + ch + e] = (float)c;
        cs[tl * d + half + ch + e] = (float)sn;
      }
    }
    m = largest16(x, &all);
  }
  __syncthreads();
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
  if ((tid & 63) == 0) atomicMax(&amax[keys ? 0 : 1], __builtin_bit_cast(uint32_t, m));
  if (mine) {
    const Angles8<float> an(cs + tl * d, half, ch);
    for (int h = h0; h < group; h += 2) {
      float y[16];
      q0.get(y);
      q1.get(y + 8);
      if (h + 2 < group) {
        q0.load(qrow + (h + 2) * d);
        q1.load(qrow + (h + 2) * d + half);
      }
      put_query(a, an, y, y + 8, q_out, t0 + tl, kvh * group + h, ch);
    }
  }
  __syncthreads();
  const float s_k = new_scale(old_k, amax[0]), s_v = new_scale(old_v, amax[1]);
  if (tid == 0) { a.k_scale[ph] = s_k; a.v_scale[ph] = s_v; }
  if (mine) {
    const float inv = 1.f / (keys ? s_k : s_v);
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      const u32x2 w = encode8(x + 8 * y, inv, all);
      if (keys) {
        const int c = ch + y * half;
        *reinterpret_cast<u32x2*>(&image[0][(c / 16 * 16 + at + tl) * 16 + c % 16]) = w;
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) image[1][(2 * ch + 8 * y + e) * 16 + at + tl] = (uint8_t)(w[e / 4] >> (8 * (e % 4)));
      }
    }
  }
  __syncthreads();
  // a unit: sixteen channels of a position (keys), sixteen positions of a channel (values)
  if (u >= PC * 16) return;
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
      cos_sin_64(freq.rev[i % half], a.tok_pos[t0 + g0 + i / half], &cs[i / half * d + i % half], &cs[i / half * d + half + i % half]);
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
      bool all;
      key8(a, cs + tl * d, row, kvh, ch, v, v + 8);
      mk = fmaxf(mk, largest16(v, &all));
      load8(row + v_col + 2 * ch, v);
      load8(row + v_col + 2 * ch + 8, v + 8);
      mv = fmaxf(mv, largest16(v, &all));
    }
  }
  atomicMax(&amax[0], __builtin_bit_cast(uint32_t, mk));
  atomicMax(&amax[1], __builtin_bit_cast(uint32_t, mv));
  __syncthreads();
  const float old_k = at ? a.k_scale[ph] : 0.f, old_v = at ? a.v_scale[ph] : 0.f;
  const float s_k = new_scale(old_k, amax[0]), s_v = new_scale(old_v, amax[1]);
  __syncthreads();                       // (every thread has read the old scales)
  if (tid == 0) { a.k_scale[ph] = s_k; a.v_scale[ph] = s_v; }
  uint8_t* kc = a.k_codes + ph * ps * d;
  uint8_t* vc = a.v_codes + ph * ps * d;
  if (at)
    for (int u = tid; u < d * ps / 16; u += THREADS) {
      if (s_k > old_k) rescale_unit(kc, u, ps, at, n, old_k / s_k, true);
      if (s_v > old_v) rescale_unit(vc, u, ps, at, n, old_v / s_v, false);
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
        *reinterpret_cast<u32x2*>(kc + ((size_t)(c / 16) * ps + at + g0 + tl) * 16 + c % 16) = encode8(v + 8 * x, 1.f / s_k, false);
      }
    }
    for (int u = tid; u < gn * d; u += THREADS) {
      const int tl = u / d, ch = u % d;
      const float v[4] = {kv8_storable(ld(rows + (size_t)(g0 + tl) * row_el + v_col + ch)) * (1.f / s_v), 0.f, 0.f, 0.f};
      vc[(size_t)ch * ps + at + g0 + tl] = (uint8_t)kv8_encode4(v);
    }
  }
}

// FORM 0: every run is one token or outside the batch, a block each.  Else a block per (run, kv head), runs of one token to one of them; FORM 4, 8: pages of
// sixteen, head_dim 16 FORM; 1: any.
template <typename T, int FORM>
__global__ __launch_bounds__(THREADS) void kv8_append_kernel(AppendArgs a, RopeFreq freq, const T* qkv, T* q_out) {
  // angles [tokens][d] (pages of sixteen: fp32), then largest magnitudes: two, or of a single token 2 nkv with as many old scales and nkv d codes
  extern __shared__ double cs[];
  const int run = FORM == 0 ? blockIdx.x : blockIdx.x / a.nkv, kvh = FORM == 0 ? 0 : blockIdx.x % a.nkv;
  constexpr int QP = FORM == 0 ? 2 : 0;
  TokenRow<T, QP> held;
  int sl = 0, pos = 0;
  // (a single token each and as many runs: run i is token i unless the caller has put them in an order of their own, so that its row, slot and position are asked
  // for along with the run itself: one token, a launch of its own 7.8 -> 7.2 us, 512 11.6 -> 11.2)
  if (FORM == 0) {
    held.load(a, row_of(a, qkv, run));
    sl = a.slot[run];
    pos = a.tok_pos[run];
  }
  const int t0 = a.runs[2 * run], n = a.runs[2 * run + 1];
  if (t0 < 0 || n < 1 || n > a.ps || t0 > a.T - n) return;              // (whole block, as below)
  // (by turns: the blocks of one head all run on one part of the chip.  309 tokens beside 87 of chunks, 8 kv heads: 16.7 us there, 11.3 by turns.)
  if (FORM != 0 && n == 1 && kvh != run % a.nkv) return;
  if (FORM != 0 || t0 != run) sl = a.slot[t0];
  const int page = sl / a.ps, at = sl % a.ps;
  if (sl < 0 || page >= a.num_pages || at + n > a.ps) return;
  uint32_t* amax = reinterpret_cast<uint32_t*>(cs + (n == 1 ? 1 : FORM == 1 ? GROUP : GROUP / 2) * a.d);
  if (n == 1) {
    const T* row = row_of(a, qkv, t0);
    if (FORM != 0 || t0 != run) {
      held.load(a, row);
      pos = a.tok_pos[t0];
    }
    append_token<T, QP>(a, freq, row, held, q_out, t0, pos, page, at, cs, amax);
  } else if constexpr (FORM >= 4) {
    append_page16<T, FORM>(a, freq, qkv, q_out, t0, n, kvh, page, at, reinterpret_cast<float*>(cs), amax);
  } else if constexpr (FORM == 1) {
    append_any(a, freq, qkv, q_out, t0, n, kvh, page, at, cs, amax);
  }
}

// Expand.  One block per (page, kv head): 2 d ps codes in, as many elements out, keys beside values so that a page of 16 x 128 is one unit of
// sixteen codes a thread.  Bound by HBM: 32749 tokens of 8 x 128 to bf16 46 us, 4.3 TB/s; 2048 tokens 5.1 us, a launch's time.
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
  // (as many runs as tokens are not enough for form 0, which takes single tokens alone: places of a list may be free, runs outside the batch.  A token
  // per request, or per page, is.)
  const bool single_tokens = n_runs == m.T && (m.n_req == m.T || c.page_size == 1);
  const int form = single_tokens ? 0 : c.page_size == 16 && c.head_dim == 128 ? 8 : c.page_size == 16 && c.head_dim == 64 ? 4 : 1;
  const dim3 grid(form == 0 ? (unsigned)n_runs : (unsigned)n_runs * c.n_kv_heads);
  // (a block holds a single token or a run of several, and either lies where the other would; kv8_append_token_lds is checked by the entry points)
  const size_t several = form == 0 ? 0 : sizeof(double) * (form == 1 ? GROUP : GROUP / 2) * c.head_dim + 2 * sizeof(uint32_t);
  const size_t shm = std::max(kv8_append_token_lds(c), several);
#define FLEXCO_KV8_APPEND(T_, FORM_) \
  hipLaunchKernelGGL((kv8_append_kernel<T_, FORM_>), grid, dim3(THREADS), shm, s, a, freq, (const T_*)qkv, (T_*)q_out)
#define FLEXCO_KV8_APPEND_FORMS(T_)                  \
  if (form == 0) FLEXCO_KV8_APPEND(T_, 0);           \
  else if (form == 8) FLEXCO_KV8_APPEND(T_, 8);      \
  else if (form == 4) FLEXCO_KV8_APPEND(T_, 4);      \
  else FLEXCO_KV8_APPEND(T_, 1);
  if (c.dtype == FLEXCO_BF16) { FLEXCO_KV8_APPEND_FORMS(bf16_t) } else { FLEXCO_KV8_APPEND_FORMS(float) }
#undef FLEXCO_KV8_APPEND_FORMS
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
