// Attention over the 8-bit cache on the matrix cores: bf16 activations, head_dim 128, page_size 16, at most 16 query heads per kv
// head (any other shape: kv8_attn_generic.hip).  Work list, partial rows and merge are those of the 16-bit kernels.
//
// A column is a (token, query head) pair, a tile sixteen of them over one kv head.  Codes are widened to bf16 in registers, by
// conversions that multiply by their page's scale on the way, a power of two: code x scale is a bf16 number, so nothing is rounded there,
// and from then on the products are those of a 16-bit cache.  Single tokens (v_mfma_f32_16x16x32_bf16; chunks: below):
//   S^T[key, col] = K[key, :] . Q[col, :]^T         A = a K page (16 keys), lane (key, g): channels 16 g .. + 15 and 64 + 16 g .. + 15
//   O^T[d, col] += V^T[d, keys] . P^T[keys, col]    A = V rows as they lie, lane (d = lane % 16, g): the 16 keys of the g-th of four pages
// (The 8-bit products of the chip, with the other operand as the sum of two e4m3 numbers, need no conversion and were tried first:
// they drop what lies 2^-13 below the largest product of a sum, and scores came out 1e-5 off.)
// A lane (col = lane % 16, g = lane / 16) gets keys 4 g .. 4 g + 3 of each page from the first product and supplies page g's sixteen
// keys of four pages to the second: eight words change places between the rows of lanes, by swaps of halves and of pairs.
// Scores, running maxima and sums, and the products' sums are fp32.  Probabilities are rounded to bf16 for the second product, as the 16-bit cache's
// are, and summed unrounded: a row is off by 2^-8 of its sum of p |v| at most, on the order of the output's storage (outputs 0.0020 - 0.0022 from
// 64 bits, relative to their norm, the storage alone 0.0016 - 0.0017).  Two bf16 terms of each would double that product's instructions.
//
// Key positions behind a column's own are masked in the scores, and what lies in V at such positions never meets the sums: slots
// behind the item's last position are cleared, and a NaN code between (a later token of the same chunk) is taken out and
// given to the columns that see it only.
#include <algorithm>
#include "attn_plan.h"
#include "flexco_internal.h"
#include "kv8_codes.h"
#include "kv8_internal.h"
#include "kv8_plan.h"

namespace flexco {

namespace {

constexpr int D = 128, PS = 16;
constexpr int PAGE = PS * D;             // bytes of one K (or V) block of a page and head
constexpr int MAXSP = KV8_MAX_PAGES;     // pages of a block's key range at most
constexpr int SP = 4;                    // pages of a step
constexpr int CHUNK_NW = 2;              // wavefronts of a chunk's block
constexpr float NO_KEY = -3.402823466e38f;   // the maximum of no key yet: finite, so that a masked score less this is still -inf
constexpr float MOST = 256.f;            // the most that a lane's exponentials of a step may come to before the reference point follows the maximum
#define FLEXCO_GP(p) ((const __attribute__((address_space(1))) void*)(p))
#define FLEXCO_LP(p) ((__attribute__((address_space(3))) void*)(p))

struct Args {
  const int32_t *tok_pos, *block_table, *tile_req, *tile_tok0, *tile_ntok, *tile_nsplit, *tile_part0, *item_tile,
      *item_split, *item_ntiles, *req_tok_off;
  int max_pages, nq, nkv, n_items, split_pages, fold;
  bool whole;         // fold holds for every request, not for those of one token alone
  float scale_log2;   // log2(e) / sqrt(d)
  const bf16_t* q;
  size_t ldq;
  const uint8_t *k_codes, *v_codes;
  const float *k_scale, *v_scale;
  float *part_ml, *part_acc;
  bf16_t* out;
  size_t ldo;
  float* lse;         // or NULL
  AttnKeep keep;
};

// sixteen codes times a power of two
__device__ inline void widen(const u32x4& w, float s, bf16x8& lo, bf16x8& hi) {
  bf16x2 t[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    t[2 * i] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w[i], s, false);
    t[2 * i + 1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w[i], s, true);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    lo[2 * i] = t[i][0]; lo[2 * i + 1] = t[i][1];
    hi[2 * i] = t[4 + i][0]; hi[2 * i + 1] = t[4 + i][1];
  }
}

// lane (col, g): words of pages 0 .. 3  ->  page g's words of lanes (col, 0 .. 3)
__device__ inline void turn_words(uint32_t* w) {
  const auto a = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false);
  const auto b = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
  const auto c = __builtin_amdgcn_permlane16_swap(a[0], b[0], false, false);
  const auto e = __builtin_amdgcn_permlane16_swap(a[1], b[1], false, false);
  w[0] = c[0]; w[1] = c[1]; w[2] = e[0]; w[3] = e[1];
}

__device__ inline uint32_t has_nan(uint32_t w) { return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }   // bit 7 of bytes 0x7f, 0xff
__device__ inline uint32_t bytes_of(uint32_t bits, uint32_t value) { return (bits >> 7) * value; }            // value in those bytes
// mask of the first n (clamped to 0 .. 4) bytes of a word
__device__ inline uint32_t first_bytes(int n) { return n >= 4 ? 0xffffffffu : n <= 0 ? 0u : (1u << (8 * n)) - 1u; }

// Running state of a tile's column, the same in its four lanes but for l (each lane's own keys).
struct Column {
  bf16x8 q[4];        // channels 16 g .. + 7, + 8 .. + 15, 64 + 16 g .. + 7, + 8 .. + 15
  float m, l;         // reference point of the exponentials (log2), sum of exp2(s - m)
  f32x4 o[8];         // d = 16 mt + 4 g + j: sum of exp2(s - m) v

  __device__ void start(const bf16_t* qr, int g) {
#pragma unroll
    for (int i = 0; i < 4; ++i) q[i] = *reinterpret_cast<const bf16x8*>(qr + (i >> 1) * 64 + g * 16 + (i & 1) * 8);
    m = NO_KEY;
    l = 0.f;
#pragma unroll
    for (int mt = 0; mt < 8; ++mt) o[mt] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  // raw scores of a page
  __device__ f32x4 scores(const bf16x8 (&k)[4]) const {
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 4; ++i) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[i], q[i], acc, 0, 0, 0);
    return acc;
  }
  // Softmax of the raw scores of a step's four pages in three parts.  Any reference point gives the same row in the end: it stays where it
  // is unless a lane's sixteen exponentials come to more than MOST (or NaN), and the largest score is looked for only then.
  __device__ float exponentials(const f32x4 (&acc)[SP], float scale_log2, f32x4 (&p)[SP]) const {
    float sum[SP];
#pragma unroll
    for (int n = 0; n < SP; ++n) {
#pragma unroll
      for (int j = 0; j < 4; ++j) p[n][j] = __builtin_amdgcn_exp2f(__builtin_fmaf(acc[n][j], scale_log2, -m));
      sum[n] = (p[n][0] + p[n][1]) + (p[n][2] + p[n][3]);
    }
    return (sum[0] + sum[1]) + (sum[2] + sum[3]);
  }
  __device__ void follow(const f32x4 (&acc)[SP], float scale_log2) {
    float mx = acc[0][0];
#pragma unroll
    for (int n = 0; n < SP; ++n)
#pragma unroll
      for (int j = 0; j < 4; ++j) mx = fmaxf(mx, acc[n][j]);
    const float m_new = fmaxf(m, max_xor32(max_xor16(mx)) * scale_log2), alpha = __builtin_amdgcn_exp2f(m - m_new);
    m = m_new;
    l *= alpha;
#pragma unroll
    for (int mt = 0; mt < 8; ++mt)
#pragma unroll
      for (int j = 0; j < 4; ++j) o[mt][j] *= alpha;
  }
  // the probabilities as the second product takes them
  __device__ static void turn(const f32x4 (&p)[SP], bf16x8& p0, bf16x8& p1) {
    uint32_t w0[SP], w1[SP];
#pragma unroll
    for (int n = 0; n < SP; ++n) {
      const bf16x2 a = {(bf16_t)p[n][0], (bf16_t)p[n][1]}, b = {(bf16_t)p[n][2], (bf16_t)p[n][3]};
      w0[n] = __builtin_bit_cast(uint32_t, a);
      w1[n] = __builtin_bit_cast(uint32_t, b);
    }
    turn_words(w0);                          // word j: keys 4 j, 4 j + 1 of the lane's page ...
    turn_words(w1);                          // ... and 4 j + 2, 4 j + 3
    p0 = __builtin_bit_cast(bf16x8, u32x4{w0[0], w1[0], w0[1], w1[1]});
    p1 = __builtin_bit_cast(bf16x8, u32x4{w0[2], w1[2], w0[3], w1[3]});
  }
  __device__ void add(int mt, const bf16x8& v0, const bf16x8& v1, const bf16x8& p0, const bf16x8& p1) {
    o[mt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v0, p0, o[mt], 0, 0, 0);
    o[mt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v1, p1, o[mt], 0, 0, 0);
  }
};

// The row of a column whose whole key range has been summed, or its partial row: n4 groups of four channels dd, dd + stride, ...
__device__ inline void write_column(const Args& a, int tile, int split, int fold, int kvh, int group, int c, int dd, const float* row4,
                                    int n4, int stride, float m, float lsum, bool first) {
  const int cpt = (16 / group > 1 ? 16 / group : 1) * group;
  // (a piece without a visible key is one whose sum is zero: NaN scores leave m where it was too, and their NaN has to get past the join)
  const float mn = m == NO_KEY && lsum == 0.f ? -INFINITY : m * 0.6931471805599453f;
  if (a.tile_nsplit[tile] <= fold) {
    const int t = a.tile_tok0[tile] + c / group, h = kvh * group + c % group;
    const float inv = 1.0f / lsum;
    bf16_t* po = a.out + (size_t)t * a.ldo + h * D + dd;
    const bool kept = a.keep.lse2 && t >= a.keep.tok0 && t < a.keep.tok0 + a.keep.n;
    bf16_t* p2 = kept ? (bf16_t*)a.keep.out2 + ((size_t)(t - a.keep.tok0) * a.nq + h) * D + dd : nullptr;
#pragma unroll
    for (int i = 0; i < n4; ++i) {
      bf16x4 v;
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = (bf16_t)(row4[4 * i + j] * inv);
      *reinterpret_cast<bf16x4*>(po + i * stride) = v;
      if (kept) *reinterpret_cast<bf16x4*>(p2 + i * stride) = v;
    }
    if (first) {
      const float z = mn + __logf(lsum);
      if (a.lse) a.lse[(size_t)t * a.nq + h] = z;
      if (kept) a.keep.lse2[(size_t)(t - a.keep.tok0) * a.nq + h] = z;
    }
    return;
  }
  const size_t idx = ((size_t)(a.tile_part0[tile] + split) * a.nkv + kvh) * cpt + c;
  if (first) {
    a.part_ml[idx * 2] = mn;
    a.part_ml[idx * 2 + 1] = lsum;
  }
  float* pa = a.part_acc + idx * D + dd;
#pragma unroll
  for (int i = 0; i < n4; ++i) *reinterpret_cast<f32x4*>(pa + i * stride) = f32x4{row4[4 * i], row4[4 * i + 1], row4[4 * i + 2], row4[4 * i + 3]};
}

// What a block keeps in LDS beside its tiles: the pages of its key range.
struct Tables {
  int page[MAXSP];
  float ks[MAXSP], vs[MAXSP];
};

// ---- single tokens -------------------------------------------------------------------------------------------
// Bound by the codes' way from HBM (256 requests of 512 - 4096 keys over 32/8 heads, 1.21 GB: 212 us, 5.7 TB/s).  The wavefronts of a block take its pages four at a time in turn, straight into registers (a
// page's K block in two whole KB, four pages' V rows of 16 bytes), the next four on their way while one set is multiplied, and
// add up in LDS at the end: no barrier holds the stream.  Sixteen columns are one product's width; a token has as many as its
// group has heads, and the matrix cores time to spare.
struct TokenLds {
  float* o;                // sums [wavefronts][16][D]
  float (*m)[16], (*l)[16];
  // four channels of a column (turned from column to column, so that sixteen of them written at once lie in all banks)
  __device__ float* at(int wave, int c, int d) const { return o + (wave * 16 + c) * D + ((d + 4 * c) & (D - 1)); }
};

template <int NW, typename Scales>
__device__ inline void token_block(const Args& a, const Tables& tab, const TokenLds& sh, int tile, int split, int fold, int kvh, int npg, int keys,
                                   Scales&& keep_scales) {
  const int tid = threadIdx.x, lane = tid & 63, c = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int group = a.nq / a.nkv, t = a.tile_tok0[tile];
  const bool col_ok = c < group;
  Column col;
  col.start(a.q + (size_t)t * a.ldq + (size_t)(kvh * group + (col_ok ? c : 0)) * D, g);
  const int n_steps = (npg + SP - 1) / SP;

  auto load = [&](int st, u32x4 (&k)[2 * SP], u32x4 (&v)[8]) {
    st = min(st, n_steps - 1);
#pragma unroll
    for (int n = 0; n < SP; ++n) {
      const size_t page = (size_t)__builtin_amdgcn_readfirstlane(tab.page[min(SP * st + n, npg - 1)]);
      const uint8_t* kb = a.k_codes + (page * a.nkv + kvh) * (size_t)PAGE + lane * 16;
      k[2 * n] = *reinterpret_cast<const u32x4*>(kb);
      k[2 * n + 1] = *reinterpret_cast<const u32x4*>(kb + 1024);
    }
    const uint8_t* vb = a.v_codes + ((size_t)tab.page[min(SP * st + g, npg - 1)] * a.nkv + kvh) * (size_t)PAGE + c * 16;
#pragma unroll
    for (int mt = 0; mt < 8; ++mt) v[mt] = *reinterpret_cast<const u32x4*>(vb + mt * 256);
  };
  auto step = [&](int st, const u32x4 (&k)[2 * SP], u32x4 (&v)[8]) {
    f32x4 acc[SP];
#pragma unroll
    for (int n = 0; n < SP; ++n) {
      const float ks = tab.ks[min(SP * st + n, npg - 1)];
      bf16x8 kf[4];
      widen(k[2 * n], ks, kf[0], kf[1]);
      widen(k[2 * n + 1], ks, kf[2], kf[3]);
      acc[n] = col.scores(kf);
    }
    if (SP * (st + 1) * PS > keys) {                         // the last pages: slots behind the token's position
#pragma unroll
      for (int n = 0; n < SP; ++n)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if ((SP * st + n) * PS + 4 * g + j >= keys) acc[n][j] = -INFINITY;
      const int left = keys - (SP * st + g) * PS;            // of the page whose V rows this lane holds
#pragma unroll
      for (int mt = 0; mt < 8; ++mt)
#pragma unroll
        for (int i = 0; i < 4; ++i) v[mt][i] &= first_bytes(left - 4 * i);
    }
    bf16x8 p0, p1;
    f32x4 p[SP];
    float sum = col.exponentials(acc, a.scale_log2, p);
    if (__builtin_amdgcn_ballot_w64(!(sum <= MOST)) != 0) {
      col.follow(acc, a.scale_log2);
      sum = col.exponentials(acc, a.scale_log2, p);
    }
    col.l += sum;
    Column::turn(p, p0, p1);
    const float vs = tab.vs[min(SP * st + g, npg - 1)];
#pragma unroll
    for (int mt = 0; mt < 8; ++mt) {
      bf16x8 v0, v1;
      widen(v[mt], vs, v0, v1);
      col.add(mt, v0, v1, p0, p1);
    }
  };
  // (past the last step the loads repeat it, unused: as many are on their way on every path)
  u32x4 k0[2 * SP], k1[2 * SP], v0[8], v1[8];
  load(wave, k0, v0);
  keep_scales();
  if (wave < n_steps) {
    for (int st = wave; st < n_steps; st += 2 * NW) {
      load(st + NW, k1, v1);
      step(st, k0, v0);
      load(st + 2 * NW, k0, v0);
      if (st + NW < n_steps) step(st + NW, k1, v1);
    }
  }
  const float lsum = sum_xor32(sum_xor16(col.l));
  if (col_ok) {
#pragma unroll
    for (int mt = 0; mt < 8; ++mt) *reinterpret_cast<f32x4*>(sh.at(wave, c, 16 * mt + 4 * g)) = col.o[mt];
    if (g == 0) { sh.m[wave][c] = col.m; sh.l[wave][c] = lsum; }
  }
  __syncthreads();
  // 32 threads per column
  const int dd = (tid & 31) * 4;
  for (int cc = tid >> 5; cc < group; cc += 2 * NW) {
    float M = sh.m[0][cc];
#pragma unroll
    for (int w = 1; w < NW; ++w) M = fmaxf(M, sh.m[w][cc]);
    float L = 0.f, row[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float e = __builtin_amdgcn_exp2f(sh.m[w][cc] - M);
      L += sh.l[w][cc] * e;
      const f32x4 v = *reinterpret_cast<const f32x4*>(sh.at(w, cc, dd));
#pragma unroll
      for (int j = 0; j < 4; ++j) row[j] += v[j] * e;
    }
    write_column(a, tile, split, fold, kvh, group, cc, dd, row, 1, 0, M, L, (tid & 31) == 0);
  }
}

// ---- chunks --------------------------------------------------------------------------------------------------
// Bound by vector instructions beside the products (conversions and exponentials: issued on 57 % of the cycles, matrix pipes busy on 39 %), and
// by the card's power where launches follow each other: 4096 new tokens over 40/8 heads (171 GFLOP, 142 us at a large product's rate)
// 200 - 216 us on several cards, 177 with codes and queries of zeros.  Each of the block's two wavefronts takes two tiles as 32 columns; the pages of a step lie once in LDS for
// both, as they lie in memory, and the next step's are on their way meanwhile.  v_mfma_f32_32x32x16_bf16:
//   S^T[key, col]: A = two K pages, lane (r = lane % 32, h = lane / 32): channels 32 i + 16 h .. + 15, two products' worth, of the key in
//                  slot (r with bits 2 and 3 exchanged) % 16 of page r / 16
//   O^T[d, col]:   A = V rows of a page, lane (d = lane % 32, h): slots 8 h .. + 7, which with the exchange are the keys whose
//                  scores a lane (col, h) has got: no word changes places
// (The 16x16x32 form has the same rate, but every product takes 7 cycles of the vector instructions' time, and it needs twice as
// many: two wavefronts of a SIMD spend 105 ns on eight of them with four conversions each, 76 on four of this form with eight each.  The
// kernel in that form 204 us in a row of launches and 241 in one of its own, in this 200 and 223.)
struct StepLds {
  uint8_t k[SP * PAGE], v[SP * PAGE];
};

__device__ inline void load_step(const Args& a, const Tables& tab, StepLds& to, int st, int kvh, int npg, int wave, int lane) {
#pragma unroll
  for (int x = 0; x < SP / CHUNK_NW; ++x) {
    const int n = CHUNK_NW * x + wave;                                                    // this wavefront's page
    const size_t page = (size_t)__builtin_amdgcn_readfirstlane(tab.page[min(SP * st + n, npg - 1)]);
    const uint8_t* kb = a.k_codes + (page * a.nkv + kvh) * (size_t)PAGE + lane * 16;
    const uint8_t* vb = a.v_codes + (page * a.nkv + kvh) * (size_t)PAGE + lane * 16;
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      __builtin_amdgcn_global_load_lds(FLEXCO_GP(kb + y * 1024), FLEXCO_LP(to.k + n * PAGE + y * 1024), 16, 0, 0);
      __builtin_amdgcn_global_load_lds(FLEXCO_GP(vb + y * 1024), FLEXCO_LP(to.v + n * PAGE + y * 1024), 16, 0, 0);
    }
  }
}

constexpr int TILES = FLEXCO_ATTN_ITEM_TILES / CHUNK_NW;      // of a wavefront
static_assert(TILES == 2, "two tiles are a product's 32 columns");

// Running state of a lane's column (col = lane % 32), half of its channels, the sums of its own keys.
struct Wide {
  bf16x8 q[8];        // channels 32 i + 16 h .. + 7, + 8 .. + 15
  float m, l;
  f32x16 o[4];        // d = 32 mt + 8 b + 4 h + j in 4 b + j

  __device__ void start(const bf16_t* qr, int h, bool used) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const u32x4 w = *reinterpret_cast<const u32x4*>(qr + (i >> 1) * 32 + h * 16 + (i & 1) * 8);
      q[i] = __builtin_bit_cast(bf16x8, used ? w : u32x4{0, 0, 0, 0});       // (products of zeros draw less power)
    }
    m = NO_KEY;
    l = 0.f;
#pragma unroll
    for (int mt = 0; mt < 4; ++mt)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[mt][i] = 0.f;
  }
  __device__ float exponentials(const f32x16 (&acc)[2], float scale_log2, f32x16 (&p)[2]) const {
    float sum[8];
#pragma unroll
    for (int n = 0; n < 8; ++n) {
      const int x = n >> 2, i = 4 * (n & 3);
#pragma unroll
      for (int j = 0; j < 4; ++j) p[x][i + j] = __builtin_amdgcn_exp2f(__builtin_fmaf(acc[x][i + j], scale_log2, -m));
      sum[n] = (p[x][i] + p[x][i + 1]) + (p[x][i + 2] + p[x][i + 3]);
    }
    return ((sum[0] + sum[1]) + (sum[2] + sum[3])) + ((sum[4] + sum[5]) + (sum[6] + sum[7]));
  }
  __device__ void follow(const f32x16 (&acc)[2], float scale_log2) {
    float mx = acc[0][0];
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int i = 0; i < 16; ++i) mx = fmaxf(mx, acc[x][i]);
    const float m_new = fmaxf(m, max_xor32(mx) * scale_log2), alpha = __builtin_amdgcn_exp2f(m - m_new);
    m = m_new;
    l *= alpha;
#pragma unroll
    for (int mt = 0; mt < 4; ++mt)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[mt][i] *= alpha;
  }
};

__device__ inline bf16x8 widen8(uint32_t w0, uint32_t w1, float s) {
  const bf16x2 t[4] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w0, s, false), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w0, s, true),
                       __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w1, s, false), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w1, s, true)};
  bf16x8 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) { r[2 * i] = t[i][0]; r[2 * i + 1] = t[i][1]; }
  return r;
}

// EDGE: a key of the step may lie behind some column's position or the block's range (else no mask, no clearing).  pos: the column's own
// position (-1: no column), end: one past the item's last, both relative to the block's key range
template <bool EDGE>
__device__ inline void chunk_step(float scale_log2, const Tables& tab, const StepLds& in, Wide& col, int st, int npg, int pos, int end,
                                  int lane) {
  const int r = lane & 31, h = lane >> 5;
  const int k0 = SP * st * PS;
  f32x16 acc[2];
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    const int n = 2 * x + (r >> 4);
    const float ks = tab.ks[EDGE ? min(SP * st + n, npg - 1) : SP * st + n];
    const uint8_t* krow = in.k + n * PAGE + h * 256 + ((r & 3) | (r & 4) << 1 | (r & 8) >> 1) * 16;
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[x][i] = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      bf16x8 lo, hi;
      widen(*reinterpret_cast<const u32x4*>(krow + i * 512), ks, lo, hi);
      acc[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(lo, col.q[2 * i], acc[x], 0, 0, 0);
      acc[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(hi, col.q[2 * i + 1], acc[x], 0, 0, 0);
    }
  }
  if constexpr (EDGE) {
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int key = k0 + (2 * x + (i >> 3)) * PS + 8 * h + (i & 7);
        if (key > pos || key >= npg * PS) acc[x][i] = -INFINITY;
      }
  }
  f32x16 p[2];
  float sum = col.exponentials(acc, scale_log2, p);
  if (__builtin_amdgcn_ballot_w64(!(sum <= MOST)) != 0) {
    col.follow(acc, scale_log2);
    sum = col.exponentials(acc, scale_log2, p);
  }
  col.l += sum;
  bf16x8 pb[SP];
#pragma unroll
  for (int n = 0; n < SP; ++n)
#pragma unroll
    for (int i = 0; i < 8; ++i) pb[n][i] = (bf16_t)p[n >> 1][8 * (n & 1) + i];
  // slots behind the item's last position are cleared; NaN codes before it are taken out, and a product of their places with the
  // places that a column sees says whose rows they belong in
  const uint8_t* vrow = in.v + r * 16 + h * 8;
  const int limit = min(end, npg * PS) - k0 - 8 * h;
  uint32_t odd = 0;
#pragma unroll
  for (int n = 0; n < SP; ++n) {
    const float vs = tab.vs[EDGE ? min(SP * st + n, npg - 1) : SP * st + n];
#pragma unroll
    for (int mt = 0; mt < 4; ++mt) {
      u32x2 w = *reinterpret_cast<const u32x2*>(vrow + n * PAGE + mt * 512);
      if constexpr (EDGE) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          w[i] &= first_bytes(limit - n * PS - 4 * i);
          const uint32_t nan = has_nan(w[i]);
          odd |= nan;
          w[i] &= ~bytes_of(nan, 0xffu);
        }
      }
      col.o[mt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen8(w[0], w[1], vs), pb[n], col.o[mt], 0, 0, 0);
    }
  }
  if constexpr (EDGE) {
    if (__builtin_amdgcn_ballot_w64(odd != 0) == 0) return;
    bf16x8 seen[SP];
#pragma unroll
    for (int n = 0; n < SP; ++n)
#pragma unroll
      for (int i = 0; i < 8; ++i) seen[n][i] = (bf16_t)(k0 + n * PS + 8 * h + i <= pos ? 1.f : 0.f);
#pragma unroll
    for (int mt = 0; mt < 4; ++mt) {
      f32x16 hits;
#pragma unroll
      for (int i = 0; i < 16; ++i) hits[i] = 0.f;
#pragma unroll
      for (int n = 0; n < SP; ++n) {
        u32x2 w = *reinterpret_cast<const u32x2*>(vrow + n * PAGE + mt * 512);
#pragma unroll
        for (int i = 0; i < 2; ++i) w[i] = bytes_of(has_nan(w[i] & first_bytes(limit - n * PS - 4 * i)), 0x38u);   // 1.0 where the code is NaN
        hits = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen8(w[0], w[1], 1.f), seen[n], hits, 0, 0, 0);
      }
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (hits[i] > 0.f) col.o[mt][i] = __builtin_nanf("");
    }
  }
}

// MODE: 1 single tokens only, 2 chunks only, 3 both.  NW: wavefronts of a block (chunks: two)
template <int MODE, int NW>
__global__ __launch_bounds__(64 * NW, 2) void kv8_attn_kernel(Args a) {
  static_assert(MODE == 1 || NW == CHUNK_NW, "a chunk's four tiles are two wavefronts' work");
  constexpr int NT = 64 * NW;
  __shared__ Tables tab;
  __shared__ __attribute__((aligned(1024))) StepLds ring0, ring1;
  __shared__ float token_o[MODE == 1 ? NW * 16 * D : 4];
  __shared__ float token_m[NW][16], token_l[NW][16];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int turn = blockIdx.x / a.nkv, kvh = blockIdx.x % a.nkv;
  const int item = a.fold > 1 ? item_of_turn(turn, a.n_items, a.fold) : turn;
  if (item >= a.n_items) return;
  const int tile0 = a.item_tile[item], split = a.item_split[item], ntl = a.item_ntiles[item];
  const int tl = tile0 + ntl - 1, r = a.tile_req[tile0];
  const int tok_first = a.tile_tok0[tile0], ntok_first = a.tile_ntok[tile0];
  const int tok_last = a.tile_tok0[tl] + a.tile_ntok[tl] - 1;
  const bool lone = ntl == 1 && ntok_first == 1;
  // (a chunk's odd last token is a single token too, but keeps the key ranges of its request)
  const int fold = a.fold > 1 && (a.whole || a.req_tok_off[r + 1] - a.req_tok_off[r] == 1) ? a.fold : 1;
  if (split % fold != 0) return;                           // the block of an earlier split takes this one's keys (whole block)
  const int pb = split * a.split_pages;
  // The block's start is a chain of lookups in front of its first codes: each step asks for all it can.  The page ids of the range, and
  // what may follow them in the request's row of the table (never used), come with the positions; their scales are on their way
  // while the first codes are asked for.
  const int n_range = min(fold * a.split_pages, a.max_pages - pb);
  int ids[MAXSP / NT];
#pragma unroll
  for (int i = 0; i < MAXSP / NT; ++i)
    if (i == 0 || i * NT < n_range) ids[i] = a.block_table[(size_t)r * a.max_pages + pb + min(tid + i * NT, n_range - 1)];
  const int last_pos = a.tok_pos[tok_last], first_pos = a.tok_pos[tok_first];
  const int npg = min(n_range, last_pos / PS + 1 - pb);   // >= 1: an item's splits lie inside its visible range
  float ks[MAXSP / NT], vs[MAXSP / NT];
#pragma unroll
  for (int i = 0; i < MAXSP / NT; ++i)
    if (tid + i * NT < npg) {
      const size_t ph = (size_t)ids[i] * a.nkv + kvh;
      ks[i] = a.k_scale[ph];
      vs[i] = a.v_scale[ph];
      tab.page[tid + i * NT] = ids[i];
    }
  __syncthreads();
  auto keep_scales = [&]() {
#pragma unroll
    for (int i = 0; i < MAXSP / NT; ++i)
      if (tid + i * NT < npg) {
        tab.ks[tid + i * NT] = ks[i];
        tab.vs[tid + i * NT] = vs[i];
      }
    __syncthreads();
  };
  if (MODE == 1 || (MODE == 3 && lone)) {
    static_assert(MODE == 1 || sizeof(StepLds) >= NW * 16 * D * sizeof(float), "the sums of a single token fit a step's buffer");
    const TokenLds token{MODE == 1 ? token_o : reinterpret_cast<float*>(ring0.k), token_m, token_l};
    token_block<NW>(a, tab, token, tile0, split, fold, kvh, npg, min(last_pos + 1 - pb * PS, npg * PS), keep_scales);
    return;
  }
  if constexpr (MODE != 1) {
    const int group = a.nq / a.nkv, c = lane & 15, x = (lane >> 4) & 1, h = lane >> 5;
    load_step(a, tab, ring0, 0, kvh, npg, wave, lane);
    keep_scales();
    const bool work = TILES * wave < ntl;                          // (a wavefront without a tile only helps with the loads)
    const bool mine = TILES * wave + x < ntl;
    const int tile = mine ? tile0 + TILES * wave + x : tile0, t0 = a.tile_tok0[tile];
    const bool ok = mine && c < a.tile_ntok[tile] * group;
    const int t = ok ? t0 + c / group : t0;
    const int pos = ok ? a.tok_pos[t] - pb * PS : -1;
    Wide col;
    col.start(a.q + (size_t)t * a.ldq + (size_t)(kvh * group + (ok ? c % group : 0)) * D, h, ok);
    const int n_st = (npg + SP - 1) / SP;
    const int first = first_pos - pb * PS, end = last_pos + 1 - pb * PS;
    // my loads have landed and my reads of the buffer that is handed over have returned -> barrier -> everyone's have
#define FLEXCO_KV8_HAND_OVER()                \
  {                                           \
    __builtin_amdgcn_s_waitcnt(0x0070);       \
    asm volatile("" ::: "memory");            \
    __builtin_amdgcn_s_barrier();             \
    asm volatile("" ::: "memory");            \
  }
    const float scale_log2 = a.scale_log2;
    // first the steps that lie wholly before every column's own position, in pairs, then the rest
    int st = 0;
    for (const int n_free = (min(first + 1, npg * PS) / (SP * PS)) & ~1; st < n_free; st += 2) {
      FLEXCO_KV8_HAND_OVER()
      load_step(a, tab, ring1, st + 1, kvh, npg, wave, lane);
      if (work) chunk_step<false>(scale_log2, tab, ring0, col, st, npg, pos, end, lane);
      FLEXCO_KV8_HAND_OVER()
      if (st + 2 < n_st) load_step(a, tab, ring0, st + 2, kvh, npg, wave, lane);
      if (work) chunk_step<false>(scale_log2, tab, ring1, col, st + 1, npg, pos, end, lane);
    }
    for (; st < n_st; st += 2) {
      FLEXCO_KV8_HAND_OVER()
      if (st + 1 < n_st) load_step(a, tab, ring1, st + 1, kvh, npg, wave, lane);
      if (work) chunk_step<true>(scale_log2, tab, ring0, col, st, npg, pos, end, lane);
      if (st + 1 >= n_st) break;
      FLEXCO_KV8_HAND_OVER()
      if (st + 2 < n_st) load_step(a, tab, ring0, st + 2, kvh, npg, wave, lane);
      if (work) chunk_step<true>(scale_log2, tab, ring1, col, st + 1, npg, pos, end, lane);
    }
#undef FLEXCO_KV8_HAND_OVER
    const float lsum = sum_xor32(col.l);
    if (!ok || split >= a.tile_nsplit[tile]) return;               // (the tile's own keys end before this split)
    float row[64];
#pragma unroll
    for (int i = 0; i < 64; ++i) row[i] = col.o[i >> 4][i & 15];
    write_column(a, tile, split, fold, kvh, group, c, 4 * h, row, 16, 8, col.m, lsum, h == 0);
  }
}

}  // namespace

int32_t launch_kv8_attention_mfma(const flexco_layer_cfg& c, const flexco_maps& m, const void* q, size_t ldq, const flexco_kv8_pool& pool,
                                  float* part_ml, float* part_acc, void* out, size_t ldo, float* lse, hipStream_t s,
                                  const AttnKeep* keep) {
  const Kv8Plan plan = plan_kv8_attention(m, c.n_kv_heads);
  const int fold = plan.fold, group = c.n_q_heads / c.n_kv_heads;
  if (c.dtype != FLEXCO_BF16 || c.head_dim != D || c.page_size != PS || group > 16 || ldq % 8 != 0 ||
      m.kv_split_pages * fold > MAXSP || ldo % 4 != 0 || ((uintptr_t)out & 7))
    return FLEXCO_EUNSUPPORTED;
  Args a;
  a.tok_pos = m.tok_pos; a.block_table = m.block_table; a.tile_req = m.tile_req; a.tile_tok0 = m.tile_tok0;
  a.tile_ntok = m.tile_ntok; a.tile_nsplit = m.tile_nsplit; a.tile_part0 = m.tile_part0; a.item_tile = m.item_tile;
  a.item_split = m.item_split; a.item_ntiles = m.item_ntiles; a.req_tok_off = m.req_tok_off;
  a.max_pages = m.max_pages; a.nq = c.n_q_heads; a.nkv = c.n_kv_heads; a.n_items = m.n_items; a.split_pages = m.kv_split_pages;
  a.fold = fold; a.whole = plan.whole;
  a.scale_log2 = 1.4426950408889634f / sqrtf((float)D);
  a.q = (const bf16_t*)q; a.ldq = ldq;
  a.k_codes = pool.k_codes; a.v_codes = pool.v_codes; a.k_scale = pool.k_scale; a.v_scale = pool.v_scale;
  a.part_ml = part_ml; a.part_acc = part_acc;
  a.out = (bf16_t*)out; a.ldo = ldo; a.lse = lse;
  a.keep = keep ? *keep : AttnKeep{nullptr, nullptr, 0, 0};
  const dim3 grid((unsigned)turns_of(m.n_items, fold) * c.n_kv_heads);
  {
    KernelTimerScope ts(FLEXCO_K_ATTN_FWD, s);
    if (m.n_single == m.n_items) {
      if (plan.wavefronts == 4) hipLaunchKernelGGL((kv8_attn_kernel<1, 4>), grid, dim3(256), 0, s, a);
      else hipLaunchKernelGGL((kv8_attn_kernel<1, 2>), grid, dim3(128), 0, s, a);
    } else if (m.n_single == 0) {
      hipLaunchKernelGGL((kv8_attn_kernel<2, CHUNK_NW>), grid, dim3(64 * CHUNK_NW), 0, s, a);
    } else {
      hipLaunchKernelGGL((kv8_attn_kernel<3, CHUNK_NW>), grid, dim3(64 * CHUNK_NW), 0, s, a);
    }
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return fail(FLEXCO_EHIP, "launch of kv8_attn failed: %s", hipGetErrorString(e));
  // every request in one piece: nothing to join
  if (m.n_parts == m.n_tiles || plan.whole || (m.n_single == m.n_items && m.max_pages <= fold * m.kv_split_pages)) return FLEXCO_OK;
  return launch_kv8_merge(c, m, part_ml, part_acc, out, ldo, lse, s, fold, keep);
}

}  // namespace flexco
