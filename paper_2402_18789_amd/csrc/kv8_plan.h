#pragma once
// How the 8-bit attention cuts a work list for its blocks.  Host arithmetic on the maps' sums alone.
#include <algorithm>
#include <cstdint>
#include "flexco.h"

namespace flexco {

constexpr int KV8_MAX_PAGES = 512;        // pages of a block's table

// fold: neighbouring key splits of a request of one token that its block takes as one.  wavefronts: of a block of a list of nothing but single
// tokens (chunks, and what lies in a list with them: two).  whole: every request's splits are taken as one, there is nothing to join.
struct Kv8Plan { int fold, wavefronts; bool whole; };

// The work list is cut for one wavefront per item and head, finer than blocks of several need.  Us of attention and joining, measured with
// 1 - 512 requests of 50 - 32000 keys over 1 and 8 kv heads, every fold and 2, 4 and 8 wavefronts (8 were never ahead):
//   * contexts of up to 64 pages stay whole, there is nothing to join: 4 of 1000 keys in eights 9.2, whole 8.4; 32 of 100 - 1000 20 / 14.1;
//     125 pages whole 12.0, in 16s 9.3;
//   * else pieces of 8 pages are joined to 16 where there are few (one context of 2000 9.3, 32s 10.2), to 32 (64 of 500 - 4096 over
//     one head 22 / 17.8, 64s 20.3) or 64 (one of 32000 33 / 19.2) as their number grows, longer ones to 64 (three of 9001 - 32765 44 / 34.6,
//     8 of 8000 34.8 / 32.0; in 128s 38);
//   * whole requests of up to 256 pages that fill the chip stay whole: 96 of 4000 in 128s 149, whole 140.
// A list with chunks whose requests have at most 16 pages: whole (a prompt of 189 tokens over 40/8 heads 15.0 / 12.7, of 300 with up to 32 pages 19.9 /
// 17.2, but 13 new tokens behind 372 14.7 / 15.4, 100 behind 400 beside 8 single tokens 20.4 / 23.8).
// Two wavefronts where there are more short pieces than the chip holds blocks of four (256 of 10 - 600 keys 37.8 / 44.1, 512 of 16 - 400
// 52.9 / 68.6), else four (one context of 700 keys 10.0 / 7.9, 128 of 100 - 4096 112 / 100, 256 of 512 - 4096 215 / 213).
inline Kv8Plan plan_kv8_attention(const flexco_maps& m, int nkv) {
  const int sp = m.kv_split_pages;
  const bool alone = m.n_single == m.n_items;
  const bool whole = m.n_parts > m.n_tiles && m.max_pages <= 16;
  if (sp <= 0 || (m.n_single == 0 && !whole)) return {1, 2, false};
  const int64_t blocks = (int64_t)m.n_single * nkv;
  int pages = m.max_pages;                // of a piece
  if (m.n_parts > m.n_tiles && m.max_pages > 64 && !(alone && m.max_pages <= 256 && (int64_t)m.n_tiles * nkv >= 768))
    pages = sp > 8 || blocks > 1500 ? 64 : blocks > 512 ? 32 : 16;
  int fold = 1;
  if (m.n_parts > m.n_tiles)
    while (fold * sp < pages && 2 * fold * sp <= KV8_MAX_PAGES) fold *= 2;
  const int64_t left = (blocks + fold - 1) / fold;
  const bool few_pages = (int64_t)m.stream_pages * nkv < 24 * left;
  return {fold, alone && !(few_pages && left > 1024) ? 4 : 2, whole};
}

}  // namespace flexco
