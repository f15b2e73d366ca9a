#pragma once
// How many neighbouring key splits of the work list a block of the 8-bit attention takes as one (requests of one token).  Host
// arithmetic on the maps' sums alone.
#include <algorithm>
#include <cstdint>
#include "flexco.h"

namespace flexco {

constexpr int KV8_MAX_PAGES = 512;        // pages of a block's table

// The work list is cut for one wavefront per item and head; a block here has two, and four of them fit a CU: 1024 on the chip.
// Us of attention and joining, one fold / another:
//   * contexts of up to 48 pages stay whole: 64 requests of 30 - 500 keys 18.5 / 14.0, 16 of 300 10.9 / 8.5, one of 700 11.2 / 9.9 (up to 62
//     pages level, 125 in one 15 against 11);
//   * pieces of 8 and 16 pages are taken together while there are more blocks than the chip holds, up to 64 pages: one context of 32000
//     28 / 22.7, three of 9001 - 32765 38 / 33.7, 32 requests of 100 - 1000 18 / 16.5; with fewer blocks they stay as they are (4 of 4000
//     15.1 / 16.0, 12 of 700 - 1500 14.6 / 16);
//   * longer pieces stay (64 requests of 500 - 4096 in pieces of 64 pages 65 / 72) unless whole requests fill the chip: 96 of 4000
//     164 / 145.
inline int plan_kv8_fold(const flexco_maps& m, int nkv) {
  const int sp = m.kv_split_pages;
  if (m.n_single == 0 || m.n_parts == m.n_tiles || sp <= 0) return 1;
  auto up_to = [&](int pages) {
    int f = 1;
    while (f * sp < pages && 2 * f * sp <= KV8_MAX_PAGES) f *= 2;
    return f;
  };
  if (m.max_pages <= 48) return up_to(m.max_pages);
  if (m.n_single == m.n_items && m.max_pages <= 256 && (int64_t)m.n_tiles * nkv >= 768) return up_to(m.max_pages);
  int f = 1;
  if (sp <= 16)
    while ((int64_t)m.n_single * nkv > 1100 * f && 2 * f * sp <= 64) f *= 2;
  return f;
}

}  // namespace flexco
