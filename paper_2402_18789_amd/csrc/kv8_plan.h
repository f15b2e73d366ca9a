#pragma once
// How many neighbouring key splits of the work list a block of the 8-bit attention takes as one.  Host arithmetic on the maps' sums.
#include <cstdint>
#include <cstdlib>
#include "flexco.h"

namespace flexco {

inline int plan_kv8_fold(const flexco_maps& m, int nkv) {
  if (const char* e = getenv("KV8_FOLD")) return atoi(e);
  return 1;
}

}  // namespace flexco
