// Host side of the 8-bit cache: which tokens of a batch share a page.  No device calls.
#include <new>
#include <unordered_set>

#include "flexco_host.h"
#include "flexco_kv8.h"

using namespace flexco;

extern "C" int32_t flexco_kv8_abi_version(void) { return 1; }

namespace {
int32_t find_runs(const flexco_maps* host_maps, int32_t* runs, int32_t capacity, int32_t* n_runs) {
  FLEXCO_CHECK(host_maps && runs && n_runs, FLEXCO_EINVAL, "NULL argument");
  FLEXCO_CHECK(capacity >= 0, FLEXCO_EINVAL, "negative capacity");
  const flexco_maps& m = *host_maps;
  FLEXCO_CHECK(m.T > 0 && m.n_req > 0 && m.page_size > 0, FLEXCO_EINVAL, "maps describe an empty batch");
  FLEXCO_CHECK(m.slot && m.tok_pos && m.tok_req, FLEXCO_EINVAL, "maps hold a NULL array");
  // Pages in the order of their runs; a second run into one page is a fault wherever it stands in the batch.
  std::unordered_set<int32_t> pages;
  int32_t n = 0;
  for (int32_t t = 0; t < m.T;) {
    const int32_t at = m.tok_pos[t] % m.page_size;
    int32_t len = 1;
    while (t + len < m.T && at + len < m.page_size && m.tok_req[t + len] == m.tok_req[t]) ++len;
    const int32_t page = m.slot[t] / m.page_size;
    FLEXCO_CHECK(pages.insert(page).second, FLEXCO_EPAGE, "request %d, token %d: page %d is written to by another run of the batch",
                 m.tok_req[t], t, page);
    FLEXCO_CHECK(n < capacity, FLEXCO_EWORKSPACE, "more runs than the %d there is room for", capacity);
    runs[2 * n] = t;
    runs[2 * n + 1] = len;
    ++n;
    t += len;
  }
  *n_runs = n;
  return FLEXCO_OK;
}
}  // namespace

extern "C" int32_t flexco_kv8_runs(const flexco_maps* host_maps, int32_t* runs, int32_t capacity, int32_t* n_runs) {
  clear_error();
  try {
    return find_runs(host_maps, runs, capacity, n_runs);
  } catch (const std::bad_alloc&) {                          // (no exception passes the C boundary)
    return fail(FLEXCO_EWORKSPACE, "no host memory for the batch's pages");
  }
}
