// The host layer of the serving calls (da_paged_api.cpp, compiled for the host only) with stub
// launchers that keep what a kernel would get, and the sums that host and kernels share.  Built
// under AddressSanitizer and UndefinedBehaviorSanitizer by tests/test_sanitizers.py: sizes at the
// ends of what the calls take must neither wrap nor pass as others.
#include <stdint.h>
#include <stdio.h>

#include "da_paged.hpp"
#include "delta_attn.h"

namespace da {
static int g_launched = 0;
static SelectArgs g_select;
static PagedArgs g_paged;
da_status check_device() { return DA_OK; }
da_status fail_hip(hipError_t) { return DA_ERR_HIP; }
hipError_t launch_pages_fork(const Table&, const int32_t*, const int32_t*, int, int32_t*, hipStream_t) { ++g_launched; return hipSuccess; }
hipError_t launch_pages_resize(const Table&, const Pages&, const int32_t*, const int32_t*, int, int32_t*, hipStream_t) { ++g_launched; return hipSuccess; }
hipError_t launch_pages_append(const Table&, const Pages&, const uint16_t*, const uint16_t*, int64_t, const int32_t*, const int32_t*, int, int, const int32_t*, hipStream_t) { ++g_launched; return hipSuccess; }
hipError_t launch_pages_compact(const Table&, const Pages&, const int32_t*, const int32_t*, const int32_t*, int64_t, const int32_t*, int, int32_t*, hipStream_t) { ++g_launched; return hipSuccess; }
hipError_t launch_summary(const SummaryArgs&, hipStream_t) { ++g_launched; return hipSuccess; }
hipError_t launch_select_blocks(const SelectArgs& a, hipStream_t) { ++g_launched; g_select = a; return hipSuccess; }
hipError_t launch_select_pages(const SelectArgs& a, hipStream_t) { ++g_launched; g_select = a; return hipSuccess; }
hipError_t launch_paged_attn(const PagedArgs& a, hipStream_t) { ++g_launched; g_paged = a; return hipSuccess; }
}  // namespace da

using namespace da;

static int failures = 0;
static void expect(int64_t got, int64_t want, const char* what) {
  if (got != want) {
    fprintf(stderr, "%s: %lld, expected %lld\n", what, (long long)got, (long long)want);
    ++failures;
  }
}

// Lists of a query block's candidates begin where the sizes before them add up, whatever top_k.
static void lists_of_any_top_k() {
  alignas(16) char p[16];
  int32_t* const i = (int32_t*)p;
  for (int block_q : {64, 128, 256})
    for (int top_k : {2, 7, 8, 100, INT32_MAX - 1, INT32_MAX}) {
      const int N = 5000, R = block_q / 64, nqb = (N + block_q - 1) / block_q;
      expect(da_select_blocks(p, p, (float*)p, nullptr, 1, N, 8, 2, 128, top_k, 1, 1, block_q, i, i, nullptr), DA_OK, "select_blocks");
      expect(g_select.nqb, nqb, "query blocks");
      int64_t sum = 0;
      for (int qb = 0; qb <= nqb; ++qb) {
        expect(list_entries_before(qb, g_select.top_k, R), sum, "entries before a list");
        sum += (int64_t)qb * R < top_k ? qb * R : top_k;
      }
      expect(da_select_blocks_entries(1, N, 2, top_k, block_q), 2 * list_entries_before(nqb, top_k, R), "entries");
      expect(g_select.total, list_entries_before(nqb, top_k, R), "total");
    }
}

// As many pages as are counted at all are shared out whole, however many workgroups there are.
static void shares_of_any_total() {
  for (int total : {0, 1, 7, 1000, INT32_MAX - 511, INT32_MAX - 1, INT32_MAX})
    for (int n : {1, 3, 85, 256, 511, 512})
      for (int least : {1, 2, 16}) {
        const int64_t share = share_of(least, total, n);
        expect(share >= least && share * n >= total, 1, "shares hold all units");
        expect(share == least || (share - 1) * n < total, 1, "shares are even");
      }
}

int main() {
  lists_of_any_top_k();
  shares_of_any_total();
  if (failures) return 1;
  printf("paged driver ok\n");
  return 0;
}
