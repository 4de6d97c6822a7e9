// Host-only check of branch_plan.h's debug check of shared prefixes, built with
// AddressSanitizer and UndefinedBehaviorSanitizer by tests/test_branch_edges_cpu.py.
// Prints "ALL OK" and exits 0 on success.
#include <cstdio>
#include <vector>

#include "branch_plan.h"

static int g_fail = 0;
#define CHECK(cond)                                                     \
  do {                                                                  \
    if (!(cond)) {                                                      \
      std::fprintf(stderr, "FAIL %s:%d: %s\n", __FILE__, __LINE__, #cond); \
      ++g_fail;                                                         \
    }                                                                   \
  } while (0)

int main() {
  // two groups; the first's first member has no rows, its other two share 35 tokens on pages of 16
  const std::vector<int32_t> groups{0, 3, 4}, q{0, 1, 2, 1}, ip{0, 1, 4, 8, 9};
  const std::vector<int32_t> ix{99, 1, 2, 3, 1, 2, 7, 8, 5};
  std::vector<sa::SharedCopy> differ;
  std::string err;
  auto go = [&](std::vector<int32_t> shared, const std::vector<int32_t>& pages, int64_t slots) {
    return sa::debug_check_shared(2, groups.data(), shared.data(), q.data(), ip.data(), pages.data(), 16, slots, differ, err);
  };
  CHECK(go({35, 16}, ix, 10) == SA_OK);                       // slot 99 is of a member whose table is not read
  CHECK(differ.size() == 1);
  CHECK(differ[0].group == 0 && differ[0].seq == 2 && differ[0].of == 1 && differ[0].page == 2);
  CHECK(differ[0].slot == 7 && differ[0].of_slot == 3 && differ[0].rows == 3);
  CHECK(go({48, 0}, ix, 10) == SA_OK && differ.size() == 1 && differ[0].rows == 16);
  CHECK(go({32, 16}, ix, 10) == SA_OK && differ.empty());
  CHECK(go({0, 0}, ix, 10) == SA_OK && differ.empty());
  CHECK(go({49, 0}, ix, 10) == SA_ERR_RANGE);                 // a fourth page that sequence 1 lacks
  CHECK(go({35, 17}, ix, 10) == SA_ERR_RANGE);
  CHECK(go({35, 16}, ix, 7) == SA_ERR_RANGE);                 // slot 7 of 7
  std::vector<int32_t> bad = ix;
  bad[4] = -1;
  CHECK(go({35, 16}, bad, 10) == SA_ERR_RANGE);
  if (g_fail) return 1;
  std::puts("ALL OK");
  return 0;
}
