// Host planner of sa_kvq_attn on its own (AddressSanitizer, UBSan): every visible
// (row, key) pair is in exactly one item, partial rows do not overlap and are joined
// by exactly one unit, over seeded batches of all kinds.
#include <cstdio>
#include <cstdlib>
#include <map>
#include <random>
#include <set>
#include <string>
#include <vector>

#include "kvq_plan.h"

#define CHECK(x)                                                        \
  do {                                                                  \
    if (!(x)) {                                                         \
      printf("FAILED %s:%d: %s\n", __FILE__, __LINE__, #x);             \
      exit(1);                                                          \
    }                                                                   \
  } while (0)

static void check(const sa_layout& L, const std::vector<int32_t>& q, const std::vector<int32_t>& kv, bool causal, int cus) {
  std::string err;
  sa::KvqPlan plan;
  const int B = (int)q.size(), G = L.num_q_heads / L.num_kv_heads;
  CHECK(sa::plan_kvq_items(&L, B, q.data(), kv.data(), causal, cus, plan, err) == SA_OK);
  // per (sequence, head, first row): the key ranges and partial rows
  struct Part {
    int begin, end, part, cls;
  };
  std::map<std::vector<int>, std::vector<Part>> tiles;
  std::vector<int32_t> q_start(B + 1, 0);
  for (int b = 0; b < B; ++b) q_start[b + 1] = q_start[b] + q[b];
  {
    for (const sa::KvqItem& it : plan.items) {
      const int c = it.cls;
      CHECK(c >= 0 && c < sa::kKvqClasses && (c == 0 || !plan.few));
      CHECK(it.seq >= 0 && it.seq < B && it.kvh >= 0 && it.kvh < L.num_kv_heads);
      CHECK(it.q_start == q_start[it.seq] && it.q_len == q[it.seq] && it.kv_len == kv[it.seq]);
      CHECK(it.row0 % 128 == 0 && it.row0 < it.q_len * G);
      CHECK(it.kv_begin % sa::kKvqKeys == 0 && it.kv_begin <= it.kv_end && it.kv_end <= it.kv_len);
      tiles[{it.seq, it.kvh, it.row0}].push_back({it.kv_begin, it.kv_end, it.part, c});
    }
  }
  std::map<int, int> joined;                                 // first partial row -> rows
  int64_t joined_rows = 0;
  std::map<int, std::vector<const sa::KvqItem*>> groups;     // joined by the launch itself: every tile at counters of its own
  for (const sa::KvqItem& it : plan.items) {
    CHECK((it.part >= 0) == (it.n_parts > 1) && (it.counter < 0 || it.part >= 0));
    if (it.counter >= 0) groups[it.counter].push_back(&it);
  }
  CHECK((int64_t)groups.size() * sa::kKvqCounted == plan.counters && plan.counters <= sa::kKvqCounters);
  for (auto& [c, items] : groups) {
    const int rows = std::min(128, items[0]->q_len * G - items[0]->row0);
    CHECK(c % sa::kKvqCounted == 0 && c < plan.counters && (int)items.size() == items[0]->n_parts);
    CHECK(sa::kvq_joins(items[0]->cls, items[0]->n_parts, rows) && items[0]->n_parts * rows <= sa::kKvqMostJoin);
    for (const sa::KvqItem* it : items) {
      CHECK(it->part0 == items[0]->part0 && it->n_parts == items[0]->n_parts);
      CHECK(it->part >= it->part0 && it->part + rows <= it->part0 + it->n_parts * rows);
      CHECK(it->seq == items[0]->seq && it->kvh == items[0]->kvh && it->row0 == items[0]->row0);
      CHECK(joined.emplace(it->part, rows).second);
    }
    joined_rows += (int64_t)items.size() * rows;
  }
  for (const sa::MergeUnit& u : plan.units) {
    CHECK(u.b_n == 0 && u.a_n >= 2 && u.n >= 1 && u.n <= plan.most_rows && u.a_n <= plan.most_parts);
    for (int h = 0; h < L.num_kv_heads; ++h)
      for (int s = 0; s < u.a_n; ++s) CHECK(joined.emplace(u.a_row + (h * u.a_n + s) * u.a_stride, u.n).second);
    joined_rows += (int64_t)L.num_kv_heads * u.a_n * u.n;
  }
  CHECK(joined_rows == plan.part_rows);
  size_t n_tiles = 0;
  for (int b = 0; b < B; ++b) {
    const int rows = q[b] * G;
    int step = 0;
    for (int r0 = 0; r0 < rows; r0 += step) {
      for (int h = 0; h < L.num_kv_heads; ++h) {
        auto found = tiles.find({b, h, r0});
        CHECK(found != tiles.end());
        auto parts = found->second;
        ++n_tiles;
        step = 128;
        for (const Part& x : parts) CHECK(std::min(128, rows - r0) <= sa::kKvqRows[x.cls] && x.cls == parts[0].cls);
        const int n = std::min(step, rows - r0);
        const int keys = causal ? kv[b] - q[b] + (r0 + n - 1) / G + 1 : kv[b];
        std::sort(parts.begin(), parts.end(), [](const Part& x, const Part& y) { return x.begin < y.begin; });
        CHECK(parts.front().begin == 0 && parts.back().end == keys);
        for (size_t i = 0; i < parts.size(); ++i) {
          if (i > 0) CHECK(parts[i].begin == parts[i - 1].end && parts[i].begin < parts[i].end);
          if (parts.size() == 1) {
            CHECK(parts[i].part == -1);
          } else {
            auto j = joined.find(parts[i].part);
            CHECK(j != joined.end() && j->second == n);
            joined.erase(j);
          }
        }
      }
    }
  }
  CHECK(joined.empty() && n_tiles == tiles.size());
}

int main() {
  std::mt19937 r(5);
  auto pick = [&](int lo, int hi) { return lo + (int)(r() % (unsigned)(hi - lo + 1)); };
  const int heads[][2] = {{32, 8}, {8, 2}, {64, 8}, {1, 1}, {7, 7}, {16, 1}, {65, 1}, {40, 8}};
  for (int n = 0; n < 3000; ++n) {
    const auto& h = heads[pick(0, 7)];
    const sa_layout L{h[0], h[1], 128, pick(0, 1) ? 16 : 32, 1, 1000};
    const bool causal = pick(0, 1);
    const int B = pick(1, 20), most = 1 << pick(0, 15);
    std::vector<int32_t> q, kv;
    for (int b = 0; b < B; ++b) {
      kv.push_back(pick(0, most));
      const int mq = pick(0, 2) == 0 ? 1 : pick(0, 100);
      q.push_back(causal ? std::min(mq, kv.back()) : mq);
    }
    check(L, q, kv, causal, pick(0, 1) ? 256 : pick(1, 300));
  }
  const sa_layout big{8, 1, 128, 16, 1, 1000};
  check(big, {1}, {sa::kKvqMaxLen}, true, 256);              // the longest cache
  check(big, {1, 1}, {sa::kKvqMaxLen, 3}, false, 256);
  std::string err;
  sa::KvqPlan plan;
  const sa_layout wide{1, 1, 128, 16, 1, 1000};
  const int32_t q[1] = {INT32_MAX - sa::kMaxRows}, kv[1] = {64};
  CHECK(sa::plan_kvq_items(&wide, 1, q, kv, false, 256, plan, err) == SA_ERR_SHAPE && !err.empty());
  printf("ALL OK\n");
  return 0;
}
