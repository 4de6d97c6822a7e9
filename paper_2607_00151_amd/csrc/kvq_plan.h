// Host planner of sa_kvq_attn: work items and the rows whose parts are joined.
// Plain C++: no HIP.
#pragma once

#include <algorithm>
#include <cstdint>
#include <string>
#include <vector>

#include "branch_plan.h"
#include "plan.h"
#include "sa.h"

namespace sa {

constexpr int kKvqKeys = 64;                 // keys of a tile
// Classes of items by their packed rows: up to 16 and 32, whose waves split the keys, and
// up to 64 and 128, whose waves split the rows.
constexpr int kKvqClasses = 4;
constexpr int kKvqRows[kKvqClasses] = {16, 32, 64, 128};
// Microseconds of a tile of keys with the CUs' places taken, of an item's start and end,
// and of the launch that joins parts.
constexpr double kKvqTileUs[kKvqClasses] = {0.86, 1.1, 1.4, 2.1};
constexpr double kKvqItemUs = 4.0, kKvqJoinUs = 6.0;
constexpr int kKvqLeast[kKvqClasses] = {4, 4, 4, 2};    // tiles of a part
constexpr int32_t kKvqMaxLen = INT32_MAX / kKvqKeys * kKvqKeys;   // the end of its last tile fits an int32
constexpr int64_t kKvqMaxItems = int64_t(1) << 22;   // work items before they are cut

struct KvqPlan {
  std::vector<AttnItem> items;               // one per workgroup, in launch order; boost: its class; part: first row of its partial (-1: none)
  bool few = false;                          // all of class 0
  std::vector<MergeUnit> units;
  int64_t part_rows = 0;
  int32_t most_rows = 0, most_parts = 0;     // of a unit
};

inline sa_status kvq_attn_check(const sa_layout* layout, int32_t layer, int32_t batch, const int32_t* h_q_len,
                                const int32_t* h_kv_len, bool causal, float softmax_scale, int64_t& total_q,
                                int64_t& total_kv, std::string& err) {
  const sa_status s = check_attn_call(layout, layer, batch, h_q_len, h_kv_len, softmax_scale, err);
  if (s != SA_OK) return s;
  const int G = layout->num_q_heads / layout->num_kv_heads;
  total_q = total_kv = 0;
  for (int b = 0; b < batch; ++b) {
    if (h_q_len[b] < 0 || h_kv_len[b] < 0 || (causal && h_q_len[b] > h_kv_len[b]) || h_kv_len[b] > kKvqMaxLen)
      return plan_fail(err, SA_ERR_SHAPE, "sequence %d: q_len %d, kv_len %d (0 <= %s <= %d)", b, h_q_len[b],
                       h_kv_len[b], causal ? "q_len <= kv_len" : "q_len, kv_len", kKvqMaxLen);
    if ((int64_t)h_q_len[b] * G > INT32_MAX - kMaxRows)
      return plan_fail(err, SA_ERR_SHAPE, "sequence %d: q_len * G too large", b);
    total_q += h_q_len[b];
    if (h_q_len[b] > 0) total_kv += h_kv_len[b];
    if (total_q > INT32_MAX) return plan_fail(err, SA_ERR_SHAPE, "too many query tokens");
  }
  return SA_OK;
}

// Row tiles of 128 rows, the last one of a sequence in the smallest class that holds it,
// cut by key range into parts of at most `most` us: the one of a few such limits whose
// launch, by the longest part and an even share of the work, ends first.
inline sa_status plan_kvq_items(const sa_layout* layout, int32_t batch, const int32_t* h_q_len, const int32_t* h_kv_len,
                                bool causal, int num_cu, KvqPlan& out, std::string& err) {
  const int Hkv = layout->num_kv_heads, G = layout->num_q_heads / Hkv;
  constexpr int kMost = kKvqRows[kKvqClasses - 1];
  out = KvqPlan{};
  struct Tile {
    int seq, row0, rows, cls, keys, q_start, n_tiles;
  };
  std::vector<Tile> tiles;
  double work = 0, longest = 0;
  int64_t n_items = 0;
  int32_t q_start = 0;
  out.few = true;
  for (int b = 0; b < batch; ++b) {
    const int rows = h_q_len[b] * G;
    n_items += (int64_t)Hkv * ((rows + kMost - 1) / kMost);
    if (n_items > kKvqMaxItems)
      return plan_fail(err, SA_ERR_SHAPE, "too many query rows for one launch (%lld work items)", (long long)n_items);
    for (int r0 = 0; r0 < rows; r0 += kMost) {
      const int n = std::min(kMost, rows - r0);
      int cls = 0;
      while (n > kKvqRows[cls]) ++cls;
      const int keys = causal ? h_kv_len[b] - h_q_len[b] + (r0 + n - 1) / G + 1 : h_kv_len[b];
      const int n_tiles = (keys + kKvqKeys - 1) / kKvqKeys;
      tiles.push_back({b, r0, n, cls, keys, q_start, n_tiles});
      const double us = n_tiles * kKvqTileUs[cls];
      work += Hkv * us;
      longest = std::max(longest, us);
      out.few = out.few && cls == 0;
    }
    q_start += h_q_len[b];
  }
  const int slots = (out.few ? 3 : 2) * num_cu;
  auto parts_of = [&](const Tile& t, double most) {
    const int per = std::max(kKvqLeast[t.cls], (int)std::min<double>(t.n_tiles, most / kKvqTileUs[t.cls]));
    const int parts = std::max(1, (t.n_tiles + per - 1) / per);
    const int even = std::max(1, (t.n_tiles + parts - 1) / parts);
    return std::pair<int, int>(std::max(1, (t.n_tiles + even - 1) / even), even);
  };
  double best = 0, best_us = -1;
  for (const double f : {0., 2., 1.5, 1., 0.75, 0.5, 0.35, 0.25}) {
    const double most = f == 0. ? longest : f * work / slots;
    if (f != 0. && most >= longest) continue;
    double blocks = 0, top = 0;
    bool split = false;
    for (const Tile& t : tiles) {
      const auto [parts, even] = parts_of(t, most);
      blocks += (double)Hkv * parts;
      top = std::max(top, std::min(even, t.n_tiles) * kKvqTileUs[t.cls]);
      split = split || parts > 1;
    }
    const double share = (work + blocks * kKvqItemUs) / slots;
    const double us = (blocks <= slots ? top + kKvqItemUs : std::max(top + kKvqItemUs, share + 0.5 * top)) + (split ? kKvqJoinUs : 0.);
    if (best_us < 0 || us < best_us) {
      best = most;
      best_us = us;
    }
  }
  for (const Tile& t : tiles) {
    const auto [used, per] = parts_of(t, best);
    const int64_t row = out.part_rows;
    if (used > 1) {
      out.units.push_back({t.q_start, t.row0, t.rows, (int32_t)row, used, t.rows, 0, 0, 0});
      out.part_rows += (int64_t)Hkv * used * t.rows;
      if (out.part_rows > kMaxPartRows)
        return plan_fail(err, SA_ERR_SHAPE, "too many query rows for one launch (partial results)");
      out.most_rows = std::max(out.most_rows, t.rows);
      out.most_parts = std::max(out.most_parts, used);
    }
    for (int h = 0; h < Hkv; ++h)
      for (int s = 0; s < used; ++s)
        out.items.push_back({t.seq, h, t.row0, s * per * kKvqKeys, (int32_t)std::min<int64_t>(t.keys, (int64_t)(s + 1) * per * kKvqKeys),
                             used > 1 ? (int32_t)(row + ((int64_t)h * used + s) * t.rows) : -1, t.cls, t.q_start,
                             h_q_len[t.seq], h_kv_len[t.seq]});
  }
  std::stable_sort(out.items.begin(), out.items.end(), [](const AttnItem& x, const AttnItem& y) {
    auto us = [](const AttnItem& it) { return (it.kv_end - it.kv_begin) * kKvqTileUs[it.boost]; };
    return us(x) > us(y);
  });
  return SA_OK;
}

}  // namespace sa
