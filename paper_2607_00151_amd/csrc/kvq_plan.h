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
constexpr int kKvqCost[kKvqClasses] = {4, 5, 12, 16};   // of a tile of keys, relative
constexpr int32_t kKvqMaxLen = INT32_MAX / kKvqKeys * kKvqKeys;   // the end of its last tile fits an int32
constexpr int64_t kKvqMaxItems = int64_t(1) << 22;   // work items before they are cut

struct KvqPlan {
  std::vector<AttnItem> items[kKvqClasses];  // one per workgroup, in launch order; part: first row of its partial (-1: none)
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

// Row tiles of kKvqRows rows, the last one of a sequence in the smallest class that
// holds it, each cut by key range into parts of about equal cost.
inline sa_status plan_kvq_items(const sa_layout* layout, int32_t batch, const int32_t* h_q_len, const int32_t* h_kv_len,
                                bool causal, int num_cu, KvqPlan& out, std::string& err) {
  const int Hkv = layout->num_kv_heads, G = layout->num_q_heads / Hkv;
  constexpr int kMost = kKvqRows[kKvqClasses - 1];
  out = KvqPlan{};
  struct Tile {
    int seq, row0, rows, cls, keys, q_start;
  };
  std::vector<Tile> tiles;
  int64_t work = 0, n_items = 0;
  int32_t q_start = 0;
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
      tiles.push_back({b, r0, n, cls, keys, q_start});
      work += (int64_t)Hkv * kKvqCost[cls] * ((keys + kKvqKeys - 1) / kKvqKeys);
    }
    q_start += h_q_len[b];
  }
  const int64_t share = std::max<int64_t>(32, (work + 2 * num_cu - 1) / (2 * num_cu));
  for (const Tile& t : tiles) {
    const int n_tiles = (t.keys + kKvqKeys - 1) / kKvqKeys;
    const int parts = (int)std::max<int64_t>(1, ((int64_t)n_tiles * kKvqCost[t.cls] + share - 1) / share);
    const int per = std::max(1, (n_tiles + parts - 1) / parts);
    const int used = std::max(1, (n_tiles + per - 1) / per);
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
        out.items[t.cls].push_back({t.seq, h, t.row0, s * per * kKvqKeys, (int32_t)std::min<int64_t>(t.keys, (int64_t)(s + 1) * per * kKvqKeys),
                                    used > 1 ? (int32_t)(row + ((int64_t)h * used + s) * t.rows) : -1, 0, t.q_start,
                                    h_q_len[t.seq], h_kv_len[t.seq]});
  }
  for (auto& items : out.items)
    std::stable_sort(items.begin(), items.end(), [](const AttnItem& x, const AttnItem& y) {
      return x.kv_end - x.kv_begin > y.kv_end - y.kv_begin;
    });
  return SA_OK;
}

}  // namespace sa
