// Host planner of sa_kvq_attn: work items and the rows whose parts are joined.
// Plain C++: no HIP.
#pragma once

#include <algorithm>
#include <cstdint>
#include <functional>
#include <string>
#include <utility>
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
// What a launch's time is made of, in microseconds.  Measured to 5%, 32/8 heads: a tile of keys
// where two blocks share every CU.  Fitted, with the rates in plan_kvq_items, to 70 drawn
// batches under nine limits each: the start and end of an item, the launch that joins parts,
// each part of a row and each partial row, and where the launch joins itself, a start, a
// partial row that a block reads and a part that a wave reads.
constexpr double kKvqTileUs[kKvqClasses] = {0.8, 0.84, 1.31, 2.0};
constexpr double kKvqItemUs = 3.0, kKvqJoinUs = 8.0, kKvqPartUs = 0.08, kKvqPartRowUs = 4e-4;
constexpr double kKvqInLaunchUs = 1.0, kKvqReadRowUs = 0.03, kKvqReadTileUs = 0.6;
// Which parts the launch joins itself, and a second one does not have to: of a tile whose
// waves split the keys up to so many rows (parts times rows), which the block that ends
// last reads in a trip or two to memory; of one whose waves split the rows up to so many
// parts, which each wave joins for its own rows.
constexpr int kKvqJoinRows = 128, kKvqJoinParts = 8;
constexpr int kKvqMostJoin = kKvqJoinParts * 128 > kKvqJoinRows ? kKvqJoinParts * 128 : kKvqJoinRows;   // rows
constexpr int kKvqCounted = 4;               // counters of a tile: one for every 16 rows, or for every wave
constexpr int64_t kKvqCounters = 32768;
inline bool kvq_joins(int cls, int parts, int rows) {
  return cls < 2 ? parts * rows <= kKvqJoinRows : parts <= kKvqJoinParts;
}
constexpr int kKvqLeast[kKvqClasses] = {8, 8, 4, 4};    // tiles of a part
constexpr int32_t kKvqMaxLen = INT32_MAX / kKvqKeys * kKvqKeys;   // the end of its last tile fits an int32
constexpr int64_t kKvqMaxItems = int64_t(1) << 22;   // work items before they are cut
constexpr int kKvqSimulated = 2048;                  // parts of one KV head whose launch is played through

// A work item: rows row0 .. (of the class) of a sequence's packed rows of one KV head over
// keys kv_begin .. kv_end - 1.  part: the first row of its partial among all (-1: the
// item is whole); of its row tile's parts, part0 is the first one's, n_parts their number
// and counter the first of kKvqCounted counters, at which the launch joins them (-1: it does not).
struct KvqItem {
  int32_t seq, kvh, row0, kv_begin, kv_end, cls;
  int32_t q_start, q_len, kv_len;
  int32_t part, part0, n_parts, counter;
};

struct KvqPlan {
  std::vector<KvqItem> items;                // one per workgroup, in launch order
  bool few = false;                          // all of class 0
  int64_t counters = 0;
  std::vector<MergeUnit> units;              // the row tiles that a second launch joins
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
// cut by key range into parts of at most so many us: the one of a few such limits whose
// launch ends first.
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
  // How many tile microseconds n blocks do in one.  A block with a CU to itself is quicker
  // than one of two (0.6 of the time; of class 0 half or less, where HBM is what they share),
  // so the end of a launch, when places are empty, does not cost what they would have done.
  // Over 70 drawn batches and six listed ones the parts chosen so take 1.04 times the best limit's time in the
  // geometric mean, at the worst 1.15.
  auto rate = [&](double n) {
    if (out.few) return std::min(2.1 * n, 2.05 * num_cu);
    return n <= num_cu ? 1.67 * n : std::min(2. * num_cu, 1.67 * num_cu + 0.33 * (n - num_cu));
  };
  // The end of a launch whose parts are at most `most` long, taken longest first: blocks in
  // place go equally fast, one that ends leaves its place to the next part.  The KV heads'
  // items are alike, so one head's, on its share of the places, tell for all; of very many, an even share.
  std::vector<double> parts_us, place;
  auto ends = [&](double most) {
    parts_us.clear();
    double rows = 0, sum = 0;
    int64_t blocks = 0;
    double in_launch = 0;
    int most_parts = 0;
    bool again = false;
    for (const Tile& t : tiles) {
      const auto [parts, even] = parts_of(t, most);
      blocks += parts;
      if (parts > 1) rows += (double)parts * t.rows;
      if (parts > 1 && kvq_joins(t.cls, parts, t.rows))
        in_launch = std::max(in_launch, kKvqInLaunchUs + parts * (t.cls < 2 ? kKvqReadRowUs * t.rows : kKvqReadTileUs));
      else
        again = again || parts > 1;
      most_parts = std::max(most_parts, parts);
      const double us = std::min(even, t.n_tiles) * kKvqTileUs[t.cls] + kKvqItemUs;
      sum += parts * us;
      if (blocks <= kKvqSimulated) parts_us.insert(parts_us.end(), (size_t)parts, us);
    }
    const double join = rows == 0 ? 0. : Hkv * rows * kKvqPartRowUs + (again ? kKvqJoinUs + kKvqPartUs * most_parts : in_launch);
    if (blocks > kKvqSimulated) return Hkv * sum / rate(slots) + join;
    std::sort(parts_us.begin(), parts_us.end(), std::greater<double>());
    // the first blocks go round the CUs: one that has to share its CU from the start does so to its end
    const size_t second = std::max(1, num_cu / Hkv);
    const double shared = parts_us.size() > second ? parts_us[second] * (out.few ? 0.8 : 1.) : 0.;
    const size_t n = std::min(parts_us.size(), (size_t)std::max(1, slots / Hkv));
    place.assign(parts_us.begin(), parts_us.begin() + n);    // a heap: what each block's clock shows at its end
    std::make_heap(place.begin(), place.end(), std::greater<double>());
    double at = 0, clock = 0;
    for (size_t next = n; !place.empty();) {
      std::pop_heap(place.begin(), place.end(), std::greater<double>());
      const double busy = (double)place.size() * Hkv;
      at += (place.back() - clock) * busy / rate(busy);
      clock = place.back();
      place.pop_back();
      if (next == parts_us.size()) continue;
      place.push_back(clock + parts_us[next++]);
      std::push_heap(place.begin(), place.end(), std::greater<double>());
    }
    return std::max(at, shared) + join;
  };
  double best = longest, best_us = ends(longest);
  for (const double f : {3., 2., 1.5, 1., 0.75, 0.5, 0.35, 0.25}) {
    const double most = f * work / slots;
    if (most >= longest) continue;
    const double us = ends(most);
    if (us < best_us) {
      best = most;
      best_us = us;
    }
  }
  for (const Tile& t : tiles) {
    const auto [used, per] = parts_of(t, best);
    const int64_t row = out.part_rows;
    const bool joins = used > 1 && kvq_joins(t.cls, used, t.rows) && out.counters + (int64_t)Hkv * kKvqCounted <= kKvqCounters;
    if (used > 1) {
      if (!joins) out.units.push_back({t.q_start, t.row0, t.rows, (int32_t)row, used, t.rows, 0, 0, 0});
      out.part_rows += (int64_t)Hkv * used * t.rows;
      if (out.part_rows > kMaxPartRows)
        return plan_fail(err, SA_ERR_SHAPE, "too many query rows for one launch (partial results)");
    }
    if (used > 1 && !joins) {
      out.most_rows = std::max(out.most_rows, t.rows);
      out.most_parts = std::max(out.most_parts, used);
    }
    for (int h = 0; h < Hkv; ++h) {
      const int64_t part0 = row + (int64_t)h * used * t.rows;
      for (int s = 0; s < used; ++s)
        out.items.push_back({t.seq, h, t.row0, s * per * kKvqKeys,
                             (int32_t)std::min<int64_t>(t.keys, (int64_t)(s + 1) * per * kKvqKeys), t.cls, t.q_start,
                             h_q_len[t.seq], h_kv_len[t.seq], used > 1 ? (int32_t)(part0 + s * t.rows) : -1,
                             used > 1 ? (int32_t)part0 : -1, used, joins ? (int32_t)out.counters : -1});
      if (joins) out.counters += kKvqCounted;
    }
  }
  std::stable_sort(out.items.begin(), out.items.end(), [](const KvqItem& x, const KvqItem& y) {
    auto us = [](const KvqItem& it) { return (it.kv_end - it.kv_begin) * kKvqTileUs[it.cls]; };
    return us(x) > us(y);
  });
  return SA_OK;
}

}  // namespace sa
