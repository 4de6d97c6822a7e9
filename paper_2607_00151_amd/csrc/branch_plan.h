// Host-side planning of the calls that keep several branches of one context
// alive: the fork of cached contexts and the attention of a batch whose
// members share a prefix.  Plain C++17 with no HIP dependency, like plan.h.
//
// The records defined here are also the device-side plan formats, so they are
// plain int32 structs.
#pragma once

#include <tuple>

#include "plan.h"

namespace sa {

// ------------------------------------------------------------------ fork

// One child of a fork: the first `full` pages of its table are its parent's,
// the others fresh slots from position `fresh0` of the free list on, the first
// of which takes `rows` rows of the parent's partial page (0: it has none).  raise:
// what the shared pages' counts rise by with this child's entries -- the number of
// the parent's children for the first of them, 0 for the others.
struct ForkChild {
  int32_t parent, full, rows, fresh0, dst0, raise;
};

struct ForkPlan {
  std::vector<ForkChild> children;
  std::vector<int32_t> dst_indptr;     // [children + 1]
  std::vector<int32_t> copies;         // children with a partial page
  int64_t n_dst = 0, fresh_used = 0;
};

inline sa_status plan_fork(const sa_layout* layout, int32_t batch, const int32_t* h_src_len, int32_t num_children,
                           const int32_t* h_parent, const int32_t* h_reserve, int32_t num_fresh, int32_t dst_capacity,
                           ForkPlan& out, std::string& err) {
  sa_status s = check_layout(layout, err);
  if (s != SA_OK) return s;
  if (batch < 1) return plan_fail(err, SA_ERR_SHAPE, "batch %d < 1", batch);
  if (num_children < 1) return plan_fail(err, SA_ERR_SHAPE, "num_children %d < 1", num_children);
  if (!h_src_len || !h_parent || !h_reserve) return plan_fail(err, SA_ERR_NULL, "a host array is NULL");
  if (num_fresh < 0 || dst_capacity < 0) return plan_fail(err, SA_ERR_SHAPE, "negative capacity");
  for (int b = 0; b < batch; ++b)
    if (h_src_len[b] < 0) return plan_fail(err, SA_ERR_SHAPE, "sequence %d: src_len %d", b, h_src_len[b]);
  const int P = layout->page_size;
  out = ForkPlan{};
  out.dst_indptr.assign((size_t)num_children + 1, 0);
  std::vector<int32_t> first((size_t)batch, -1);               // first child of each sequence
  for (int c = 0; c < num_children; ++c) {
    const int b = h_parent[c];
    if (b < 0 || b >= batch) return plan_fail(err, SA_ERR_RANGE, "child %d: parent %d outside [0, %d)", c, b, batch);
    if (h_reserve[c] < 0) return plan_fail(err, SA_ERR_SHAPE, "child %d: reserve %d", c, h_reserve[c]);
    const int64_t len = h_src_len[b], full = len / P, rows = len % P;
    const int64_t pages = (len + h_reserve[c] + P - 1) / P;
    if (out.n_dst + pages > INT32_MAX - 1024) return plan_fail(err, SA_ERR_SHAPE, "destination table too large");
    if (first[b] < 0) first[b] = c;
    out.children.push_back({b, (int32_t)full, (int32_t)rows, (int32_t)out.fresh_used, (int32_t)out.n_dst, 0});
    ++out.children[first[b]].raise;
    if (rows > 0) out.copies.push_back(c);
    out.n_dst += pages;
    out.fresh_used += pages - full;
    out.dst_indptr[c + 1] = (int32_t)out.n_dst;
  }
  if (out.fresh_used > num_fresh)
    return plan_fail(err, SA_ERR_NO_PAGES, "need %lld fresh slots, %d given", (long long)out.fresh_used, num_fresh);
  if (out.n_dst > dst_capacity)
    return plan_fail(err, SA_ERR_NO_PAGES, "destination table needs %lld entries, capacity %d", (long long)out.n_dst,
                     dst_capacity);
  return SA_OK;
}

// SA_DEBUG check of a fork against host copies of the source table and of the
// free list's first entries: every page in range, the fresh slots distinct and
// none of them a page of a source context.
inline sa_status debug_check_fork(const ForkPlan& plan, const int32_t* indptr, const int32_t* indices,
                                  const int32_t* fresh, int64_t num_slots, std::string& err) {
  std::vector<int32_t> used;
  for (size_t c = 0; c < plan.children.size(); ++c) {
    const ForkChild& ch = plan.children[c];
    const int32_t pages = ch.full + (ch.rows > 0);
    const int32_t have = indptr[ch.parent + 1] - indptr[ch.parent];
    if (pages > have)
      return plan_fail(err, SA_ERR_RANGE, "child %d: its parent's table has %d of %d pages", (int)c, have, pages);
    for (int j = 0; j < pages; ++j) {
      const int32_t slot = indices[indptr[ch.parent] + j];
      if (slot < 0 || slot >= num_slots)
        return plan_fail(err, SA_ERR_RANGE, "sequence %d: page %d has slot %d outside [0, %lld)", ch.parent, j, slot,
                         (long long)num_slots);
      used.push_back(slot);
    }
  }
  std::sort(used.begin(), used.end());
  std::vector<int32_t> taken(fresh, fresh + plan.fresh_used);
  std::sort(taken.begin(), taken.end());
  for (size_t i = 0; i < taken.size(); ++i) {
    if (taken[i] < 0 || taken[i] >= num_slots)
      return plan_fail(err, SA_ERR_RANGE, "a free-list entry is slot %d, outside [0, %lld)", taken[i],
                       (long long)num_slots);
    if (i > 0 && taken[i] == taken[i - 1])
      return plan_fail(err, SA_ERR_OVERLAP, "slot %d appears twice in the free list", taken[i]);
    if (std::binary_search(used.begin(), used.end(), taken[i]))
      return plan_fail(err, SA_ERR_OVERLAP, "fresh slot %d is also a page of a source context", taken[i]);
  }
  return SA_OK;
}

// ------------------------------------------------------------------ shared prefix

// Rows of one member whose parts the merge joins, of every KV head: packed rows
// r0 .. r0 + n - 1 of the member whose first token is q_start.  Of the rows that
// partials are kept by, row r0's of KV head 0 are a_row, a_row + a_stride, ... (a_n
// of them: the shared prefix) and b_row, b_row + b_stride, ... (b_n: the member's
// own keys), the next rows' follow each, and the next KV head's are a_n * a_stride
// and b_n * b_stride further.
struct MergeUnit {
  int32_t q_start, r0, n;
  int32_t a_row, a_n, a_stride;
  int32_t b_row, b_n, b_stride;
};
constexpr int64_t kMaxPartRows = INT32_MAX - 1024;   // rows of all partials: places are int32
constexpr int kMergeUnitRows = 32;     // most rows of a unit
// rows per block of the merge, for rows of at most so many parts
inline int merge_block_rows(int most_parts) { return most_parts <= 8 ? 8 : most_parts <= 16 ? 4 : most_parts <= 32 ? 2 : 1; }

// part of an item: the row its partial starts at among all partials (-1: none)
struct SharedPlan {
  bool shared = false;                 // some group's prefix is computed once for its members
  std::vector<uint8_t> once;           // per group: its prefix is computed once (where shared)
  std::vector<AttnItem> items;         // one per workgroup, in launch order
  std::vector<MergeUnit> units;
  int64_t part_rows = 0;               // rows of all partials
  int32_t most_rows = 0, most_parts = 0;   // of a unit
};

inline sa_status check_groups(int32_t batch, const int32_t* h_q_len, const int32_t* h_kv_len, int32_t num_groups,
                              const int32_t* h_group_indptr, const int32_t* h_shared_len, std::string& err) {
  if (num_groups < 1) return plan_fail(err, SA_ERR_SHAPE, "num_groups %d < 1", num_groups);
  if (!h_group_indptr || !h_shared_len) return plan_fail(err, SA_ERR_NULL, "h_group_indptr / h_shared_len is NULL");
  if (h_group_indptr[0] != 0 || h_group_indptr[num_groups] != batch)
    return plan_fail(err, SA_ERR_SHAPE, "group_indptr must run from 0 to the batch size %d", batch);
  for (int g = 0; g < num_groups; ++g)
    if (h_group_indptr[g + 1] < h_group_indptr[g])
      return plan_fail(err, SA_ERR_SHAPE, "group_indptr decreases at %d", g);
  for (int g = 0; g < num_groups; ++g) {
    if (h_shared_len[g] < 0) return plan_fail(err, SA_ERR_SHAPE, "group %d: shared_len %d", g, h_shared_len[g]);
    for (int b = h_group_indptr[g]; b < h_group_indptr[g + 1]; ++b)
      if (h_shared_len[g] > h_kv_len[b] - h_q_len[b])
        return plan_fail(err, SA_ERR_SHAPE, "group %d: shared_len %d beyond the %d cached tokens of sequence %d", g,
                         h_shared_len[g], h_kv_len[b] - h_q_len[b], b);
  }
  return SA_OK;
}

// SA_DEBUG check of the groups against a host copy of the page table: every page
// of a shared prefix in range in the tables of all members with query rows.  Where
// a member lists another slot than the member whose pages are read, `differ` names
// both, whose first `rows` rows have to be equal copies.
struct SharedCopy {
  int32_t group, seq, of, page, slot, of_slot, rows;     // page of sequence seq, and of sequence `of`
};

inline sa_status debug_check_shared(int32_t num_groups, const int32_t* h_group_indptr, const int32_t* h_shared_len,
                                    const int32_t* h_q_len, const int32_t* indptr, const int32_t* indices, int P,
                                    int64_t num_slots, std::vector<SharedCopy>& differ, std::string& err) {
  differ.clear();
  for (int g = 0; g < num_groups; ++g) {
    const int32_t S = h_shared_len[g];
    const int64_t pages = ((int64_t)S + P - 1) / P;
    int first = -1;
    for (int b = h_group_indptr[g]; b < h_group_indptr[g + 1]; ++b) {
      if (h_q_len[b] == 0) continue;
      if (first < 0) first = b;
      if (pages > indptr[b + 1] - indptr[b])
        return plan_fail(err, SA_ERR_RANGE, "sequence %d: its table has %d of the %lld pages that group %d shares", b,
                         indptr[b + 1] - indptr[b], (long long)pages, g);
      for (int32_t j = 0; j < pages; ++j) {
        const int32_t slot = indices[indptr[b] + j], of = indices[indptr[first] + j];
        if (slot < 0 || slot >= num_slots)
          return plan_fail(err, SA_ERR_RANGE, "sequence %d: page %d has slot %d outside [0, %lld)", b, j, slot,
                           (long long)num_slots);
        if (slot != of) differ.push_back({g, b, first, j, slot, of, std::min<int32_t>(P, S - j * P)});
      }
    }
  }
  return SA_OK;
}

// Row tiles of one KV head that the choice of a chunk need not tell apart.
struct SharedShape {
  int64_t tiles;             // 64-key tiles of each
  bool decode;               // takes the kernel's path for few rows
  bool streams;              // reads its keys from memory (a group's other row tiles find them in L2)
  int64_t count, rows;       // how many, and their packed rows in all
};

inline int64_t shared_parts(int64_t tiles, int64_t chunk) {
  return std::max<int64_t>(1, std::min<int64_t>((tiles + chunk - 1) / chunk, kMaxItemParts));
}

// Time of the two launches at a chunk size, in units of 10 ns.  Measured
// (MI355X): a prefill tile 120 and a block's start and end 400 where at most one
// long prefill block has each CU, 185 and 900 where two share one; a decode tile 80 and
// its block 300; the keys stream at 54.6 per tile and 100 blocks (6 TB/s), with a
// quarter of the shorter of work and stream not overlapping; the merge 530, and
// 1032 bytes written and read per row and part at 9 TB/s.
inline int64_t shared_chunk_cost(const std::vector<SharedShape>& shapes, int Hkv, int num_cu, int64_t chunk) {
  struct Run {
    int64_t time, blocks;
  };
  std::vector<Run> runs;
  int64_t n = 0, n_long = 0, longest = 0, streamed = 0, part_rows = 0;
  auto length = [&](const SharedShape& s) { return (s.tiles + shared_parts(s.tiles, chunk) - 1) / shared_parts(s.tiles, chunk); };
  for (const SharedShape& s : shapes)
    if (!s.decode) longest = std::max(longest, length(s));
  for (const SharedShape& s : shapes) {
    const int64_t k = shared_parts(s.tiles, chunk);
    n += k * Hkv * s.count;
    if (!s.decode && 2 * length(s) > longest) n_long += k * Hkv * s.count;
    part_rows += k * Hkv * s.rows;
    if (s.streams) streamed += s.tiles * Hkv * s.count;
  }
  const bool pairs = n_long > num_cu;
  for (const SharedShape& s : shapes) {
    const int64_t k = shared_parts(s.tiles, chunk), t = length(s);
    runs.push_back({s.decode ? t * 80 + 300 : pairs ? t * 185 + 900 : t * 120 + 400, k * Hkv * s.count});
  }
  std::sort(runs.begin(), runs.end(), [](const Run& x, const Run& y) { return x.time > y.time; });
  // the busiest of the slots: the mean, and of any k slots + 1 longest blocks some slot has k + 1
  const int64_t slots = (n > num_cu ? 2 : 1) * (int64_t)num_cu;
  int64_t sum = 0, before = 0, busy = 0;
  for (const Run& r : runs) {
    sum += r.time * r.blocks;
    before += r.blocks;
    busy = std::max(busy, ((before - 1) / slots + 1) * r.time);
  }
  busy = std::max(busy, sum / slots);
  const int64_t stream = streamed * 546 / 1000;
  return std::max(busy, stream) + std::min(busy, stream) / 4 + 530 + part_rows * 1032 / 90000;
}

// The same work by sa_segment_prefill_attn, every member over all of its keys:
// the larger of its throughput (members' repeated reads of the shared keys come
// out of the caches, 14 TB/s over all; row tiles at two blocks per CU) and of the
// slowest item's way through its parts and their merge, whose costs are those that
// plan_attn_items splits by; 700 for the launch, 1400 for the partials of 512
// prefill parts.
inline int64_t segment_cost(const std::vector<SeqDesc>& seqs, int G, int Hkv, int num_cu) {
  int64_t stream = 0, compute = 0, items = 0;
  for (const SeqDesc& s : seqs) {
    const int64_t rows = (int64_t)s.q_len * G, tiles = ((int64_t)s.kv_len + kKT - 1) / kKT * Hkv;
    if (rows == 0) continue;
    items += (rows + 127) / 128 * Hkv;
    if (rows <= kDecodeRows) stream += tiles;
    else compute += tiles * ((rows + 127) / 128);
  }
  const int64_t slots = 2 * (int64_t)num_cu;
  const double least = (double)(stream + compute) / slots;    // tiles of a part where the slots are shared evenly
  double slowest = 0, parts = 0;
  for (const SeqDesc& s : seqs) {
    const double rows = (double)s.q_len * G, t = (double)(((int64_t)s.kv_len + kKT - 1) / kKT);
    if (rows == 0) continue;
    const bool decode = rows <= kDecodeRows;
    const double finest = decode ? std::sqrt(rows * t / 64) : std::sqrt(t / 2);
    const double c = items >= slots ? t : std::min(t, std::max({4.0, finest, least}));
    const double k = t / c;
    slowest = std::max(slowest, decode ? 60 * c + (k > 1 ? 1.25 * rows * k : 0) : 93 * c + (k > 1 ? 60 * k : 0));
    if (!decode && k > 1) parts += k * Hkv * std::ceil(rows / 128);
  }
  const int64_t flow = std::max(stream * 234 / 1000, compute * 180 / slots) + stream * 80 / slots / 4;
  return 700 + std::max(flow, (int64_t)slowest) + (int64_t)(1400 * parts / 512);
}

// The launch's work items.  A group whose prefix is computed once gives row
// tiles of all its members' packed rows over the keys [0, S), S its shared
// length rounded down to whole 64-key tiles, and row tiles of each member over
// [S, kv_len); every other member gives row tiles over all of its keys.  Tiles
// are split by key range into parts; a tile that is the only one to see its
// rows and has one part writes the output itself.  Where no group's prefix is
// worth it, out.shared is false and there are no items.
inline void plan_shared_items(const sa_layout* layout, const std::vector<SeqDesc>& seqs, int32_t num_groups,
                              const int32_t* h_group_indptr, const int32_t* h_shared_len, int num_cu,
                              SharedPlan& out) {
  const int Hkv = layout->num_kv_heads, G = layout->num_q_heads / Hkv;
  constexpr int kRows = 128;
  out = SharedPlan{};
  struct Tile {
    int32_t seq, row0, rows, q_start, q_len, kv_len, k0, k1;   // rows: of this tile
    bool prefix;
    int32_t parts = 1;
    int64_t place = -1;                                         // row of its first part, KV head 0, among the partials
    int64_t tiles() const { return ((int64_t)k1 - k0 + kKT - 1) / kKT; }
  };
  std::vector<Tile> tiles;
  struct Member {
    int32_t seq, prefix0, row_in_group, own0;                  // first prefix tile of its group (-1), its first row there
  };
  std::vector<Member> members;
  bool any = false;
  out.once.assign((size_t)num_groups, 0);
  for (int g = 0; g < num_groups; ++g) {
    const int b0 = h_group_indptr[g], b1 = h_group_indptr[g + 1];
    int64_t rows = 0, apart = 0, active = 0;
    int first = -1;
    for (int b = b0; b < b1; ++b) {
      const int64_t r = (int64_t)seqs[b].q_len * G;
      rows += r;
      active += r > 0;
      apart += (r + kRows - 1) / kRows;
      if (first < 0 && r > 0) first = b;
    }
    if (first < 0) continue;
    const int32_t S = h_shared_len[g] / kKT * kKT;
    // Worth it where packing the members' rows leaves clearly fewer row tiles over
    // the prefix: every row then goes through partials.  8 segments of 45 to 64 tokens
    // on 16K, us with the prefix computed once and member by member: 12 row tiles of
    // 16 112 and 116, 13 of 16 125 and 125, 14 of 16 132 and 125, 16 of 16 145 and 137.
    // With more than kDecodeRows rows a member the two partials of a row tile cost
    // about as much as 20 key tiles, which the tiles saved have to outweigh: 16
    // segments of 36 tokens on 4K (18 tiles of 32, 64 key tiles) 63 and 68, of 45
    // (23 of 32) 74 and 67; 51 of 4 to 26 on 130, 32/4 heads, 30 and 20.
    const int64_t packed = (rows + kRows - 1) / kRows;
    const bool shared = S > 0 && rows + S <= INT32_MAX / 2 && 5 * packed <= 4 * apart &&
                        (rows <= (int64_t)kDecodeRows * active || (apart - packed) * (S / kKT) >= 20 * apart);
    const int32_t prefix0 = shared ? (int32_t)tiles.size() : -1;
    if (shared) {
      any = true;
      out.once[g] = 1;
      const int32_t q_len = (int32_t)(rows / G);
      for (int64_t r0 = 0; r0 < rows; r0 += kRows)
        tiles.push_back({first, (int32_t)r0, (int32_t)std::min<int64_t>(kRows, rows - r0), seqs[first].q_start, q_len,
                         S + q_len, 0, S, true});
    }
    int64_t at = 0;
    for (int b = b0; b < b1; ++b) {
      const SeqDesc& q = seqs[b];
      const int32_t n = q.q_len * G;
      if (n == 0) continue;
      members.push_back({b, prefix0, (int32_t)at, (int32_t)tiles.size()});
      for (int r0 = 0; r0 < n; r0 += kRows) {
        const int last = std::min(r0 + kRows, n) - 1;
        tiles.push_back({b, r0, last + 1 - r0, q.q_start, q.q_len, q.kv_len, shared ? S : 0,
                         q.kv_len - q.q_len + last / G + 1, false});
      }
      at += n;
    }
  }
  if (!any) return;

  // Key-range parts of one chunk size, the one that the model ends first.
  std::map<std::tuple<int64_t, bool, bool>, std::pair<int64_t, int64_t>> classes;
  int64_t longest = 1;
  for (const Tile& t : tiles) {
    auto& c = classes[{t.tiles(), (int64_t)t.q_len * G <= kDecodeRows, !t.prefix || t.row0 == 0}];
    ++c.first;
    c.second += t.rows;
    longest = std::max(longest, t.tiles());
  }
  std::vector<SharedShape> shapes;
  for (const auto& c : classes)
    shapes.push_back({std::get<0>(c.first), std::get<1>(c.first), std::get<2>(c.first), c.second.first, c.second.second});
  int64_t best = INT64_MAX;
  int64_t chunk = longest;
  const int64_t most = std::min<int64_t>(64, (longest + 3) / 4);
  for (int64_t k = 1; k <= most; k += 1 + k / 8) {
    const int64_t c = std::min(std::max<int64_t>((longest + k - 1) / k, 4), longest);
    const int64_t t = shared_chunk_cost(shapes, Hkv, num_cu, c);
    if (t < best) {
      best = t;
      chunk = c;
    }
  }
  if (best >= segment_cost(seqs, G, Hkv, num_cu)) return;
  out.shared = true;

  int64_t rows_used = 0;
  for (Tile& t : tiles) t.parts = (int32_t)shared_parts(t.tiles(), chunk);
  auto place = [&](Tile& t) {
    t.place = rows_used;
    rows_used += (int64_t)t.parts * Hkv * t.rows;
  };
  for (const Member& m : members) {
    const int32_t n = seqs[m.seq].q_len * G;
    for (int32_t r0 = 0, t = m.own0; r0 < n; r0 += kRows, ++t)
      if (m.prefix0 >= 0 || tiles[t].parts > 1) place(tiles[t]);
  }
  for (Tile& t : tiles)
    if (t.prefix) place(t);
  out.part_rows = rows_used;
  if (rows_used > kMaxPartRows) return;                         // refused by the caller

  auto part_begin = [](const Tile& t, int k) { return t.tiles() * k / t.parts; };   // in tiles from t.k0
  // blocks: longest first, the row tiles of one key range next to each other on
  // one XCD (block i runs on XCD i % 8), which reads it through its L2 once.  Parts of
  // one length throughout: of 58 batches with one to two prefix parts per CU, parts of
  // two lengths with the members' own blocks between them were 2.7% slower in the
  // geometric mean (0.82 to 1.14 of the time; 64 branches of 64K 171 and 173 us, 16
  // segments of 16 to 64 tokens on 16K 188 and 182).
  struct Bundle {
    int64_t length;                                              // tiles of each of its items
    int32_t tile, count, kvh, part;                              // row tiles tile .. tile + count - 1
  };
  std::vector<Bundle> bundles;
  for (size_t i = 0; i < tiles.size();) {
    size_t j = i + 1;
    while (j < tiles.size() && tiles[i].prefix && tiles[j].prefix && tiles[j].seq == tiles[i].seq) ++j;
    for (int k = 0; k < tiles[i].parts; ++k) {
      const int64_t length = part_begin(tiles[i], k + 1) - part_begin(tiles[i], k);
      for (int h = 0; h < Hkv; ++h) bundles.push_back({length, (int32_t)i, (int32_t)(j - i), h, k});
    }
    i = j;
  }
  std::stable_sort(bundles.begin(), bundles.end(), [](const Bundle& x, const Bundle& y) { return x.length > y.length; });
  std::vector<int32_t> queue[kNumXcd];                          // bundles
  int64_t load[kNumXcd] = {0};
  size_t blocks[kNumXcd] = {0}, depth = 0;
  for (size_t i = 0; i < bundles.size(); ++i) {
    const Bundle& b = bundles[i];
    const int x = (int)(std::min_element(load, load + kNumXcd) - load);
    load[x] += b.length * b.count;
    queue[x].push_back((int32_t)i);
    blocks[x] += b.count;
    depth = std::max(depth, blocks[x]);
  }
  out.items.assign(depth * kNumXcd, AttnItem{0, 0, 0, 0, 0, -1, 0, 0, 0, 0});
  for (int x = 0; x < kNumXcd; ++x) {
    size_t at = 0;
    for (int32_t i : queue[x]) {
      const Bundle& b = bundles[i];
      for (int32_t y = b.tile; y < b.tile + b.count; ++y) {
        const Tile& t = tiles[y];
        AttnItem it{t.seq, b.kvh, t.row0, 0, 0, -1, 0, t.q_start, t.q_len, t.kv_len};
        it.kv_begin = (int32_t)(t.k0 + part_begin(t, b.part) * kKT);
        it.kv_end = (int32_t)std::min<int64_t>(t.k0 + part_begin(t, b.part + 1) * kKT, t.k1);
        if (t.place >= 0) it.part = (int32_t)(t.place + ((int64_t)b.kvh * t.parts + b.part) * t.rows);
        out.items[at++ * kNumXcd + x] = it;
      }
    }
  }

  // merge units: rows of one member, one own tile and one prefix tile
  for (const Member& m : members) {
    const int32_t n = seqs[m.seq].q_len * G;
    for (int32_t r = 0; r < n;) {
      const Tile& own = tiles[m.own0 + r / kRows];
      int32_t e = std::min(r + kMergeUnitRows, std::min(own.row0 + own.rows, n));
      MergeUnit u{seqs[m.seq].q_start, r, 0, 0, 0, 0, (int32_t)own.place + r - own.row0, own.parts, own.rows};
      if (m.prefix0 >= 0) {
        const Tile& pre = tiles[m.prefix0 + (m.row_in_group + r) / kRows];
        e = std::min(e, pre.row0 + kRows - m.row_in_group);
        u.a_row = (int32_t)pre.place + m.row_in_group + r - pre.row0;
        u.a_n = pre.parts;
        u.a_stride = pre.rows;
      }
      u.n = e - r;
      r = e;
      if (own.place < 0) continue;
      out.units.push_back(u);
      out.most_rows = std::max(out.most_rows, u.n);
      out.most_parts = std::max(out.most_parts, u.a_n + u.b_n);
    }
  }
}

}  // namespace sa
