// Host-only checks of branch_plan.h (forks and shared-prefix attention), built
// with AddressSanitizer and UndefinedBehaviorSanitizer by tests/test_branches_cpu.py.
//
// Over seeded random shapes it checks that
//   * a fork plan matches a direct page-by-page count, and refuses bad arguments;
//   * the shared-prefix work list sees every (query row, visible key) pair
//     exactly once, each item's pages are its group's or its member's, partials
//     do not overlap, and every row split over parts is in one merge unit
//     that names exactly the rows of the partials that hold it; a batch that is
//     passed on has no items.
// Prints "ALL OK" and exits 0 on success.
#include <cstdio>
#include <cstdlib>
#include <map>
#include <random>
#include <set>
#include <tuple>
#include <vector>

#include "branch_plan.h"

static int g_fail = 0, g_shared = 0, g_passed_on = 0;
#define CHECK(cond, ...)                                                   \
  do {                                                                     \
    if (!(cond)) {                                                         \
      std::fprintf(stderr, "FAIL %s:%d: %s: ", __FILE__, __LINE__, #cond); \
      std::fprintf(stderr, __VA_ARGS__);                                   \
      std::fprintf(stderr, "\n");                                          \
      if (++g_fail > 20) std::exit(1);                                     \
    }                                                                      \
  } while (0)

static sa_layout layout(int Hq, int Hkv, int P) {
  sa_layout L;
  L.num_q_heads = Hq;
  L.num_kv_heads = Hkv;
  L.head_dim = 128;
  L.page_size = P;
  L.num_layers = 1;
  L.num_slots = 1 << 20;
  return L;
}

static void fork_case(std::mt19937_64& r, int id) {
  const int P = r() % 2 ? 16 : 32, B = 1 + r() % 5, C = 1 + r() % 12;
  sa_layout L = layout(8, 2, P);
  std::vector<int32_t> len(B), parent(C), reserve(C);
  for (int& x : len) x = r() % 4 == 0 ? 0 : r() % 200;
  for (int& x : parent) x = (int)(r() % B);
  for (int& x : reserve) x = r() % 3 == 0 ? 0 : (int)(r() % 100);
  int64_t fresh = 0, entries = 0;
  for (int c = 0; c < C; ++c) {
    const int pages = (len[parent[c]] + reserve[c] + P - 1) / P;
    entries += pages;
    fresh += pages - len[parent[c]] / P;
  }
  sa::ForkPlan plan;
  std::string err;
  auto go = [&](int nf, int cap) {
    return sa::plan_fork(&L, B, len.data(), C, parent.data(), reserve.data(), nf, cap, plan, err);
  };
  CHECK(go((int)fresh, (int)entries) == SA_OK, "case %d: %s", id, err.c_str());
  CHECK(plan.n_dst == entries && plan.fresh_used == fresh, "case %d", id);
  int64_t at = 0, used = 0;
  size_t copies = 0;
  for (int c = 0; c < C; ++c) {
    const sa::ForkChild& ch = plan.children[c];
    const int n = len[parent[c]], pages = (n + reserve[c] + P - 1) / P;
    CHECK(ch.parent == parent[c] && ch.full == n / P && ch.rows == n % P && ch.dst0 == at && ch.fresh0 == used,
          "case %d child %d", id, c);
    CHECK(plan.dst_indptr[c] == at, "case %d child %d", id, c);
    int others = 0, before = 0;
    for (int x = 0; x < C; ++x) {
      others += parent[x] == parent[c];
      before += x < c && parent[x] == parent[c];
    }
    CHECK(ch.raise == (before ? 0 : others), "case %d child %d: raises counts by %d", id, c, ch.raise);
    if (n % P) {
      CHECK(copies < plan.copies.size() && plan.copies[copies] == c, "case %d child %d", id, c);
      CHECK(pages > n / P, "case %d: the partial page's copy has a slot", id);
      ++copies;
    }
    at += pages;
    used += pages - n / P;
  }
  CHECK(copies == plan.copies.size(), "case %d", id);
  if (fresh > 0) CHECK(go((int)fresh - 1, (int)entries) == SA_ERR_NO_PAGES, "case %d", id);
  if (entries > 0) CHECK(go((int)fresh, (int)entries - 1) == SA_ERR_NO_PAGES, "case %d", id);
  std::vector<int32_t> bad = parent;
  bad[C - 1] = B;
  CHECK(sa::plan_fork(&L, B, len.data(), C, bad.data(), reserve.data(), 1 << 20, 1 << 20, plan, err) == SA_ERR_RANGE,
        "case %d", id);
  bad = reserve;
  bad[0] = -1;
  CHECK(sa::plan_fork(&L, B, len.data(), C, parent.data(), bad.data(), 1 << 20, 1 << 20, plan, err) == SA_ERR_SHAPE,
        "case %d", id);
}

static void shared_case(std::mt19937_64& r, int id) {
  const int Hkv = 1 << (r() % 4);
  const int Gs[] = {1, 2, 3, 4, 5, 8, 16};
  const int G = Gs[r() % 7];
  sa_layout L = layout(Hkv * G, Hkv, r() % 2 ? 16 : 32);
  const int groups = 1 + r() % 6;
  std::vector<int32_t> indptr{0}, shared, q, kv;
  for (int g = 0; g < groups; ++g) {
    const int n = r() % 5 == 0 ? (int)(r() % 2) : (int)(r() % 20);
    const int S = r() % 4 == 0 ? (int)(r() % 70) : (int)(r() % (r() % 3 ? 3000 : 30000));
    shared.push_back(S);
    for (int i = 0; i < n; ++i) {
      const int ql = r() % 6 == 0 ? 0 : r() % 3 == 0 ? (int)(1 + r() % 90) : 1;
      q.push_back(ql);
      kv.push_back(S + ql + (int)(r() % 2 ? 0 : r() % 300));
    }
    indptr.push_back((int)q.size());
  }
  const int B = (int)q.size();
  if (B == 0) return;
  std::string err;
  std::vector<sa::SeqDesc> seqs;
  int64_t total = 0;
  CHECK(sa::plan_attn_check(&L, 0, B, q.data(), kv.data(), 1.f, seqs, total, err) == SA_OK, "case %d", id);
  CHECK(sa::check_groups(B, q.data(), kv.data(), groups, indptr.data(), shared.data(), err) == SA_OK, "case %d: %s",
        id, err.c_str());
  sa::SharedPlan plan;
  const int cus[] = {1, 8, 64, 256};
  sa::plan_shared_items(&L, seqs, groups, indptr.data(), shared.data(), cus[r() % 4], plan);
  if (!plan.shared) {
    CHECK(plan.items.empty() && plan.units.empty(), "case %d", id);
    ++g_passed_on;
    return;
  }
  ++g_shared;
  std::vector<int> seq_of(total), group_of(B);
  for (int b = 0; b < B; ++b)
    for (int t = 0; t < q[b]; ++t) seq_of[seqs[b].q_start + t] = b;
  for (int g = 0; g < groups; ++g)
    for (int b = indptr[g]; b < indptr[g + 1]; ++b) group_of[b] = g;
  // (token, head) -> keys seen, and the rows of its partials
  typedef std::tuple<int, int> Row;                  // token, query head
  std::map<Row, std::vector<std::pair<int, int>>> keys;
  std::map<Row, std::vector<int>> places;
  std::map<Row, int> whole;
  std::set<int> parts;
  for (const sa::AttnItem& it : plan.items) {
    if (it.kv_end <= it.kv_begin) continue;
    CHECK(it.kv_begin % sa::kKT == 0, "case %d", id);
    const int pre = it.kv_len - it.q_len;
    for (int x = 0; x < 128; ++x) {
      const int row = it.row0 + x;
      if (row >= it.q_len * G) break;
      const int tok = row / G, head = it.kvh * G + row % G;
      const int end = std::min(it.kv_end, pre + tok + 1);   // keys the kernel shows this row
      const int b = seq_of[it.q_start + tok];
      CHECK(end <= kv[b] - q[b] + (it.q_start + tok - seqs[b].q_start) + 1, "case %d: a key past the row's own", id);
      CHECK(it.seq == b || (group_of[it.seq] == group_of[b] && it.kv_end <= shared[group_of[b]] / 64 * 64),
            "case %d: pages of another sequence", id);
      if (end > it.kv_begin) keys[Row(it.q_start + tok, head)].push_back({it.kv_begin, end});
      if (it.part >= 0) {
        CHECK(parts.insert(it.part + x).second && it.part + x < plan.part_rows, "case %d: partial row %d", id, it.part + x);
        places[Row(it.q_start + tok, head)].push_back(it.part + x);
      }
      else whole[Row(it.q_start + tok, head)]++;
    }
  }
  CHECK((int64_t)parts.size() == plan.part_rows, "case %d", id);
  std::map<Row, std::vector<int>> merged;
  for (const sa::MergeUnit& u : plan.units) {
    CHECK(u.n >= 1 && u.n <= sa::kMergeUnitRows, "case %d: %d rows", id, u.n);
    for (int i = 0; i < u.n * Hkv; ++i) {
      const int x = i % u.n, h = i / u.n, row = u.r0 + x;
      auto& m = merged[Row(u.q_start + row / G, h * G + row % G)];
      CHECK(m.empty(), "case %d: a row in two units", id);
      for (int k = 0; k < u.a_n; ++k) m.push_back(u.a_row + (h * u.a_n + k) * u.a_stride + x);
      for (int k = 0; k < u.b_n; ++k) m.push_back(u.b_row + (h * u.b_n + k) * u.b_stride + x);
    }
  }
  for (int b = 0; b < B; ++b)
    for (int t = 0; t < q[b]; ++t)
      for (int h = 0; h < Hkv * G; ++h) {
        const Row row(seqs[b].q_start + t, h);
        auto k = keys[row];
        std::sort(k.begin(), k.end());
        int at = 0;
        for (auto& x : k) {
          CHECK(x.first == at, "case %d: keys from %d, %d seen", id, x.first, at);
          at = x.second;
        }
        CHECK(at == kv[b] - q[b] + t + 1, "case %d: %d keys of %d", id, at, kv[b] - q[b] + t + 1);
        auto p = places[row], m = merged[row];
        std::sort(p.begin(), p.end());
        std::sort(m.begin(), m.end());
        CHECK(p == m, "case %d: the merge of token %d head %d", id, seqs[b].q_start + t, h);
        CHECK((whole[row] == 1) == p.empty(), "case %d: written whole and in parts", id);
      }
}

int main() {
  std::mt19937_64 r(11);
  for (int i = 0; i < 2000; ++i) fork_case(r, i);
  for (int i = 0; i < 600; ++i) shared_case(r, i);
  CHECK(g_shared > 50 && g_passed_on > 50, "%d shared, %d passed on", g_shared, g_passed_on);
  // refusals
  sa_layout L = layout(8, 2, 16);
  std::string err;
  const int32_t q[] = {1, 1}, kv[] = {10, 9}, ip[] = {0, 2}, sh[] = {8};
  CHECK(sa::check_groups(2, q, kv, 1, ip, sh, err) == SA_OK, "%s", err.c_str());
  const int32_t far[] = {9}, neg[] = {-1}, shrt[] = {0, 1}, back[] = {0, 2, 1, 2}, three[] = {0, 0, 0};
  CHECK(sa::check_groups(2, q, kv, 1, ip, far, err) == SA_ERR_SHAPE, "shared beyond a member's cache");
  CHECK(sa::check_groups(2, q, kv, 1, ip, neg, err) == SA_ERR_SHAPE, "negative");
  CHECK(sa::check_groups(2, q, kv, 1, shrt, sh, err) == SA_ERR_SHAPE, "not the whole batch");
  CHECK(sa::check_groups(2, q, kv, 3, back, three, err) == SA_ERR_SHAPE, "decreasing");
  CHECK(sa::check_groups(2, q, kv, 0, ip, sh, err) == SA_ERR_SHAPE, "no group");
  CHECK(sa::check_groups(2, q, kv, 1, nullptr, sh, err) == SA_ERR_NULL, "null");
  // debug checks of a fork
  const int32_t len[] = {20}, parent[] = {0, 0}, res[] = {4, 16};
  sa::ForkPlan plan;
  CHECK(sa::plan_fork(&L, 1, len, 2, parent, res, 8, 8, plan, err) == SA_OK, "%s", err.c_str());
  const int32_t tip[] = {0, 2}, tix[] = {5, 6}, fr[] = {1, 2, 3}, dup[] = {1, 2, 1}, used[] = {1, 6, 3}, out[] = {1, 2, 99};
  CHECK(plan.fresh_used == 3, "%lld", (long long)plan.fresh_used);
  CHECK(sa::debug_check_fork(plan, tip, tix, fr, 16, err) == SA_OK, "%s", err.c_str());
  CHECK(sa::debug_check_fork(plan, tip, tix, dup, 16, err) == SA_ERR_OVERLAP, "repeat");
  CHECK(sa::debug_check_fork(plan, tip, tix, used, 16, err) == SA_ERR_OVERLAP, "page of a source");
  CHECK(sa::debug_check_fork(plan, tip, tix, out, 16, err) == SA_ERR_RANGE, "out of range");
  const int32_t short_ip[] = {0, 1};
  CHECK(sa::debug_check_fork(plan, short_ip, tix, fr, 16, err) == SA_ERR_RANGE, "short table");
  if (g_fail) return 1;
  std::puts("ALL OK");
  return 0;
}
