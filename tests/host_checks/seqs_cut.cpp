// Host walk of the attention's work items (salt_seqs.h built without HIP).  For seeded random
// batches it simulates what the kernels do with the items: which (token, kv head) rows an item
// covers, which keys of the prefix and of the sequence each row sees there, and where it
// leaves its part; then what the joins read.  It checks:
//  - every row sees every key it should, once: the whole prefix of its domain and its
//    sequence's keys up to its own place, and no other holder's pages;
//  - an item's rows fit its kind, its units lie inside its tile, its page references inside the holder's;
//  - parts that are finished directly have no other parts; partial rows are disjoint, inside the
//    announced number, and read by their token's join exactly once;
//  - the numbers that salt_seqs_create provides buffers for (items, token order, joins, rows) suffice.
// Prints the first failure and exits 1, else prints "ok".
#include <cstdio>
#include <cstdlib>
#include <map>
#include <random>
#include <set>
#include <tuple>
#include <vector>

#include "salt_seqs.h"

using namespace salt;

static void need(bool ok, const char* what, long a = 0, long b = 0, long c = 0) {
  if (ok) return;
  std::printf("FAIL %s (%ld %ld %ld)\n", what, a, b, c);
  std::exit(1);
}

int main() {
  std::mt19937 rng(2608);
  auto pick = [&](int lo, int hi) { return std::uniform_int_distribution<int>(lo, hi)(rng); };
  const int kPage = 16;
  int kinds_seen[4] = {0, 0, 0, 0}, long_runs = 0;
  for (int trial = 0; trial < 600; ++trial) {
    const int kv_heads = 1 << pick(0, 3), gs = std::vector<int>{1, 2, 3, 4, 5, 8, 16, 17, 40, 64}[pick(0, 9)];
    const int heads = kv_heads * gs, n_cu = trial % 3 ? 256 : pick(1, 20), max_rows = trial % 2 ? 128 : 64;
    const int n = trial % 5 == 0 ? pick(100, 400) : pick(0, 12), nd = pick(0, 4);
    std::vector<int32_t> q_len(n), len(n), domain(n), pre(nd), off(n + 1), pre_off(nd + 1);
    for (int d = 0; d < nd; ++d) {
      pre[d] = pick(0, 4) ? pick(0, 700) : 0;
      pre_off[d + 1] = pre_off[d] + (pre[d] + kPage - 1) / kPage;
    }
    off[0] = pre_off[nd];
    int T = 0;
    for (int i = 0; i < n; ++i) {
      q_len[i] = n > 50 ? pick(0, 2) : (pick(0, 3) ? pick(0, 5) : pick(0, 400));
      len[i] = pick(0, 6) ? q_len[i] + pick(0, n > 50 ? 60 : 2500) : pick(0, q_len[i]);
      domain[i] = pick(-1, nd - 1);
      off[i + 1] = off[i] + (len[i] + kPage - 1) / kPage;
      T += q_len[i];
    }
    const bool no_domains = trial % 7 == 0;
    const SeqBatch b{n, no_domains ? 0 : nd, q_len.data(), len.data(), off.data(), no_domains ? nullptr : domain.data(),
                     pre.data(), pre_off.data()};
    AttWork w;
    cut_attention(b, T, heads, kv_heads, max_rows, n_cu, w);
    need(w.items.size() <= 2 * (size_t)T + n + nd + 16 * (size_t)n_cu, "items", (long)w.items.size(), T, n);
    need(w.order.size() <= 2 * (size_t)T && w.joins.size() <= (size_t)T, "order, joins");
    need(w.rows <= 2 * (int64_t)T * heads + kExtraRows, "partial rows", (long)w.rows);
    std::vector<int> seq_of(T), in_seq(T);
    for (int i = 0, t = 0; i < n; ++i)
      for (int j = 0; j < q_len[i]; ++j, ++t) seq_of[t] = i, in_seq[t] = j;
    // what each token sees: (prefix?, key) -> times, of one kv head (all are alike)
    std::vector<std::map<std::pair<int, int>, int>> seen(T);
    std::vector<int> direct(T, 0), parts(T, 0);
    std::map<int64_t, std::tuple<int, int>> part_row;         // partial row -> (token, query head)
    int kind_before = 3, count[4] = {0, 0, 0, 0};
    for (const AttItem& it : w.items) {
      const int rank = it.kind == 3 ? -1 : it.kind;
      need(it.kind >= 0 && it.kind <= 3 && rank <= kind_before, "kinds in order", it.kind);
      kind_before = rank;
      count[it.kind]++;
      kinds_seen[it.kind]++;
      need(it.n_rows > 0 && it.n_rows <= kRowTiles[it.kind] && it.n_rows % gs == 0, "rows of the item", it.n_rows);
      need(it.kind != 2 || max_rows == 128, "a tile of 128 rows");
      const int n_pre = (it.pre_len + kKeyUnit - 1) / kKeyUnit;
      const int units = n_pre + (it.own_end + kKeyUnit - 1) / kKeyUnit;
      need(0 <= it.unit0 && it.unit0 <= it.unit1 && it.unit1 <= units, "units", it.unit0, it.unit1, units);
      if (it.unit1 - it.unit0 > 40) long_runs++;
      for (int r = 0; r < it.n_rows; r += gs) {
        need(it.tok0 + r / gs < (int)w.order.size(), "token order");
        const int t = w.order[it.tok0 + r / gs], s = seq_of[t], d = no_domains ? -1 : domain[s];
        const int lim = std::min(it.pos0 + r / gs + 1, it.own_end);
        if (it.pre_len) need(d >= 0 && it.pre_ref == pre_off[d] && it.pre_len == pre[d], "another domain's prefix", t);
        if (it.own_end) need(it.own_ref == off[s] && it.own_end <= len[s], "another sequence's pages", t);
        for (int u = it.unit0; u < it.unit1; ++u) {
          const bool own = u >= n_pre;
          const int j0 = kKeyUnit * (own ? u - n_pre : u), end = own ? std::min(lim, it.own_end) : it.pre_len;
          for (int j = j0; j < std::min(end, j0 + kKeyUnit); ++j) seen[t][{own, j}]++;
        }
        if (it.out_row < 0) direct[t]++;
        else {
          parts[t]++;
          for (int k = 0; k < kv_heads; ++k)
            for (int h = 0; h < gs; ++h) {
              const int64_t row = (int64_t)it.out_row + (int64_t)k * it.n_rows + r + h;
              need(row >= 0 && row < w.rows, "partial row", (long)row, (long)w.rows);
              need(part_row.emplace(row, std::make_tuple(t, k * gs + h)).second, "partial rows overlap", (long)row);
            }
        }
      }
    }
    for (int k = 0; k < 4; ++k) need(count[k] == w.n_kind[k], "numbers of kinds", k);
    for (int t = 0; t < T; ++t) {
      const int s = seq_of[t], d = no_domains ? -1 : domain[s];
      const int np = d >= 0 ? pre[d] : 0, no = std::max(0, len[s] - q_len[s] + in_seq[t] + 1);
      need((int)seen[t].size() == np + no, "keys of a row", t, (long)seen[t].size(), np + no);
      for (const auto& e : seen[t]) need(e.second == 1, "a key seen more than once", t, e.first.second);
      need((direct[t] == 1 && parts[t] == 0) || (direct[t] == 0 && parts[t] >= 1), "finished once", t, direct[t], parts[t]);
    }
    std::vector<int> joined(T, 0);
    for (const AttJoin& j : w.joins) {
      joined[j.tok]++;
      need(j.n[0] + j.n[1] == parts[j.tok], "parts of a join", j.tok, j.n[0] + j.n[1], parts[j.tok]);
      for (int h = 0; h < heads; ++h)
        for (int k = 0; k < 2; ++k)
          for (int p = 0; p < j.n[k]; ++p) {
            const int64_t row = (int64_t)j.row[k] + (int64_t)(p * kv_heads + h / gs) * j.stride[k] + j.r0[k] + h % gs;
            const auto at = part_row.find(row);
            need(at != part_row.end() && at->second == std::make_tuple((int)j.tok, h), "a join reads another row", j.tok, h);
            part_row.erase(at);
          }
    }
    need(part_row.empty(), "partial rows that no join reads", (long)part_row.size());
    for (int t = 0; t < T; ++t) need(joined[t] == (parts[t] > 0), "one join to a token in parts", t);
  }
  for (int k = 0; k < 4; ++k) need(kinds_seen[k] > 0, "every kind occurs", k);
  need(long_runs > 0, "long runs occur");
  std::printf("ok\n");
}
