// Host check of the attention's cut (salt_seqs.h built without HIP): a token whose partial results are joined sees
// at least one key.  The join relies on it to tell a sum of 0 (every logit -inf) from a row without keys.  Random batches,
// many of whose sequences bring more new tokens than they have.  Prints the first failure and exits 1, else "ok".
#include <cstdio>
#include <random>
#include <vector>

#include "salt_seqs.h"

using namespace salt;

int main() {
  std::mt19937 rng(2609);
  auto pick = [&](int lo, int hi) { return std::uniform_int_distribution<int>(lo, hi)(rng); };
  long joined = 0, without = 0;
  for (int trial = 0; trial < 300; ++trial) {
    const int kv_heads = 1 << pick(0, 3), gs = std::vector<int>{1, 2, 3, 4, 8, 17, 64}[pick(0, 6)];
    const int n = trial % 4 ? pick(1, 12) : pick(100, 300), nd = pick(0, 3), n_cu = trial % 3 ? 256 : pick(1, 20);
    std::vector<int32_t> q(n), len(n), dom(n), pre(nd), off(n + 1, 0), pre_off(nd + 1, 0);
    for (int d = 0; d < nd; ++d) pre[d] = pick(0, 2) ? pick(0, 3000) : 0;
    int T = 0;
    for (int i = 0; i < n; ++i) {
      q[i] = n > 50 ? pick(0, 2) : pick(0, 2) ? pick(0, 5) : pick(0, 500);
      len[i] = pick(0, 2) ? q[i] + pick(0, n > 50 ? 90 : 4000) : pick(0, q[i]);
      dom[i] = pick(-1, nd - 1);
      T += q[i];
    }
    AttWork w;
    cut_attention(SeqBatch{n, nd, q.data(), len.data(), off.data(), dom.data(), pre.data(), pre_off.data()}, T,
                  kv_heads * gs, kv_heads, trial % 2 ? 128 : 64, n_cu, w);
    std::vector<int> keys(T);
    for (int i = 0, t = 0; i < n; ++i)
      for (int j = 0; j < q[i]; ++j, ++t) {
        keys[t] = (dom[i] >= 0 ? pre[dom[i]] : 0) + std::max(0, len[i] - q[i] + j + 1);
        without += keys[t] == 0;
      }
    for (const AttJoin& j : w.joins) {
      ++joined;
      if (keys[j.tok] == 0) {
        std::printf("FAIL trial %d: token %d is joined and has no keys\n", trial, j.tok);
        return 1;
      }
    }
  }
  if (joined < 1000 || without < 500) {
    std::printf("FAIL too few joined tokens (%ld) or tokens without keys (%ld)\n", joined, without);
    return 1;
  }
  std::printf("ok\n");
}
