// The numbers that buffers for a batch's work items are sized by (salt_seqs.h built without HIP), at batches
// that cut their tiles into the most pieces: many single tokens of few heads whose key runs are a little
// longer than the pieces, alone and in pairs behind prefixes.  Prints the first failure and exits 1, else "ok".
#include <cstdio>
#include <vector>

#include "salt_seqs.h"

using namespace salt;

int main() {
  for (int kv_heads : {1, 2, 8})
    for (int gs : {1, 4})
      for (int n : {1, 7, 300, 2048, 16384})
        for (int units : {9, 16, 17, 40})
          for (int pairs = 0; pairs < 2; ++pairs) {
            // every 16th holder is short, so that the mean stays at 16 units or below beside runs of 17
            const int nd = pairs ? n / 2 : 0, heads = kv_heads * gs;
            auto run = [&](int i) { return i % 16 == 15 ? 1 : units * kKeyUnit; };
            std::vector<int32_t> q(n, 1), len(n), dom(n, -1), pre(nd), off(n + 1), pre_off(nd + 1);
            for (int d = 0; d < nd; ++d) pre[d] = run(d), pre_off[d + 1] = pre_off[d] + pre[d] / 16 + 1;
            off[0] = pre_off[nd];
            for (int i = 0; i < n; ++i) {
              len[i] = run(i);
              if (i / 2 < nd) dom[i] = i / 2;
              off[i + 1] = off[i] + len[i] / 16 + 1;
            }
            AttWork w;
            cut_attention(SeqBatch{n, nd, q.data(), len.data(), off.data(), dom.data(), pre.data(), pre_off.data()}, n,
                          heads, kv_heads, kRowTiles[2], 256, w);
            if ((int64_t)w.items.size() > attend_max_items(n, heads) ||
                w.rows > 2 * (int64_t)n * heads + kExtraRows || (int)w.order.size() > 2 * n || (int)w.joins.size() > n) {
              std::printf("FAIL %d sequences, %d domains of %d units, %d / %d heads: %zu items (at most %lld), %lld rows\n",
                          n, nd, units, heads, kv_heads, w.items.size(), (long long)attend_max_items(n, heads),
                          (long long)w.rows);
              return 1;
            }
          }
  std::printf("ok\n");
}
