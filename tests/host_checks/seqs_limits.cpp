// Host arithmetic of a batch at its limits (salt_seqs.h built without HIP): page references far past a holder's
// last token have no tokens (their place passes 32 bits), and batches whose launches would have 2^32
// threads or more are seen.  Prints the first failure and exits 1, else "ok".
#include <cstdio>
#include <vector>

#include "salt_seqs.h"

using namespace salt;

static int fail(const char* what, long a) {
  std::printf("FAIL %s (%ld)\n", what, a);
  return 1;
}

int main() {
  for (int pt : {16, 64, 256})
    for (int len : {0, 1, 15, 16, 17, 300, 1 << 28}) {
      long tokens = 0;
      const int row = 1000, pages = (len + pt - 1) / pt;
      for (int k = 0; k < pages; ++k) {
        if (page_row(row, len, pt, k) != row + (long)k * pt) return fail("row", k);
        tokens += page_count(len, pt, k);
      }
      if (tokens != len) return fail("tokens", tokens);
      for (long k : {(long)pages, (long)pages + 1, 1L << 23, (1L << 23) + 1, (1L << 24) - 1})
        if (k >= pages && (page_count(len, pt, (int)k) != 0 || page_row(row, len, pt, (int)k) != row))
          return fail("a page past the end", k);
    }
  // 2^20 single tokens of 256 kv heads: a wave each; and in pairs behind prefixes, joined
  for (int kv_heads : {1, 8, 256})
    for (int shared = 0; shared < 2; ++shared) {
      const int n = 1 << 20, nd = shared ? n / 2 : 0;
      std::vector<int32_t> q(n, 1), len(n, 1), dom(n, -1), off(n + 1), pre(nd, 1), pre_off(nd + 1);
      for (int d = 0; d <= nd; ++d) pre_off[d] = d;
      for (int i = 0; i <= n; ++i) off[i] = nd + i;
      if (shared)
        for (int i = 0; i < n; ++i) dom[i] = i / 2;
      AttWork w;
      cut_attention(SeqBatch{n, nd, q.data(), len.data(), off.data(), dom.data(), pre.data(), pre_off.data()}, n,
                    kv_heads, kv_heads, kRowTiles[2], 256, w);
      const long got = most_blocks(w, n, kv_heads, kv_heads, n);
      const long waves = (long)w.items.size() * kv_heads;
      if (got < (waves + 3) / 4 || got < (long)w.joins.size() * kv_heads / 16 || got < n) return fail("blocks", got);
      if ((kv_heads == 256) != (got > kMaxBlocks)) return fail("refused", got);
    }
  std::printf("ok\n");
}
