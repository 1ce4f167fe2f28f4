// How a batch of sequences is cut into the attention's work items.  Host arithmetic
// on the batch's lengths alone: no HIP types and no pointers into device memory.
//
// A row is one (token, query head).  The rows of one kv head that read the same keys
// form a row set: the new tokens of one sequence times the query heads of a kv head, or,
// for a domain prefix that two or more sequences share, those of all of them.  A row
// set is cut into row tiles of whole tokens, and the keys of a tile into runs ("pieces")
// of whole key units; a work item is one piece of one tile, run once per kv head.  A
// row whose keys are all in one piece is finished there; others leave (max, sum,
// weighted values) per piece, which a second kernel joins.
#pragma once

#include <stdint.h>

#include <algorithm>
#include <cmath>
#include <vector>

namespace salt {

constexpr int kKeyUnit = 64;       // keys of a unit; prefix and own keys start units of their own
constexpr int kRowTiles[4] = {16, 64, 128, 16};   // rows of a tile, by item kind (0: a block each, 3: a wave each)
constexpr int kMaxGroup = 64;      // query heads that share a kv head: a token's rows fit a tile of 64
// Rows of the largest tile: fp32 operands (three bf16 terms) and wide heads take the registers of the second 64.
constexpr int attend_rows(int esize, int dim) { return esize == 2 && dim <= 128 ? kRowTiles[2] : kRowTiles[1]; }

struct AttItem {
  int32_t kind;            // rows of the tile: kRowTiles[kind]
  int32_t n_rows;          // rows in use (per kv head)
  int32_t tok0;            // the tile's first entry of the token order
  int32_t pos0;            // own position of that token (>= 0 or below), or kAllKeys where the tile reads a prefix alone
  int32_t pre_ref, pre_len;// the prefix' first page reference and its keys (0: none)
  int32_t own_ref;         // the own keys' first page reference
  int32_t own_end;         // own keys the tile's last token sees
  int32_t unit0, unit1;    // the piece: units of the prefix, then of the own keys
  int32_t out_row;         // first row of the partial results (of kv head 0), or -1: the rows are finished here
  int32_t pad_;
};
constexpr int kAllKeys = 1 << 30;
// Pieces of one token, to be joined: `n` partial rows per query head, in two runs (its
// own item's, and its domain's).  It has keys: a shared prefix is not empty, and a tile whose first tokens stand
// before their sequence's first key, with no prefix, is too short to be cut.  Partial row of piece p, kv head k and row r of the
// tile: row + (p * n_kv_heads + k) * stride + r.
struct AttJoin {
  int32_t tok;
  int32_t row[2], n[2], stride[2], r0[2];   // r0: the token's first row in the tile
  int32_t pad_;
};

struct SeqBatch {
  int n_seqs, n_domains;
  const int32_t* q_len;
  const int32_t* len;
  const int32_t* page_off;     // sequences' page references, behind the domains'
  const int32_t* domain;       // may be null
  const int32_t* prefix_len;
  const int32_t* prefix_off;
};

struct AttWork {
  std::vector<AttItem> items;  // by kind, those of most rows first, the longest first
  int n_kind[4];
  std::vector<int32_t> order;  // token order of the shared row sets, behind the identity [0, T)
  std::vector<AttJoin> joins;
  int64_t rows;                // partial rows
};

// Of page reference `k` (from 0) of a holder of `len` tokens whose first is row `row`: its tokens, and the
// row of the first of them.  References past the last token have none.
inline int32_t page_count(int len, int page_tokens, int k) {
  return (int32_t)std::max<int64_t>(0, std::min<int64_t>(page_tokens, len - (int64_t)k * page_tokens));
}
inline int32_t page_row(int row, int len, int page_tokens, int k) {
  return page_count(len, page_tokens, k) > 0 ? row + k * page_tokens : row;
}

// Blocks of 256 threads that a launch can have: fewer than 2^32 threads along x.
constexpr int64_t kMaxBlocks = ((int64_t)1 << 24) - 1;
// The most blocks of a launch on the batch: its items, joins, new tokens (16 vectors a block) and own pages.
inline int64_t most_blocks(const AttWork& w, int T, int heads, int kv_heads, int own_refs) {
  const int64_t items = (int64_t)(w.n_kind[0] + w.n_kind[1] + w.n_kind[2]) * kv_heads +
                        ((int64_t)w.n_kind[3] * kv_heads + 3) / 4;
  const int64_t joins = ((int64_t)w.joins.size() * heads + 15) / 16, rows = ((int64_t)T * kv_heads + 15) / 16;
  return std::max(std::max(items, joins), std::max<int64_t>(rows, own_refs));
}

inline int seq_cdiv(int a, int b) { return (a + b - 1) / b; }

// Rows that a sequence brings alone from which on it keeps its prefix to itself: a tile of its own rows
// is full then, and sharing would only add a join.  8 sequences of 256 tokens and 3 heads behind
// two prefixes of 8192: 307 us, shared 335; of 20 tokens behind 4096 the two are alike (65 us), and below the
// prefix would be read once per sequence.
constexpr int kOwnRows = 128;

// Tiles of few rows: units (on average) up to which one wave works faster on a tile than a block,
// and units up to which a tile stays whole.
constexpr int kOneWaveUnits = 16, kWholeUnits = 8;

struct AttTile {
  AttItem it;
  int units, n_tok;
  bool joined;             // its tokens have a part elsewhere, too
};

// Partial rows that a plan of at most T tokens can need beyond two per row (pieces of
// long key runs): the cut below keeps to it.
constexpr int64_t kExtraRows = 1 << 16;
// Items of T tokens at most: two tiles to a token, and a piece beyond a tile's first brings a partial row
// for every head or more.
constexpr int64_t attend_max_items(int64_t T, int heads) { return 2 * T + kExtraRows / heads; }

// n_cu: compute units.  T: tokens of the batch (sum of q_len).  max_rows: attend_rows().
inline void cut_attention(const SeqBatch& b, int T, int heads, int kv_heads, int max_rows, int n_cu, AttWork& w) {
  const int gs = heads / kv_heads;
  w.items.clear();
  w.joins.clear();
  w.rows = 0;
  w.order.resize((size_t)T);
  for (int t = 0; t < T; ++t) w.order[(size_t)t] = t;
  auto kind_of = [&](int64_t rows) {
    return rows <= kRowTiles[0] ? 0 : (rows <= kRowTiles[1] || max_rows < kRowTiles[2] ? 1 : 2);
  };

  // sequences whose prefix is shared within the batch
  std::vector<int> users((size_t)b.n_domains, 0);
  auto shares = [&](int s) {
    return b.domain && b.domain[s] >= 0 && b.prefix_len[b.domain[s]] > 0 && b.q_len[s] > 0 &&
           (int64_t)b.q_len[s] * gs < kOwnRows;
  };
  for (int s = 0; s < b.n_seqs; ++s)
    if (shares(s)) users[(size_t)b.domain[s]]++;
  std::vector<AttTile> tiles;
  // each token's tile and first row in it: its own, and its prefix' where shared
  std::vector<int32_t> tok_tile((size_t)T, -1), tok_pre((size_t)T, -1), tok_r0((size_t)T), pre_r0((size_t)T);
  auto cut_set = [&](int first, int n_tok, int pos, int pre_ref, int pre_len, int own_ref, bool joined,
                     std::vector<int32_t>& of, std::vector<int32_t>& r0) {
    const int per = kRowTiles[kind_of((int64_t)n_tok * gs)] / gs;   // (a token's rows fit a tile of 64)
    for (int t = 0; t < n_tok; t += per) {
      AttTile x{};
      x.n_tok = std::min(per, n_tok - t);
      x.joined = joined;
      x.it.kind = kind_of((int64_t)x.n_tok * gs);
      x.it.n_rows = x.n_tok * gs;
      x.it.tok0 = first + t;
      x.it.pos0 = pos == kAllKeys ? kAllKeys : pos + t;
      x.it.pre_ref = pre_ref;
      x.it.pre_len = pre_len;
      x.it.own_ref = own_ref;
      x.it.own_end = pos == kAllKeys ? 0 : std::max(0, pos + t + x.n_tok);
      x.units = seq_cdiv(pre_len, kKeyUnit) + seq_cdiv(x.it.own_end, kKeyUnit);
      for (int j = 0; j < x.n_tok; ++j) {
        const size_t tok = (size_t)w.order[(size_t)(first + t + j)];
        of[tok] = (int32_t)tiles.size();
        r0[tok] = j * gs;
      }
      tiles.push_back(x);
    }
  };
  int t0 = 0;
  std::vector<int> first_tok((size_t)b.n_seqs);
  for (int s = 0; s < b.n_seqs; ++s) {
    first_tok[(size_t)s] = t0;
    const int n = b.q_len[s], d = b.domain ? b.domain[s] : -1;
    const bool shared = shares(s) && users[(size_t)d] > 1;
    const bool solo = d >= 0 && !shared;
    cut_set(t0, n, b.len[s] - n, solo ? b.prefix_off[d] : 0, solo ? b.prefix_len[d] : 0, b.page_off[s], shared,
            tok_tile, tok_r0);
    t0 += n;
  }
  // (the sequences by domain, each domain's in order)
  std::vector<int> user_at((size_t)b.n_domains + 1, 0);
  for (int d = 0; d < b.n_domains; ++d) user_at[(size_t)d + 1] = user_at[(size_t)d] + users[(size_t)d];
  std::vector<int> by_domain((size_t)user_at[(size_t)b.n_domains]), next(user_at.begin(), user_at.end() - 1);
  for (int s = 0; s < b.n_seqs; ++s)
    if (shares(s)) by_domain[(size_t)next[(size_t)b.domain[s]]++] = s;
  for (int d = 0; d < b.n_domains; ++d) {
    if (users[(size_t)d] < 2) continue;
    const int first = (int)w.order.size();
    for (int u = user_at[(size_t)d]; u < user_at[(size_t)d + 1]; ++u) {
      const int s = by_domain[(size_t)u];
      for (int j = 0; j < b.q_len[s]; ++j) w.order.push_back(first_tok[(size_t)s] + j);
    }
    cut_set(first, (int)w.order.size() - first, kAllKeys, b.prefix_off[d], b.prefix_len[d], 0, true, tok_pre,
            pre_r0);
  }

  // Tiles of few rows.  A block of four waves splits its keys between the waves; one wave each
  // where the keys are few and the tiles many enough to give every SIMD one.  Of single tokens, 8 kv
  // heads, block and wave: 64 sequences of 150 keys 8.9 and 12.1 us, 128 of 150 18.0 and 13.8, 256 of 600
  // 82 and 69, 128 of 2000 114 and 129.
  auto wide = [](const AttTile& x) { return x.it.kind == 1 || x.it.kind == 2; };
  int64_t few = 0, few_units = 0;
  for (const AttTile& x : tiles)
    if (!wide(x)) ++few, few_units += x.units;
  const bool one_wave = few * kv_heads >= (int64_t)n_cu * 4 && few_units <= few * kOneWaveUnits;
  if (one_wave)
    for (AttTile& x : tiles)
      if (!wide(x)) x.it.kind = 3;
  // Their pieces: an item for every compute unit, but no more pieces than the join is worth, which
  // reads them one after the other: 16384 keys of one sequence take 42 us in pieces of 2 units, 19 of 8, 30 of
  // 32; 65000 keys 159, 57 and 37.  A join costs 3 us by itself: 150 keys 9.2 us in two pieces, 6.6 in one.
  // One wave's tiles that are joined anyway are cut to kWholeUnits, or the last ones to start end
  // long after the rest: 256 sequences of up to 1024 keys behind 16 prefixes of up to 4096 61 to 67 us
  // from batch to batch, uncut 66 to 88.
  const int64_t fill = (few_units * kv_heads + n_cu - 1) / n_cu;
  auto few_pieces = [&](const AttTile& x, int64_t least) {
    if (x.units <= kWholeUnits) return 1;
    const int64_t worth = std::max(fill, (int64_t)std::ceil(std::sqrt((double)x.units) / 2));
    const int64_t run = std::max(least, one_wave && x.joined ? (int64_t)kWholeUnits : worth);
    return (int)((x.units + run - 1) / run);
  };
  std::vector<int32_t> n_piece(tiles.size(), 1), row_of(tiles.size(), -1);
  int64_t few_extra = 0;
  for (int64_t least = 1;; least *= 2) {
    few_extra = 0;
    for (size_t i = 0; i < tiles.size(); ++i)
      if (!wide(tiles[i])) {
        n_piece[i] = few_pieces(tiles[i], least);
        few_extra += (int64_t)(n_piece[i] - 1) * tiles[i].it.n_rows * kv_heads;
      }
    if (few_extra <= kExtraRows) break;
  }
  // Tiles of many rows: the longest one in 1 to 16 pieces, the others in pieces as long, whichever
  // count is estimated to end first.
  int longest = 0;
  int64_t units = 0, few_blocks = 0;
  for (size_t i = 0; i < tiles.size(); ++i) {
    if (wide(tiles[i])) longest = std::max(longest, tiles[i].units), units += tiles[i].units;
    else few_blocks += n_piece[i];
  }
  // of the tiles of few rows: blocks (of four waves), and their work in units of the others
  const double few_work = (double)few_units * kv_heads * (one_wave ? 0.25 : 0.2);
  few_blocks = few_blocks * kv_heads / (one_wave ? 4 : 1);
  int best_run = std::max(1, longest);
  double best = 1e300;
  for (int p = 1, last = 0; p <= 16; ++p) {
    const int run = std::max(1, seq_cdiv(longest, p));
    if (p > 1 && (run < 4 || run == last)) continue;
    last = run;
    int64_t n = 0, parts = 0, extra = few_extra, part_rows = 0;
    for (const AttTile& x : tiles)
      if (wide(x)) {
        const int k = std::max(1, seq_cdiv(x.units, run));
        n += (int64_t)k * kv_heads;
        parts += k - 1;
        extra += (int64_t)(k - 1) * x.it.n_rows * kv_heads;
        if (k > 1) part_rows += (int64_t)k * x.it.n_rows * kv_heads;
      }
    if (p > 1 && (extra > kExtraRows || parts > (int64_t)n_cu * 8)) break;
    // In the time of a unit: rounds of two blocks a compute unit, of which one that has it to itself takes
    // 0.65 of the time, half a unit to begin and end a piece, the longest piece's end alone, and
    // where rows are joined a launch and 15000 partial rows to the unit.  Measured with 8 kv heads and
    // groups of 4, whole and in 2, 3 and 4 pieces: 16 x 40 tokens of 2000 keys 73, 57, 71, 71 us; 2048
    // tokens of 8192 287, 311; 256 tokens of 4096 128, 78, 61, 52.
    const int64_t blocks = n + few_blocks, full = blocks / (2 * n_cu), rest = blocks % (2 * n_cu);
    const double rounds = (double)full + (rest == 0 ? 0. : rest <= n_cu ? 0.65 : 1.);
    const double mean = ((double)units * kv_heads + few_work) / (double)std::max<int64_t>(blocks, 1);
    const double time = std::max(rounds * (mean + 0.5), 0.65 * run + 0.35 * (blocks > n_cu ? mean : 0.)) +
                        (part_rows ? 1.5 + (double)part_rows / 15000 : 0.);
    if (time < best) best = time, best_run = run;
  }
  for (size_t i = 0; i < tiles.size(); ++i)
    if (wide(tiles[i])) n_piece[i] = std::max(1, seq_cdiv(tiles[i].units, best_run));
  // a tile is finished in its one item unless its tokens have others
  std::vector<uint8_t> joined(tiles.size(), 0);
  for (int t = 0; t < T; ++t) {
    const int a = tok_tile[(size_t)t], p = tok_pre[(size_t)t];
    if (p >= 0) joined[(size_t)a] = joined[(size_t)p] = 1;
    else if (n_piece[(size_t)a] > 1) joined[(size_t)a] = 1;
  }
  for (size_t i = 0; i < tiles.size(); ++i) {
    AttTile& x = tiles[i];
    if (joined[i]) {
      row_of[i] = (int32_t)w.rows;
      w.rows += (int64_t)n_piece[i] * kv_heads * x.it.n_rows;
    }
    for (int p = 0; p < n_piece[i]; ++p) {
      AttItem it = x.it;
      it.unit0 = (int)((int64_t)x.units * p / n_piece[i]);
      it.unit1 = (int)((int64_t)x.units * (p + 1) / n_piece[i]);
      it.out_row = joined[i] ? row_of[i] + p * kv_heads * it.n_rows : -1;
      w.items.push_back(it);
    }
  }
  std::stable_sort(w.items.begin(), w.items.end(), [](const AttItem& a, const AttItem& c) {
    const int p = a.kind == 3 ? -1 : a.kind, q = c.kind == 3 ? -1 : c.kind;
    return p != q ? p > q : a.unit1 - a.unit0 > c.unit1 - c.unit0;
  });
  std::fill(w.n_kind, w.n_kind + 4, 0);
  for (const AttItem& it : w.items) w.n_kind[it.kind]++;
  for (int t = 0; t < T; ++t) {
    const int tile[2] = {tok_tile[(size_t)t], tok_pre[(size_t)t]};
    if (!joined[(size_t)tile[0]]) continue;
    AttJoin j{};
    j.tok = t;
    for (int k = 0; k < 2; ++k) {
      if (tile[k] < 0) continue;
      const AttTile& x = tiles[(size_t)tile[k]];
      j.row[k] = row_of[(size_t)tile[k]];
      j.n[k] = n_piece[(size_t)tile[k]];
      j.stride[k] = x.it.n_rows;
      j.r0[k] = k == 0 ? tok_r0[(size_t)t] : pre_r0[(size_t)t];
    }
    w.joins.push_back(j);
  }
}

}  // namespace salt
