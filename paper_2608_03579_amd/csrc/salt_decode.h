// Internal declarations of the operators that salt_decode.cpp launches: the rotation of query and key heads,
// the marks of a tracked cache, and beam search.  Not part of the public ABI (include/salt.h).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include <algorithm>

#include "salt_seqs.h"
#include "salt_serve.h"

namespace salt {

// ---- rotation ------------------------------------------------------------------------
constexpr int kMaxDim = 256;             // values of a head
constexpr double kMaxFreq = 1e4;         // radians per position
struct RotateArgs {
  const void *q, *k;        // [T][ld], head h at h * dim
  void *qo, *ko;
  int64_t ldq, ldk, ldqo, ldko;
  const void *qw, *kw;      // [dim], or null: no norm
  const int32_t* pos;       // [T]
  int32_t T, heads, kv_heads, dim, rot, interleaved;
  float eps, gain;
  double freq[kMaxDim / 2]; // revolutions per position of each pair
};
hipError_t launch_rotate(const RotateArgs& a, int bf16, int n_cu, hipStream_t s);

// ---- marks of a tracked cache ----------------------------------------------------------
// Arrays of the batch on the device.
struct BatchView {
  const int32_t* pages;     // page of each reference, the domains' first
  const int32_t *row, *count;         // of each own reference: first row of its tokens, tokens
  const int32_t* unit;      // sequence of each unit of own keys
  const SeqRec* rec;        // of each sequence
  int32_t pre_refs, own_refs, n_seqs, n_units;
};
struct ScoreArgs {
  AttArgs att;              // as for the attention (v, out and part are not used)
  BatchView b;
  const int32_t* back;      // [T]: new tokens of the sequence behind this one
  const int32_t* joined;    // [T]: the token's join, or -1: its rows are in one piece
  const int32_t* pos;       // [T], or null: places in the sequence
  float2* fin;              // [T][heads]: maximum (log2) and 1 / sum of a row's logits
  int32_t window;
  int32_t few, many;        // whether the batch has sequences of up to kFewRows counted rows, and of more
};
constexpr int64_t kScoreRow = (int64_t)1 << 24;   // elements between rows of q: 16 of them in 32-bit offsets
constexpr int kFewRows = 128;            // counted rows of a sequence (for each kv head) that one wave goes through
// Blocks of the pass that goes by keys, a block to every unit at most.
inline int64_t score_blocks(int64_t units, int kv_heads) { return units * kv_heads; }
hipError_t launch_score(const ScoreArgs& a, int bf16, hipStream_t s);
struct MarksArgs {
  KvLayer kv;
  BatchView b;
  float* weight;            // [own tokens][kv heads]
  int32_t* place;
};
hipError_t launch_marks(const MarksArgs& a, bool write, hipStream_t s);
constexpr int kEvictLen = 1 << 19;       // own tokens of a sequence: a bit each in LDS
struct EvictArgs {
  KvLayer kv;
  BatchView b;
  int32_t keep, recent, max_len;
};
hipError_t launch_evict(const EvictArgs& a, hipStream_t s);

// ---- beam search -------------------------------------------------------------------------
constexpr int kMaxBeams = 64;            // beams of a request, and
constexpr int kMaxOut = 64;              // continuations: a lane each
constexpr int kMaxSplits = 64;           // pieces of a row's vocabulary
constexpr int kMaxBeamRows = 1 << 16, kMaxVocab = 1 << 24;
constexpr int kSplitVocab = 4096;        // logits of a piece, at least
// Pieces that the vocabulary of each of `rows` rows is cut into: four blocks to a compute unit, where it has as many.
inline int beam_splits(int64_t rows, int vocab, int n_cu) {
  const int64_t want = ((int64_t)n_cu * 4 + rows - 1) / std::max<int64_t>(rows, 1);
  return (int)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(want, kMaxSplits), vocab / kSplitVocab));
}
// The most that any number of rows up to `max_rows` takes: rows * splits < 4 n_cu + 2 rows.
inline int64_t beam_pieces(int64_t max_rows, int n_cu) { return (int64_t)n_cu * 4 + 2 * max_rows; }
struct BeamArgs {
  const void* logits;       // [reqs * width][ld]
  const float* score;       // [reqs * width]
  int64_t ld;
  uint64_t* best;           // [rows][n_out][splits]: the pieces' best, (order of the value, ~token), 0: none
  double2* stat;            // [rows][splits]: maximum and sum of exponentials
  float* out_score;         // [reqs][n_out]
  int32_t *out_beam, *out_token;
  int32_t reqs, width, vocab, n_out, splits;
};
hipError_t launch_beam(const BeamArgs& a, int bf16, hipStream_t s);

// ---- copies of pages -----------------------------------------------------------------------
constexpr int kCopyPairs = 256;          // of one launch, in its arguments
struct CopyArgs {
  KvLayer kv;               // layer 0
  size_t layer, mark_layer; // bytes of a layer of the pool, and of the marks
  int32_t n_layers, n;
  int32_t src[kCopyPairs], dst[kCopyPairs];
  uint16_t tokens[kCopyPairs];
};
hipError_t launch_copy(const CopyArgs& a, hipStream_t s);

}  // namespace salt
