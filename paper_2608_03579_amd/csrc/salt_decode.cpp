// libsalt host runtime, the operators of a decoding server around the attention: the rotation of query and key
// heads, the marks of a tracked cache with its eviction, beam search, and copies of cache pages
// (include/salt.h).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

#include "salt.h"
#include "salt_decode.h"
#include "salt_objects.h"
#include "salt_seqs.h"
#include "salt_serve.h"

using salt::aligned16;
using salt::ctx_fail;

struct salt_beams {
  int32_t max_rows = 0, max_out = 0;
  int64_t entries = 0, pieces = 0;    // of the buffers
  uint64_t* best = nullptr;
  double2* stat = nullptr;
  salt::StreamOrder order;
};

namespace {

constexpr double kTurn = 6.283185307179586476925286766559;

void free_beams(void* p) {
  salt_beams* b = static_cast<salt_beams*>(p);
  if (b->best) (void)hipFree(b->best);
  if (b->stat) (void)hipFree(b->stat);
  b->order.destroy();
  delete b;
}

// Whether a page of the batch holds own tokens twice, or beside a prefix: from its tables as `staging` still has
// them, once for a batch, when it is first asked for.  (A visit to every page: salt_seqs_set of 64 sequences of 4096 tokens
// in pages of 16 takes 44 us without it, 58 with it.)
bool shares_pages(salt_seqs* q) {
  if (q->shared >= 0) return q->shared;
  const int32_t* d = q->staging + (size_t)q->stage * q->words;
  const int32_t* pages = d + q->at_page;
  const int32_t pre_refs = q->n_refs - q->n_own_refs;
  uint32_t* stamp = q->kv->stamp.data();
  const uint32_t now = salt::next_stamp(q->kv);
  for (int i = 0; i < q->n_domains; ++i)
    for (int k = 0; k < d[q->at_prefix + 2 * i + 1]; ++k) stamp[pages[d[q->at_prefix + 2 * i] + k]] = now;
  bool twice = false;
  for (int r = 0; r < q->n_own_refs; ++r) {
    if (d[q->at_count + r] == 0) continue;
    uint32_t& s = stamp[pages[pre_refs + r]];
    twice |= s == now;
    s = now;
  }
  q->shared = twice;
  return twice;
}

// A call on the marks of a set batch.
salt_status marks_call(salt_ctx* ctx, salt_seqs* q, int32_t layer, bool changes) {
  const salt_status st = salt::batch_call(ctx, q, layer);
  if (st != SALT_OK) return st;
  if (!q->kv->marks) return ctx_fail(ctx, SALT_ERR_BAD_STATE, "the cache is not tracked (salt_kv_track)");
  if (changes && shares_pages(q))
    return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "a page holds tokens of two sequences of the batch, or of a sequence and a prefix");
  return SALT_OK;
}

salt::BatchView view_of(const salt_seqs* q) {
  salt::BatchView b{};
  b.pages = q->dev + q->at_page;
  b.row = q->dev + q->at_row;
  b.count = q->dev + q->at_count;
  b.unit = q->dev + q->at_unit;
  b.rec = reinterpret_cast<const salt::SeqRec*>(q->dev + q->at_rec);
  b.pre_refs = q->n_refs - q->n_own_refs;
  b.own_refs = q->n_own_refs;
  b.n_seqs = q->n_seqs;
  b.n_units = q->n_units;
  return b;
}

salt_status marks_copy(salt_ctx* ctx, salt_seqs* q, int32_t layer, float* weight, int32_t* place, void* stream,
                       bool write) {
  salt_status st = marks_call(ctx, q, layer, write);
  if (st != SALT_OK) return st;
  if (q->own_tokens == 0) return SALT_OK;
  if (!weight || !aligned16(weight) || !place || !aligned16(place))
    return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "null or misaligned marks");
  const salt::CtxView cv = salt::ctx_view(ctx);
  SERVE_HIP(ctx, hipSetDevice(cv.device));
  const hipStream_t s = (hipStream_t)stream;
  if ((st = salt::enter(ctx, q, s)) != SALT_OK) return st;
  salt::MarksArgs a{};
  a.kv = salt::layer_of(q->kv, layer);
  a.b = view_of(q);
  a.weight = weight;
  a.place = place;
  SERVE_HIP(ctx, salt::launch_marks(a, write, s));
  if (write) q->given[(size_t)layer] = 1;
  return SALT_OK;
}

}  // namespace

extern "C" {

// ---- rotation -------------------------------------------------------------------------------
salt_status salt_rotate(salt_ctx* ctx, const salt_rotation* r, int32_t T, const int32_t* pos, const void* q, int64_t ldq,
                        void* q_out, int64_t ldqo, const void* k, int64_t ldk, void* k_out, int64_t ldko, void* stream) {
  SERVE_LIVE(ctx);
  if (!r) return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "null argument");
  if (r->n_heads < 0 || r->n_kv_heads < 0 || r->n_heads > 65536 || r->n_kv_heads > 65536 || r->n_heads + r->n_kv_heads < 1)
    return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "%d query and %d key heads", r->n_heads, r->n_kv_heads);
  if (r->head_dim < 8 || r->head_dim > salt::kMaxDim || r->head_dim % 8 != 0)
    return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "head_dim must be a multiple of 8 in [8, %d]", salt::kMaxDim);
  if (r->rot_dim < 8 || r->rot_dim > r->head_dim || r->rot_dim % 8 != 0)
    return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "rot_dim must be a multiple of 8 in [8, head_dim]");
  if (r->interleaved != 0 && r->interleaved != 1) return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "interleaved is 0 or 1");
  if (!r->freq) return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "null frequencies");
  if (!std::isfinite(r->gain)) return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "gain must be finite");
  if (!std::isfinite(r->eps) || r->eps < 0.f) return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "eps must be finite and >= 0");
  if (!aligned16(r->q_norm) || !aligned16(r->k_norm)) return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "misaligned norm weights");
  for (int i = 0; i < r->rot_dim / 2; ++i)
    if (!std::isfinite(r->freq[i]) || std::fabs(r->freq[i]) > salt::kMaxFreq)
      return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "frequency %d is not in [-%g, %g]", i, salt::kMaxFreq, salt::kMaxFreq);
  if (T < 0 || T > (1 << 20)) return ctx_fail(ctx, SALT_ERR_OUT_OF_RANGE, "T = %d not in [0, 2^20]", T);
  if (T == 0) return SALT_OK;
  if (!pos || (reinterpret_cast<uintptr_t>(pos) & 3u)) return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "null or misaligned positions");
  salt_status st = SALT_OK;
  auto rows = [&](const char* what, int heads, const void* in, int64_t& ldi, void* out, int64_t& ldo) {
    const int64_t width = (int64_t)heads * r->head_dim;
    salt_status e = salt::rows_arg(ctx, what, in, ldi, width);
    if (e == SALT_OK) e = salt::rows_arg(ctx, what, out, ldo, width);
    if (e == SALT_OK && in == out && ldi != ldo)
      e = ctx_fail(ctx, SALT_ERR_INVALID_ARG, "%s in place with rows of %lld and %lld elements", what, (long long)ldi, (long long)ldo);
    return e;
  };
  if (r->n_heads > 0) st = rows("q", r->n_heads, q, ldq, q_out, ldqo);
  if (st == SALT_OK && r->n_kv_heads > 0) st = rows("k", r->n_kv_heads, k, ldk, k_out, ldko);
  if (st != SALT_OK) return st;
  const salt::CtxView v = salt::ctx_view(ctx);
  SERVE_HIP(ctx, hipSetDevice(v.device));
  salt::RotateArgs a{};
  a.q = q;
  a.k = k;
  a.qo = q_out;
  a.ko = k_out;
  a.ldq = ldq;
  a.ldk = ldk;
  a.ldqo = ldqo;
  a.ldko = ldko;
  a.qw = r->q_norm;
  a.kw = r->k_norm;
  a.pos = pos;
  a.T = T;
  a.heads = r->n_heads;
  a.kv_heads = r->n_kv_heads;
  a.dim = r->head_dim;
  a.rot = r->rot_dim;
  a.interleaved = r->interleaved;
  a.eps = r->eps;
  a.gain = r->gain;
  for (int i = 0; i < r->rot_dim / 2; ++i) a.freq[i] = r->freq[i] / kTurn;
  SERVE_HIP(ctx, salt::launch_rotate(a, v.bf16, v.n_cu, (hipStream_t)stream));
  return SALT_OK;
}

// ---- marks ------------------------------------------------------------------------------------
salt_status salt_kv_track(salt_ctx* ctx, salt_kv* kv) {
  SERVE_LIVE(ctx);
  const salt_status st = salt::kv_of(ctx, kv);
  if (st != SALT_OK) return st;
  if (kv->marks) return SALT_OK;
  const salt::CtxView v = salt::ctx_view(ctx);
  SERVE_HIP(ctx, hipSetDevice(v.device));
  const size_t bytes = (size_t)kv->cfg.n_layers * 2 * kv->scales;
  char* marks = nullptr;
  if (hipMalloc((void**)&marks, bytes) != hipSuccess) {
    (void)hipGetLastError();
    return ctx_fail(ctx, SALT_ERR_OUT_OF_MEMORY, "marks of %zu bytes do not fit", bytes);
  }
  hipError_t e = hipMemset(marks, 0, bytes);
  if (e == hipSuccess) e = hipDeviceSynchronize();
  if (e != hipSuccess) {
    (void)hipFree(marks);
    return salt::ctx_hip_fail(ctx, e, "marks init");
  }
  kv->marks = marks;
  return SALT_OK;
}

salt_status salt_kv_score(salt_ctx* ctx, salt_seqs* q, int32_t layer, const void* queries, int64_t ldq,
                          const int32_t* pos, float scale, int32_t window, void* stream) {
  salt_status st = marks_call(ctx, q, layer, true);
  if (st != SALT_OK) return st;
  if (!std::isfinite(scale) || !(scale > 0.f)) return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "scale must be finite and > 0");
  if (window < 0) return ctx_fail(ctx, SALT_ERR_OUT_OF_RANGE, "window = %d", window);
  if (q->T == 0) return SALT_OK;
  const salt_kv* kv = q->kv;
  const int64_t width = (int64_t)kv->cfg.n_heads * kv->cfg.head_dim;
  if ((st = salt::rows_arg(ctx, "q", queries, ldq, width)) != SALT_OK) return st;
  if (ldq > salt::kScoreRow)
    return ctx_fail(ctx, SALT_ERR_OUT_OF_RANGE, "q rows of %lld elements, at most %lld", (long long)ldq, (long long)salt::kScoreRow);
  if (reinterpret_cast<uintptr_t>(pos) & 3u) return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "misaligned positions");
  const int64_t blocks = salt::score_blocks(q->n_units, kv->cfg.n_kv_heads);
  if (blocks > salt::kMaxBlocks)
    return ctx_fail(ctx, SALT_ERR_OUT_OF_RANGE, "the batch takes a launch of %lld blocks, at most %lld", (long long)blocks,
                    (long long)salt::kMaxBlocks);
  const salt::CtxView cv = salt::ctx_view(ctx);
  SERVE_HIP(ctx, hipSetDevice(cv.device));
  const hipStream_t s = (hipStream_t)stream;
  if ((st = salt::enter(ctx, q, s)) != SALT_OK) return st;
  salt::ScoreArgs a{};
  a.att.kv = salt::layer_of(kv, layer);
  a.att.q = queries;
  a.att.ldq = ldq;
  a.att.pages = q->dev + q->at_page;
  a.att.order = q->dev + q->at_order;
  a.att.items = reinterpret_cast<const salt::AttItem*>(q->dev + q->at_item);
  a.att.joins = reinterpret_cast<const salt::AttJoin*>(q->dev + q->at_join);
  a.att.stat = q->stat;
  a.att.heads = kv->cfg.n_heads;
  a.att.group = kv->cfg.n_heads / kv->cfg.n_kv_heads;
  std::copy(q->n_kind, q->n_kind + 4, a.att.n_kind);
  a.att.n_joins = q->n_joins;
  a.att.scale = scale;
  a.b = view_of(q);
  a.back = q->dev + q->at_back;
  a.pos = pos;
  // (the attention's partial sums of v, which this call has no use for: 2 T heads rows of head_dim floats and more)
  a.fin = reinterpret_cast<float2*>(q->part);
  a.joined = q->dev + q->at_joined;
  a.window = window == 0 ? INT32_MAX : window;
  const int64_t group = a.att.group;
  a.few = std::min(q->min_q, a.window) * group <= salt::kFewRows;
  a.many = std::min(q->max_q, a.window) * group > salt::kFewRows;
  SERVE_HIP(ctx, salt::launch_score(a, cv.bf16, s));
  return SALT_OK;
}

salt_status salt_kv_evict(salt_ctx* ctx, salt_seqs* q, int32_t layer, int32_t keep, int32_t recent, void* stream) {
  salt_status st = marks_call(ctx, q, layer, true);
  if (st != SALT_OK) return st;
  if (keep < 0 || recent < 0 || recent > keep)
    return ctx_fail(ctx, SALT_ERR_OUT_OF_RANGE, "keep = %d, recent = %d: need 0 <= recent <= keep", keep, recent);
  if (q->max_len <= keep || keep == 0) return SALT_OK;     // (of no tokens to keep, none has to move)
  if (q->max_len > salt::kEvictLen)
    return ctx_fail(ctx, SALT_ERR_OUT_OF_RANGE, "a sequence of %d tokens, at most %d", q->max_len, salt::kEvictLen);
  const salt_kv* kv = q->kv;
  if ((int64_t)q->n_seqs * kv->cfg.n_kv_heads * 4 > salt::kMaxBlocks)   // (blocks of up to 1024 threads)
    return ctx_fail(ctx, SALT_ERR_OUT_OF_RANGE, "%d sequences of %d kv heads", q->n_seqs, kv->cfg.n_kv_heads);
  const salt::CtxView cv = salt::ctx_view(ctx);
  SERVE_HIP(ctx, hipSetDevice(cv.device));
  const hipStream_t s = (hipStream_t)stream;
  if ((st = salt::enter(ctx, q, s)) != SALT_OK) return st;
  salt::EvictArgs a{};
  a.kv = salt::layer_of(kv, layer);
  a.b = view_of(q);
  a.keep = keep;
  a.recent = recent;
  a.max_len = q->max_len;
  SERVE_HIP(ctx, salt::launch_evict(a, s));
  return SALT_OK;
}

salt_status salt_kv_read_marks(salt_ctx* ctx, salt_seqs* q, int32_t layer, float* weight, int32_t* pos, void* stream) {
  return marks_copy(ctx, q, layer, weight, pos, stream, false);
}

salt_status salt_kv_write_marks(salt_ctx* ctx, salt_seqs* q, int32_t layer, const float* weight, const int32_t* pos,
                                void* stream) {
  return marks_copy(ctx, q, layer, const_cast<float*>(weight), const_cast<int32_t*>(pos), stream, true);
}

// ---- copies of pages -----------------------------------------------------------------------------
salt_status salt_kv_copy(salt_ctx* ctx, salt_kv* kv, int32_t n, const int32_t* src, const int32_t* dst,
                         const int32_t* tokens, void* stream) {
  SERVE_LIVE(ctx);
  salt_status st = salt::kv_of(ctx, kv);
  if (st != SALT_OK) return st;
  if (n < 0 || (n > 0 && (!src || !dst))) return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "null argument");
  if (n > kv->cfg.n_pages) return ctx_fail(ctx, SALT_ERR_OUT_OF_RANGE, "%d copies of %d pages", n, kv->cfg.n_pages);
  const int pt = kv->cfg.page_tokens;
  for (int i = 0; i < n; ++i) {
    for (const int32_t p : {src[i], dst[i]})
      if (p < 0 || p >= kv->cfg.n_pages)
        return ctx_fail(ctx, SALT_ERR_OUT_OF_RANGE, "page %d not in [0, %d)", p, kv->cfg.n_pages);
    if (tokens && (tokens[i] < 0 || tokens[i] > pt))
      return ctx_fail(ctx, SALT_ERR_OUT_OF_RANGE, "%d tokens of a page of %d", tokens[i], pt);
  }
  const uint32_t now = salt::next_stamp(kv);
  for (int i = 0; i < n; ++i) {
    uint32_t& w = kv->stamp[(size_t)dst[i]];
    if (w == now) return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "page %d is written twice", dst[i]);
    w = now;
  }
  for (int i = 0; i < n; ++i)
    if (kv->stamp[(size_t)src[i]] == now)
      return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "page %d is read and written", src[i]);
  if (n == 0) return SALT_OK;
  const salt::CtxView cv = salt::ctx_view(ctx);
  SERVE_HIP(ctx, hipSetDevice(cv.device));
  const hipStream_t s = (hipStream_t)stream;
  if ((st = salt::enter_stream(ctx, kv->order, s)) != SALT_OK) return st;
  salt::CopyArgs a{};
  a.kv = salt::layer_of(kv, 0);
  a.layer = 2 * (kv->codes + kv->scales);
  a.mark_layer = 2 * kv->scales;
  a.n_layers = kv->cfg.n_layers;
  for (int first = 0; first < n; first += salt::kCopyPairs) {
    a.n = std::min(salt::kCopyPairs, n - first);
    for (int i = 0; i < a.n; ++i) {
      a.src[i] = src[first + i];
      a.dst[i] = dst[first + i];
      a.tokens[i] = (uint16_t)(tokens ? tokens[first + i] : pt);
    }
    SERVE_HIP(ctx, salt::launch_copy(a, s));
  }
  return SALT_OK;
}

// ---- beam search -----------------------------------------------------------------------------------
salt_status salt_beams_create(salt_ctx* ctx, int32_t max_rows, int32_t max_out, salt_beams** out) {
  SERVE_LIVE(ctx);
  if (!out) return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "null argument");
  *out = nullptr;
  if (max_rows < 1 || max_rows > salt::kMaxBeamRows || max_out < 1 || max_out > salt::kMaxOut)
    return ctx_fail(ctx, SALT_ERR_OUT_OF_RANGE, "max_rows in [1, %d], max_out in [1, %d]", salt::kMaxBeamRows, salt::kMaxOut);
  const salt::CtxView v = salt::ctx_view(ctx);
  SERVE_HIP(ctx, hipSetDevice(v.device));
  salt_beams* b = new (std::nothrow) salt_beams();
  if (!b) return ctx_fail(ctx, SALT_ERR_OUT_OF_MEMORY, "beams");
  b->max_rows = max_rows;
  b->max_out = max_out;
  b->pieces = salt::beam_pieces(max_rows, v.n_cu);
  b->entries = b->pieces * max_out;
  if (hipMalloc((void**)&b->best, (size_t)b->entries * sizeof(uint64_t)) != hipSuccess ||
      hipMalloc((void**)&b->stat, (size_t)b->pieces * sizeof(double2)) != hipSuccess) {
    (void)hipGetLastError();
    free_beams(b);
    return ctx_fail(ctx, SALT_ERR_OUT_OF_MEMORY, "buffers for %d beams", max_rows);
  }
  if (!salt::ctx_own(ctx, b, free_beams)) {
    free_beams(b);
    return ctx_fail(ctx, SALT_ERR_OUT_OF_MEMORY, "beams");
  }
  *out = b;
  return SALT_OK;
}

void salt_beams_destroy(salt_ctx* ctx, salt_beams* b) {
  if (!ctx || !b) return;
  const salt::CtxView v = salt::ctx_view(ctx);
  (void)hipSetDevice(v.device);
  if (!salt::ctx_disown(ctx, b)) return;
  (void)hipDeviceSynchronize();
  free_beams(b);
}

salt_status salt_beam_select(salt_ctx* ctx, salt_beams* b, int32_t n_reqs, int32_t width, int32_t vocab,
                             const void* logits, int64_t ld, const float* score, int32_t n_out, float* out_score,
                             int32_t* out_beam, int32_t* out_token, void* stream) {
  SERVE_LIVE(ctx);
  if (!b || !salt::ctx_owns(ctx, b)) return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "not beams of this context");
  if (n_reqs < 0 || width < 1 || width > salt::kMaxBeams || (int64_t)n_reqs * width > b->max_rows)
    return ctx_fail(ctx, SALT_ERR_OUT_OF_RANGE, "%d requests of %d beams: at most %d beams in all, %d to a request", n_reqs,
                    width, b->max_rows, salt::kMaxBeams);
  if (n_out < 1 || n_out > b->max_out) return ctx_fail(ctx, SALT_ERR_OUT_OF_RANGE, "n_out = %d not in [1, %d]", n_out, b->max_out);
  if (vocab < 1 || vocab > salt::kMaxVocab)
    return ctx_fail(ctx, SALT_ERR_OUT_OF_RANGE, "vocab = %d not in [1, %d]", vocab, salt::kMaxVocab);
  if (n_reqs == 0) return SALT_OK;
  salt_status st = salt::rows_arg(ctx, "logits", logits, ld, vocab);
  if (st != SALT_OK) return st;
  for (const void* p : {(const void*)score, (const void*)out_score, (const void*)out_beam, (const void*)out_token})
    if (!p || (reinterpret_cast<uintptr_t>(p) & 3u)) return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "null or misaligned array");
  const salt::CtxView v = salt::ctx_view(ctx);
  salt::BeamArgs a{};
  a.logits = logits;
  a.score = score;
  a.ld = ld;
  a.best = b->best;
  a.stat = b->stat;
  a.out_score = out_score;
  a.out_beam = out_beam;
  a.out_token = out_token;
  a.reqs = n_reqs;
  a.width = width;
  a.vocab = vocab;
  a.n_out = n_out;
  a.splits = salt::beam_splits((int64_t)n_reqs * width, vocab, v.n_cu);
  const int64_t pieces = (int64_t)n_reqs * width * a.splits;
  if (pieces > b->pieces || pieces * n_out > b->entries || pieces > salt::kMaxBlocks)
    return ctx_fail(ctx, SALT_ERR_OUT_OF_RANGE, "%lld pieces, at most %lld", (long long)pieces, (long long)b->pieces);
  SERVE_HIP(ctx, hipSetDevice(v.device));
  const hipStream_t s = (hipStream_t)stream;
  if ((st = salt::enter_stream(ctx, b->order, s)) != SALT_OK) return st;
  SERVE_HIP(ctx, salt::launch_beam(a, v.bf16, s));
  return SALT_OK;
}

}  // extern "C"
