// libsalt host runtime, the operators around the apply: base weights in 8 bits and
// their product, the paged KV cache, and attention over it (include/salt.h).
//
// Objects are owned by their context.  A batch of sequences is validated on the host, as
// a plan's maps are, so that no index from a caller reaches a kernel unchecked; its
// arrays then travel in one copy from a page-locked ring.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>
#include <vector>

#include "salt.h"
#include "salt_seqs.h"
#include "salt_serve.h"

namespace {

using salt::ctx_fail;

#define SERVE_LIVE(ctx)                                  \
  do {                                                   \
    const salt_status st_ = salt::ctx_live(ctx);         \
    if (st_ != SALT_OK) return st_;                      \
  } while (0)
#define SERVE_HIP(ctx, call)                                              \
  do {                                                                    \
    hipError_t e_ = (call);                                               \
    if (e_ != hipSuccess) return salt::ctx_hip_fail((ctx), e_, #call);    \
  } while (0)

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
size_t round_up(size_t v, size_t a) { return (v + a - 1) / a * a; }
int ceil_div(int a, int b) { return (a + b - 1) / b; }

bool is_capturing(hipStream_t s) {
  hipStreamCaptureStatus cap = hipStreamCaptureStatusNone;
  if (hipStreamIsCapturing(s, &cap) != hipSuccess) {
    (void)hipGetLastError();
    return false;
  }
  return cap == hipStreamCaptureStatusActive;
}

// Work on an object's buffers goes to `s`: behind what went to another stream before.
struct StreamOrder {
  hipEvent_t hop = nullptr;
  hipStream_t last = nullptr;
  bool used = false;
  hipError_t enter(hipStream_t s) {
    if (used && last != s) {
      hipError_t e = hipSuccess;
      if (!hop) e = hipEventCreateWithFlags(&hop, hipEventDisableTiming);
      if (e == hipSuccess) e = hipEventRecord(hop, last);
      if (e == hipSuccess) e = hipStreamWaitEvent(s, hop, 0);
      if (e != hipSuccess) return e;
    }
    used = true;
    last = s;
    return hipSuccess;
  }
  // Work under capture cannot be ordered against work outside it.
  bool refuses(hipStream_t s) const { return used && last != s && (is_capturing(s) || is_capturing(last)); }
  void destroy() {
    if (hop) (void)hipEventDestroy(hop);
    hop = nullptr;
  }
};
salt_status enter_stream(salt_ctx* ctx, StreamOrder& o, hipStream_t s) {
  if (o.refuses(s))
    return ctx_fail(ctx, SALT_ERR_BAD_STATE, "work under capture on another stream than the object's last work");
  SERVE_HIP(ctx, o.enter(s));
  return SALT_OK;
}

// The base weights of a context: per table codes and scales, and the scratch that the
// products quantise x into.
struct Base {
  struct Table {
    uint8_t* w = nullptr;
    float* sw = nullptr;
    bool pinned = false;
  };
  std::vector<Table> tab;
  uint8_t* xq = nullptr;
  float* sx = nullptr;
  int t_pad = 0, kb_max = 0;
  StreamOrder order;
};

void free_base(void* p) {
  Base* b = static_cast<Base*>(p);
  for (Base::Table& t : b->tab) {
    if (t.w) (void)hipFree(t.w);
    if (t.sw) (void)hipFree(t.sw);
  }
  if (b->xq) (void)hipFree(b->xq);
  if (b->sx) (void)hipFree(b->sx);
  b->order.destroy();
  delete b;
}

// Codes are addressed with 32-bit offsets inside a table and inside x.
constexpr int64_t kMaxCodes = (int64_t)1 << 31;

salt::BaseTable base_table(const Base::Table& t, const salt_shape& sh) {
  salt::BaseTable b{};
  b.w = t.w;
  b.sw = t.sw;
  b.out = sh.out_dim;
  b.n_blk = (int)(round_up((size_t)sh.out_dim, salt::kBasePad) / salt::kBaseBlock);
  return b;
}

// The context's base object and `table`'s buffers in it, made when they are first needed.
salt_status base_for(salt_ctx* ctx, int32_t table, const salt::CtxView& v, Base** out) {
  Base* b = static_cast<Base*>(salt::ctx_base(ctx));
  SERVE_HIP(ctx, hipSetDevice(v.device));
  if (!b) {
    b = new (std::nothrow) Base();
    if (!b) return ctx_fail(ctx, SALT_ERR_OUT_OF_MEMORY, "base weights");
    try {
      b->tab.resize((size_t)v.n_tables);
    } catch (const std::bad_alloc&) {
      free_base(b);
      return ctx_fail(ctx, SALT_ERR_OUT_OF_MEMORY, "base weights");
    }
    int in = 0;
    for (int t = 0; t < v.n_tables; ++t) in = std::max(in, v.tables[t].in_dim);
    b->kb_max = ceil_div(in, salt::kBaseBlock);
    b->t_pad = (int)round_up((size_t)v.max_tokens, salt::kBasePad);
    if ((int64_t)b->t_pad * b->kb_max * salt::kBaseBlock > kMaxCodes) {
      const int64_t need = (int64_t)b->t_pad * b->kb_max * salt::kBaseBlock;
      free_base(b);
      return ctx_fail(ctx, SALT_ERR_OUT_OF_RANGE, "x of max_tokens x the widest table has %lld codes, at most %lld",
                      (long long)need, (long long)kMaxCodes);
    }
    if (hipMalloc((void**)&b->xq, (size_t)b->t_pad * b->kb_max * salt::kBaseBlock) != hipSuccess ||
        hipMalloc((void**)&b->sx, sizeof(float) * b->t_pad * b->kb_max) != hipSuccess) {
      (void)hipGetLastError();
      free_base(b);
      return ctx_fail(ctx, SALT_ERR_OUT_OF_MEMORY, "scratch of the base products");
    }
    if (!salt::ctx_own(ctx, b, free_base)) {
      free_base(b);
      return ctx_fail(ctx, SALT_ERR_OUT_OF_MEMORY, "base weights");
    }
    salt::ctx_base(ctx) = b;
  }
  Base::Table& t = b->tab[(size_t)table];
  if (!t.w) {
    const salt_shape sh = v.tables[table];
    const size_t out_pad = round_up((size_t)sh.out_dim, salt::kBasePad);
    const size_t kb = (size_t)ceil_div(sh.in_dim, salt::kBaseBlock);
    if ((int64_t)(out_pad * kb * salt::kBaseBlock) > kMaxCodes)
      return ctx_fail(ctx, SALT_ERR_OUT_OF_RANGE, "table %d has %zu codes, at most %lld", table,
                      out_pad * kb * salt::kBaseBlock, (long long)kMaxCodes);
    uint8_t* w = nullptr;
    float* sw = nullptr;
    if (hipMalloc((void**)&w, out_pad * kb * salt::kBaseBlock) != hipSuccess ||
        hipMalloc((void**)&sw, sizeof(float) * (out_pad / salt::kBaseBlock) * kb) != hipSuccess) {
      (void)hipGetLastError();
      if (w) (void)hipFree(w);
      return ctx_fail(ctx, SALT_ERR_OUT_OF_MEMORY, "base weight of table %d", table);
    }
    t.w = w;
    t.sw = sw;
  }
  *out = b;
  return SALT_OK;
}

salt_status pin_args(salt_ctx* ctx, int32_t table, const void* w, int64_t ld, int64_t least, const salt::CtxView& v) {
  if (table < 0 || table >= v.n_tables)
    return ctx_fail(ctx, SALT_ERR_OUT_OF_RANGE, "table %d not in [0, %d)", table, v.n_tables);
  if (!w || !aligned16(w)) return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "null or misaligned weight");
  if (ld < least || ld % 8 != 0)
    return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "row length %lld: need a multiple of 8 and >= %lld", (long long)ld,
                    (long long)least);
  return SALT_OK;
}
// A table's first pin allocates, which a capture forbids, and makes its weight ready for calls that are not
// recorded: it cannot be recorded itself.
salt_status pin_capture(salt_ctx* ctx, int32_t table, hipStream_t s) {
  const Base* b = static_cast<const Base*>(salt::ctx_base(ctx));
  if (!(b && b->tab[(size_t)table].pinned) && is_capturing(s))
    return ctx_fail(ctx, SALT_ERR_BAD_STATE, "the first pin of table %d on a stream under capture", table);
  return SALT_OK;
}

}  // namespace

// ---- KV cache objects --------------------------------------------------------------------
struct salt_kv {
  salt_kv_config cfg{};
  int log2_page = 0;
  char* pool = nullptr;
  size_t codes = 0, scales = 0;       // bytes of one layer's k (or v) codes, and scales
  std::vector<salt_seqs*> seqs;
  std::vector<uint32_t> stamp;        // per page: the salt_seqs_set that last saw it written
  uint32_t stamps = 0;
  StreamOrder order;                  // writes and reads of the pool
};

struct salt_seqs {
  salt_kv* kv = nullptr;
  int max_seqs = 0, max_tokens = 0, max_pages = 0;
  size_t words = 0;                   // 32-bit words of one staging buffer
  int32_t* dev = nullptr;
  int32_t* staging = nullptr;         // two page-locked buffers
  int stage = 0;
  hipEvent_t staged[2] = {};
  bool pending[2] = {};
  float *part = nullptr, *stat = nullptr;
  int64_t part_rows = 0;
  StreamOrder order;
  // the batch
  int T = -1;                         // -1: none was set
  int n_refs = 0, n_own_refs = 0;
  int64_t own_tokens = 0;
  bool clash = false;                 // two of its tokens' pages are one page
  bool recorded = false;              // a graph holds its launches: grid sizes and places in `dev`
  size_t at_page = 0, at_row = 0, at_count = 0, at_slot = 0, at_order = 0, at_item = 0, at_join = 0;
  int n_kind[4] = {0, 0, 0, 0}, n_joins = 0;
};

namespace {

void free_seqs(salt_seqs* q) {
  if (q->dev) (void)hipFree(q->dev);
  if (q->part) (void)hipFree(q->part);
  if (q->stat) (void)hipFree(q->stat);
  if (q->staging) (void)hipHostFree(q->staging);
  for (hipEvent_t e : q->staged)
    if (e) (void)hipEventDestroy(e);
  q->order.destroy();
  delete q;
}
void free_kv(void* p) {
  salt_kv* kv = static_cast<salt_kv*>(p);
  for (salt_seqs* q : kv->seqs) free_seqs(q);
  if (kv->pool) (void)hipFree(kv->pool);
  kv->order.destroy();
  delete kv;
}

const char* kv_config_error(const salt_kv_config& c) {
  if (c.flags != 0) return "flags must be 0";
  if (c.format != SALT_KV_E4M3 && c.format != SALT_KV_INT8) return "unknown format";
  if (c.head_dim != 64 && c.head_dim != 128 && c.head_dim != 256) return "head_dim must be 64, 128 or 256";
  if (c.page_tokens < 16 || c.page_tokens > 256 || (c.page_tokens & (c.page_tokens - 1)))
    return "page_tokens must be a power of two in [16, 256]";
  if (c.n_layers < 1 || c.n_layers > 1024) return "n_layers not in [1, 1024]";
  if (c.n_pages < 1 || c.n_pages > (1 << 23)) return "n_pages not in [1, 2^23]";
  if (c.n_kv_heads < 1 || c.n_kv_heads > 256) return "n_kv_heads not in [1, 256]";
  if (c.n_heads < c.n_kv_heads || c.n_heads % c.n_kv_heads != 0 || c.n_heads / c.n_kv_heads > salt::kMaxGroup)
    return "n_heads must be 1 to 64 times n_kv_heads";
  return nullptr;
}
// Bytes of one layer's k (or v) codes and of its scales.
void kv_sizes(const salt_kv_config& c, size_t* codes, size_t* scales) {
  const size_t vecs = (size_t)c.n_pages * c.n_kv_heads * c.page_tokens;
  *codes = round_up(vecs * (size_t)c.head_dim, 256);
  *scales = round_up(vecs * sizeof(float), 256);
}

// Whether `kv` is a live cache of `ctx` (asked before anything of it is read).
salt_status kv_of(salt_ctx* ctx, const salt_kv* kv) {
  if (!kv || !salt::ctx_owns(ctx, kv)) return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "not a cache of this context");
  return SALT_OK;
}
salt_status seqs_of(salt_ctx* ctx, const salt_seqs* q) {
  if (!q) return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "null sequences");
  return kv_of(ctx, q->kv);
}

salt::KvLayer layer_of(const salt_kv* kv, int layer) {
  salt::KvLayer l{};
  char* p = kv->pool + (size_t)layer * 2 * (kv->codes + kv->scales);
  l.k = reinterpret_cast<uint8_t*>(p);
  l.v = reinterpret_cast<uint8_t*>(p + kv->codes);
  l.ks = reinterpret_cast<float*>(p + 2 * kv->codes);
  l.vs = reinterpret_cast<float*>(p + 2 * kv->codes + kv->scales);
  l.kv_heads = kv->cfg.n_kv_heads;
  l.dim = kv->cfg.head_dim;
  l.log2_page = kv->log2_page;
  l.format = kv->cfg.format;
  return l;
}

// Common checks of the calls on a set batch.
salt_status batch_call(salt_ctx* ctx, salt_seqs* q, int32_t layer) {
  SERVE_LIVE(ctx);
  const salt_status st = seqs_of(ctx, q);
  if (st != SALT_OK) return st;
  if (q->T < 0) return ctx_fail(ctx, SALT_ERR_BAD_STATE, "no batch was set on the sequences");
  if (layer < 0 || layer >= q->kv->cfg.n_layers)
    return ctx_fail(ctx, SALT_ERR_OUT_OF_RANGE, "layer %d not in [0, %d)", layer, q->kv->cfg.n_layers);
  return SALT_OK;
}
// A row-major operand of whole heads: rows `ld` elements apart (0: dense).
salt_status rows_arg(salt_ctx* ctx, const char* what, const void* p, int64_t& ld, int64_t width) {
  if (ld == 0) ld = width;
  if (!p || !aligned16(p)) return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "null or misaligned %s", what);
  if (ld < width || ld % 8 != 0)
    return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "%s rows of %lld elements: need a multiple of 8 and >= %lld", what,
                    (long long)ld, (long long)width);
  return SALT_OK;
}
// The batch's buffers and the pool, on `s`.
salt_status enter(salt_ctx* ctx, salt_seqs* q, hipStream_t s) {
  if (q->kv->order.refuses(s))
    return ctx_fail(ctx, SALT_ERR_BAD_STATE, "work under capture on another stream than the cache's last work");
  salt_status st = enter_stream(ctx, q->order, s);
  if (st == SALT_OK) st = enter_stream(ctx, q->kv->order, s);
  if (st == SALT_OK && is_capturing(s)) q->recorded = true;
  return st;
}

}  // namespace

extern "C" {

// ---- base weights ---------------------------------------------------------------------------
salt_status salt_pin_base(salt_ctx* ctx, int32_t table, const void* w, int64_t ldw, void* stream) {
  SERVE_LIVE(ctx);
  const salt::CtxView v = salt::ctx_view(ctx);
  salt_status st = pin_args(ctx, table, w, ldw, table >= 0 && table < v.n_tables ? v.tables[table].out_dim : 0, v);
  const hipStream_t s = (hipStream_t)stream;
  if (st == SALT_OK) st = pin_capture(ctx, table, s);
  Base* b = nullptr;
  if (st == SALT_OK) st = base_for(ctx, table, v, &b);
  if (st != SALT_OK) return st;
  if ((st = enter_stream(ctx, b->order, s)) != SALT_OK) return st;
  salt::BasePinArgs a{};
  a.w = const_cast<void*>(w);
  a.ld = ldw;
  a.tab = base_table(b->tab[(size_t)table], v.tables[table]);
  a.in = v.tables[table].in_dim;
  a.kb = ceil_div(a.in, salt::kBaseBlock);
  SERVE_HIP(ctx, salt::launch_base_pin(a, v.bf16, s));
  b->tab[(size_t)table].pinned = true;
  return SALT_OK;
}

salt_status salt_pin_base_fp8(salt_ctx* ctx, int32_t table, const void* wq, int64_t ldq, const float* scales,
                              void* stream) {
  SERVE_LIVE(ctx);
  const salt::CtxView v = salt::ctx_view(ctx);
  salt_status st = pin_args(ctx, table, wq, ldq, table >= 0 && table < v.n_tables ? v.tables[table].in_dim : 0, v);
  if (st != SALT_OK) return st;
  if (!scales || (reinterpret_cast<uintptr_t>(scales) & 3u))
    return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "null or misaligned scales");
  const hipStream_t s = (hipStream_t)stream;
  st = pin_capture(ctx, table, s);
  Base* b = nullptr;
  if (st == SALT_OK) st = base_for(ctx, table, v, &b);
  if (st != SALT_OK) return st;
  if ((st = enter_stream(ctx, b->order, s)) != SALT_OK) return st;
  salt::BasePinArgs a{};
  a.q = static_cast<const uint8_t*>(wq);
  a.sq = scales;
  a.ld = ldq;
  a.tab = base_table(b->tab[(size_t)table], v.tables[table]);
  a.in = v.tables[table].in_dim;
  a.kb = ceil_div(a.in, salt::kBaseBlock);
  SERVE_HIP(ctx, salt::launch_base_pin_codes(a, s));
  b->tab[(size_t)table].pinned = true;
  return SALT_OK;
}

salt_status salt_read_base(salt_ctx* ctx, int32_t table, void* w, int64_t ldw, void* stream) {
  SERVE_LIVE(ctx);
  const salt::CtxView v = salt::ctx_view(ctx);
  salt_status st = pin_args(ctx, table, w, ldw, table >= 0 && table < v.n_tables ? v.tables[table].out_dim : 0, v);
  if (st != SALT_OK) return st;
  Base* b = static_cast<Base*>(salt::ctx_base(ctx));
  if (!b || !b->tab[(size_t)table].pinned)
    return ctx_fail(ctx, SALT_ERR_BAD_STATE, "the base weight of table %d was never pinned", table);
  SERVE_HIP(ctx, hipSetDevice(v.device));
  const hipStream_t s = (hipStream_t)stream;
  if ((st = enter_stream(ctx, b->order, s)) != SALT_OK) return st;
  salt::BasePinArgs a{};
  a.w = w;
  a.ld = ldw;
  a.tab = base_table(b->tab[(size_t)table], v.tables[table]);
  a.in = v.tables[table].in_dim;
  a.kb = ceil_div(a.in, salt::kBaseBlock);
  SERVE_HIP(ctx, salt::launch_base_read(a, v.bf16, s));
  return SALT_OK;
}

salt_status salt_base_product(salt_ctx* ctx, int32_t n, const int32_t* tables, int32_t T, const void* x,
                              void* const* ys, void* stream) {
  SERVE_LIVE(ctx);
  const salt::CtxView v = salt::ctx_view(ctx);
  salt_status st;
  if (n < 0 || (n > 0 && (!tables || !ys))) return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "null argument");
  if (T < 0 || T > v.max_tokens)
    return ctx_fail(ctx, SALT_ERR_OUT_OF_RANGE, "T = %d not in [0, %d]", T, v.max_tokens);
  Base* b = static_cast<Base*>(salt::ctx_base(ctx));
  for (int i = 0; i < n; ++i) {
    const int t = tables[i];
    if (t < 0 || t >= v.n_tables)
      return ctx_fail(ctx, SALT_ERR_OUT_OF_RANGE, "table %d not in [0, %d)", t, v.n_tables);
    if (!b || !b->tab[(size_t)t].pinned)
      return ctx_fail(ctx, SALT_ERR_BAD_STATE, "the base weight of table %d was never pinned", t);
    if (v.tables[t].in_dim != v.tables[tables[0]].in_dim)
      return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "tables %d and %d read one x but have %d and %d inputs", tables[0], t,
                      v.tables[tables[0]].in_dim, v.tables[t].in_dim);
    if (T > 0 && (!ys[i] || !aligned16(ys[i])))
      return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "null or misaligned y of table %d", t);
  }
  if (n == 0 || T == 0) return SALT_OK;
  if (!x || !aligned16(x)) return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "null or misaligned x");
  SERVE_HIP(ctx, hipSetDevice(v.device));
  const hipStream_t s = (hipStream_t)stream;
  if ((st = enter_stream(ctx, b->order, s)) != SALT_OK) return st;
  salt::BaseArgs a{};
  a.x = x;
  a.xq = b->xq;
  a.sx = b->sx;
  a.T = T;
  a.T_pad = (int)round_up((size_t)T, salt::kBasePad);
  a.in = v.tables[tables[0]].in_dim;
  a.kb = ceil_div(a.in, salt::kBaseBlock);
  for (int first = 0; first < n; first += salt::kBaseTables) {
    a.n_tables = std::min(salt::kBaseTables, n - first);
    for (int i = 0; i < a.n_tables; ++i) {
      a.tab[i] = base_table(b->tab[(size_t)tables[first + i]], v.tables[tables[first + i]]);
      a.tab[i].y = ys[first + i];
    }
    SERVE_HIP(ctx, salt::launch_base_product(a, v.bf16, v.n_cu, s));
  }
  return SALT_OK;
}

// ---- KV cache ---------------------------------------------------------------------------------
size_t salt_kv_bytes(const salt_kv_config* cfg) {
  if (!cfg || kv_config_error(*cfg)) return 0;
  size_t codes, scales;
  kv_sizes(*cfg, &codes, &scales);
  return (size_t)cfg->n_layers * 2 * (codes + scales);
}

salt_status salt_kv_create(salt_ctx* ctx, const salt_kv_config* cfg, salt_kv** out) {
  SERVE_LIVE(ctx);
  if (!out) return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "null argument");
  *out = nullptr;
  if (!cfg) return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "null argument");
  if (const char* why = kv_config_error(*cfg)) return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "cache: %s", why);
  const salt::CtxView v = salt::ctx_view(ctx);
  SERVE_HIP(ctx, hipSetDevice(v.device));
  salt_kv* kv = new (std::nothrow) salt_kv();
  if (!kv) return ctx_fail(ctx, SALT_ERR_OUT_OF_MEMORY, "cache");
  kv->cfg = *cfg;
  while ((1 << kv->log2_page) < cfg->page_tokens) ++kv->log2_page;
  kv_sizes(*cfg, &kv->codes, &kv->scales);
  const size_t bytes = salt_kv_bytes(cfg);
  try {
    kv->stamp.assign((size_t)cfg->n_pages, 0);
  } catch (const std::bad_alloc&) {
    free_kv(kv);
    return ctx_fail(ctx, SALT_ERR_OUT_OF_MEMORY, "cache");
  }
  if (hipMalloc((void**)&kv->pool, bytes) != hipSuccess) {
    (void)hipGetLastError();
    kv->pool = nullptr;
    free_kv(kv);
    return ctx_fail(ctx, SALT_ERR_OUT_OF_MEMORY, "cache of %zu bytes does not fit", bytes);
  }
  hipError_t e = hipMemset(kv->pool, 0, bytes);
  if (e == hipSuccess) e = hipDeviceSynchronize();
  if (e != hipSuccess) {
    free_kv(kv);
    return salt::ctx_hip_fail(ctx, e, "cache init");
  }
  if (!salt::ctx_own(ctx, kv, free_kv)) {
    free_kv(kv);
    return ctx_fail(ctx, SALT_ERR_OUT_OF_MEMORY, "cache");
  }
  *out = kv;
  return SALT_OK;
}

void salt_kv_destroy(salt_ctx* ctx, salt_kv* kv) {
  if (!ctx || !kv) return;
  const salt::CtxView v = salt::ctx_view(ctx);
  (void)hipSetDevice(v.device);
  if (!salt::ctx_disown(ctx, kv)) return;
  (void)hipDeviceSynchronize();
  free_kv(kv);
}

salt_status salt_seqs_create(salt_ctx* ctx, salt_kv* kv, int32_t max_seqs, int32_t max_tokens, int32_t max_pages,
                             salt_seqs** out) {
  SERVE_LIVE(ctx);
  if (!out) return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "null argument");
  *out = nullptr;
  const salt_status st = kv_of(ctx, kv);
  if (st != SALT_OK) return st;
  if (max_seqs < 1 || max_seqs > (1 << 20) || max_tokens < 1 || max_tokens > (1 << 20) || max_pages < 1 ||
      max_pages > (1 << 24))
    return ctx_fail(ctx, SALT_ERR_OUT_OF_RANGE, "max_seqs, max_tokens in [1, 2^20], max_pages in [1, 2^24]");
  const salt::CtxView v = salt::ctx_view(ctx);
  SERVE_HIP(ctx, hipSetDevice(v.device));
  salt_seqs* q = new (std::nothrow) salt_seqs();
  if (!q) return ctx_fail(ctx, SALT_ERR_OUT_OF_MEMORY, "sequences");
  q->kv = kv;
  q->max_seqs = max_seqs;
  q->max_tokens = max_tokens;
  q->max_pages = max_pages;
  const size_t T = (size_t)max_tokens;
  const size_t items = (size_t)salt::attend_max_items(max_tokens, kv->cfg.n_heads);
  // (each of the six arrays behind the first starts at a multiple of 16 words)
  q->words = 3 * (size_t)max_pages + 3 * T + 6 * 16 + items * (sizeof(salt::AttItem) / 4) + T * (sizeof(salt::AttJoin) / 4);
  q->part_rows = (int64_t)(2 * T * (size_t)kv->cfg.n_heads) + salt::kExtraRows;
  if (q->part_rows > INT32_MAX) {
    free_seqs(q);
    return ctx_fail(ctx, SALT_ERR_OUT_OF_RANGE, "%d new tokens of %d heads have too many rows", max_tokens, kv->cfg.n_heads);
  }
  if (hipMalloc((void**)&q->dev, q->words * 4) != hipSuccess ||
      hipMalloc((void**)&q->part, (size_t)q->part_rows * kv->cfg.head_dim * sizeof(float)) != hipSuccess ||
      hipMalloc((void**)&q->stat, (size_t)q->part_rows * 2 * sizeof(float)) != hipSuccess ||
      hipHostMalloc((void**)&q->staging, 2 * q->words * 4, hipHostMallocDefault) != hipSuccess ||
      hipEventCreateWithFlags(&q->staged[0], hipEventDisableTiming) != hipSuccess ||
      hipEventCreateWithFlags(&q->staged[1], hipEventDisableTiming) != hipSuccess) {
    (void)hipGetLastError();
    free_seqs(q);
    return ctx_fail(ctx, SALT_ERR_OUT_OF_MEMORY, "buffers for %d sequences of %d new tokens", max_seqs, max_tokens);
  }
  try {
    kv->seqs.push_back(q);
  } catch (const std::bad_alloc&) {
    free_seqs(q);
    return ctx_fail(ctx, SALT_ERR_OUT_OF_MEMORY, "sequences");
  }
  *out = q;
  return SALT_OK;
}

void salt_seqs_destroy(salt_ctx* ctx, salt_seqs* q) {
  if (!ctx || !q) return;
  const salt::CtxView v = salt::ctx_view(ctx);
  (void)hipSetDevice(v.device);
  std::vector<salt_seqs*>& all = q->kv->seqs;
  const auto it = std::find(all.begin(), all.end(), q);
  if (it == all.end()) return;
  all.erase(it);
  (void)hipDeviceSynchronize();
  free_seqs(q);
}

salt_status salt_seqs_set(salt_ctx* ctx, salt_seqs* q, const salt_seq_batch* b, void* stream) {
  SERVE_LIVE(ctx);
  salt_status st = seqs_of(ctx, q);
  if (st != SALT_OK) return st;
  if (!b) return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "null argument");
  // (replays would read another batch's arrays in the places of this one's)
  if (q->recorded) return ctx_fail(ctx, SALT_ERR_BAD_STATE, "the batch was recorded into a graph, which keeps it");
  const int n = b->n_seqs, nd = b->n_domains;
  if (n < 0 || nd < 0 || (int64_t)n + nd > q->max_seqs)
    return ctx_fail(ctx, SALT_ERR_OUT_OF_RANGE, "%d sequences and %d domains, at most %d", n, nd, q->max_seqs);
  if ((n > 0 && (!b->q_len || !b->len || !b->page_off)) || (nd > 0 && (!b->prefix_len || !b->prefix_off)))
    return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "null array");
  salt_kv* kv = q->kv;
  const int pt = kv->cfg.page_tokens;
  // page references of one kind of holder: offsets from 0 on, enough pages for the tokens
  auto refs = [&](const char* what, int count, const int32_t* off, const int32_t* len, const int32_t* pages) {
    if (count > 0 && off[0] != 0) return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "%s: page offsets start at 0", what);
    for (int i = 0; i < count; ++i) {
      if (len[i] < 0 || len[i] > (1 << 28))
        return ctx_fail(ctx, SALT_ERR_OUT_OF_RANGE, "%s %d has length %d", what, i, len[i]);
      const int64_t has = (int64_t)off[i + 1] - off[i];
      if (has < 0 || off[i + 1] > q->max_pages)
        return ctx_fail(ctx, SALT_ERR_OUT_OF_RANGE, "%s %d: page offset %d", what, i, off[i + 1]);
      if (has < ceil_div(len[i], pt))
        return ctx_fail(ctx, SALT_ERR_OUT_OF_RANGE, "%s %d: %lld pages of %d for %d tokens", what, i, (long long)has, pt,
                        len[i]);
    }
    const int total = count > 0 ? off[count] : 0;
    if (total > 0 && !pages) return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "null pages");
    for (int i = 0; i < total; ++i)
      if (pages[i] < 0 || pages[i] >= kv->cfg.n_pages)
        return ctx_fail(ctx, SALT_ERR_OUT_OF_RANGE, "%s: page %d not in [0, %d)", what, pages[i], kv->cfg.n_pages);
    return SALT_OK;
  };
  st = refs("domain", nd, b->prefix_off, b->prefix_len, b->prefix_pages);
  if (st != SALT_OK) return st;
  st = refs("sequence", n, b->page_off, b->len, b->pages);
  if (st != SALT_OK) return st;
  const int pre_refs = nd > 0 ? b->prefix_off[nd] : 0, own_refs = n > 0 ? b->page_off[n] : 0;
  if ((int64_t)pre_refs + own_refs > q->max_pages)
    return ctx_fail(ctx, SALT_ERR_OUT_OF_RANGE, "%d + %d page references, at most %d", pre_refs, own_refs, q->max_pages);
  int64_t T64 = 0, own = 0;
  for (int i = 0; i < n; ++i) {
    if (b->q_len[i] < 0) return ctx_fail(ctx, SALT_ERR_OUT_OF_RANGE, "sequence %d has %d new tokens", i, b->q_len[i]);
    if (b->domain && (b->domain[i] < -1 || b->domain[i] >= nd))
      return ctx_fail(ctx, SALT_ERR_OUT_OF_RANGE, "domain %d of sequence %d not in [-1, %d)", b->domain[i], i, nd);
    T64 += b->q_len[i];
    own += b->len[i];
  }
  if (T64 > q->max_tokens)
    return ctx_fail(ctx, SALT_ERR_OUT_OF_RANGE, "%lld new tokens, at most %d", (long long)T64, q->max_tokens);
  if (own > INT32_MAX) return ctx_fail(ctx, SALT_ERR_OUT_OF_RANGE, "%lld tokens in the sequences", (long long)own);
  const hipStream_t s = (hipStream_t)stream;
  const salt::CtxView v = salt::ctx_view(ctx);
  SERVE_HIP(ctx, hipSetDevice(v.device));
  if (is_capturing(s) || (q->order.used && is_capturing(q->order.last)))
    return ctx_fail(ctx, SALT_ERR_BAD_STATE, "a batch of sequences cannot be set under capture");
  const int T = (int)T64;
  try {
    salt::AttWork w;
    std::vector<int32_t> off((size_t)n + 1);
    for (int i = 0; i <= n; ++i) off[(size_t)i] = n > 0 ? pre_refs + b->page_off[i] : 0;
    const salt::SeqBatch sb{n, nd, b->q_len, b->len, off.data(), b->domain, b->prefix_len, b->prefix_off};
    salt::cut_attention(sb, T, kv->cfg.n_heads, kv->cfg.n_kv_heads,
                        salt::attend_rows(v.bf16 ? 2 : 4, kv->cfg.head_dim), v.n_cu, w);
    const int64_t blocks = salt::most_blocks(w, T, kv->cfg.n_heads, kv->cfg.n_kv_heads, own_refs);
    if (blocks > salt::kMaxBlocks)
      return ctx_fail(ctx, SALT_ERR_OUT_OF_RANGE, "the batch takes launches of %lld blocks, at most %lld",
                      (long long)blocks, (long long)salt::kMaxBlocks);
    const int n_refs = pre_refs + own_refs;
    auto words = [](size_t k) { return round_up(k, 16); };
    const size_t at_page = 0, at_row = words((size_t)n_refs), at_count = at_row + words((size_t)own_refs);
    const size_t at_slot = at_count + words((size_t)own_refs), at_order = at_slot + words((size_t)T);
    const size_t at_item = at_order + words(w.order.size());
    const size_t at_join = at_item + words(w.items.size() * (sizeof(salt::AttItem) / 4));
    const size_t total = at_join + w.joins.size() * (sizeof(salt::AttJoin) / 4);
    if (total > q->words || w.rows > q->part_rows)
      return ctx_fail(ctx, SALT_ERR_BAD_STATE, "%zu words and %lld partial rows exceed the sequences' %zu and %lld",
                      total, (long long)w.rows, q->words, (long long)q->part_rows);
    const int stage = q->stage ^ 1;
    if (q->pending[stage]) {
      SERVE_HIP(ctx, hipEventSynchronize(q->staged[stage]));
      q->pending[stage] = false;
    }
    int32_t* d = q->staging + (size_t)stage * q->words;
    if (pre_refs) std::memcpy(d + at_page, b->prefix_pages, (size_t)pre_refs * 4);
    if (own_refs) std::memcpy(d + at_page + pre_refs, b->pages, (size_t)own_refs * 4);
    // two tokens of the batch written into one page from two sequences would race
    bool clash = false;
    if (++kv->stamps == 0) {
      std::fill(kv->stamp.begin(), kv->stamp.end(), 0u);
      kv->stamps = 1;
    }
    int t = 0, row = 0;
    for (int i = 0; i < n; ++i) {
      const int len = b->len[i], first = len - b->q_len[i];
      const int32_t* pages = b->pages + b->page_off[i];
      for (int j = 0; j < b->q_len[i]; ++j, ++t) {
        const int pos = first + j;
        d[at_slot + t] = pos < 0 ? -1 : pages[pos / pt] * pt + pos % pt;
        if (pos >= 0 && (pos % pt == 0 || pos == std::max(first, 0))) {
          uint32_t& st_ = kv->stamp[(size_t)pages[pos / pt]];
          clash |= st_ == kv->stamps;
          st_ = kv->stamps;
        }
      }
      for (int r = b->page_off[i]; r < b->page_off[i + 1]; ++r) {
        const int k = r - b->page_off[i];
        d[at_row + r] = salt::page_row(row, len, pt, k);
        d[at_count + r] = salt::page_count(len, pt, k);
      }
      row += len;
    }
    std::memcpy(d + at_order, w.order.data(), w.order.size() * 4);
    if (!w.items.empty()) std::memcpy(d + at_item, w.items.data(), w.items.size() * sizeof(salt::AttItem));
    if (!w.joins.empty()) std::memcpy(d + at_join, w.joins.data(), w.joins.size() * sizeof(salt::AttJoin));
    if ((st = enter_stream(ctx, q->order, s)) != SALT_OK) return st;
    if (total > 0) {
      SERVE_HIP(ctx, hipMemcpyAsync(q->dev, d, total * 4, hipMemcpyHostToDevice, s));
      SERVE_HIP(ctx, hipEventRecord(q->staged[stage], s));
      q->pending[stage] = true;
    }
    q->stage = stage;
    q->T = T;
    q->n_refs = n_refs;
    q->n_own_refs = own_refs;
    q->own_tokens = own;
    q->clash = clash;
    q->at_page = at_page;
    q->at_row = at_row;
    q->at_count = at_count;
    q->at_slot = at_slot;
    q->at_order = at_order;
    q->at_item = at_item;
    q->at_join = at_join;
    std::copy(w.n_kind, w.n_kind + 4, q->n_kind);
    q->n_joins = (int)w.joins.size();
  } catch (const std::bad_alloc&) {
    return ctx_fail(ctx, SALT_ERR_OUT_OF_MEMORY, "cutting the batch");
  }
  return SALT_OK;
}

salt_status salt_kv_write(salt_ctx* ctx, salt_seqs* q, int32_t layer, const void* k, int64_t ldk, const void* v,
                          int64_t ldv, void* stream) {
  salt_status st = batch_call(ctx, q, layer);
  if (st != SALT_OK) return st;
  if (q->clash) return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "two sequences of the batch write into one page");
  if (q->T == 0) return SALT_OK;
  const salt_kv* kv = q->kv;
  const int64_t width = (int64_t)kv->cfg.n_kv_heads * kv->cfg.head_dim;
  if ((st = rows_arg(ctx, "k", k, ldk, width)) != SALT_OK || (st = rows_arg(ctx, "v", v, ldv, width)) != SALT_OK)
    return st;
  const salt::CtxView cv = salt::ctx_view(ctx);
  SERVE_HIP(ctx, hipSetDevice(cv.device));
  const hipStream_t s = (hipStream_t)stream;
  if ((st = enter(ctx, q, s)) != SALT_OK) return st;
  salt::KvWriteArgs a{};
  a.kv = layer_of(kv, layer);
  a.k = k;
  a.v = v;
  a.ldk = ldk;
  a.ldv = ldv;
  a.slot = q->dev + q->at_slot;
  a.T = q->T;
  SERVE_HIP(ctx, salt::launch_kv_write(a, cv.bf16, s));
  return SALT_OK;
}

salt_status salt_kv_read(salt_ctx* ctx, salt_seqs* q, int32_t layer, int32_t what, void* k, int64_t ldk, void* v,
                         int64_t ldv, void* stream) {
  salt_status st = batch_call(ctx, q, layer);
  if (st != SALT_OK) return st;
  if (what != SALT_KV_NEW && what != SALT_KV_OWN)
    return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "what = %d is neither SALT_KV_NEW nor SALT_KV_OWN", what);
  if (what == SALT_KV_NEW ? q->T == 0 : q->own_tokens == 0) return SALT_OK;
  const salt_kv* kv = q->kv;
  const int64_t width = (int64_t)kv->cfg.n_kv_heads * kv->cfg.head_dim;
  if ((st = rows_arg(ctx, "k", k, ldk, width)) != SALT_OK || (st = rows_arg(ctx, "v", v, ldv, width)) != SALT_OK)
    return st;
  const salt::CtxView cv = salt::ctx_view(ctx);
  SERVE_HIP(ctx, hipSetDevice(cv.device));
  const hipStream_t s = (hipStream_t)stream;
  if ((st = enter(ctx, q, s)) != SALT_OK) return st;
  salt::KvReadArgs a{};
  a.kv = layer_of(kv, layer);
  a.k = k;
  a.v = v;
  a.ldk = ldk;
  a.ldv = ldv;
  if (what == SALT_KV_NEW) {
    a.slot = q->dev + q->at_slot;
    a.n = q->T;
  } else {
    a.page = q->dev + q->at_page + (q->n_refs - q->n_own_refs);
    a.row = q->dev + q->at_row;
    a.count = q->dev + q->at_count;
    a.n = q->n_own_refs;
  }
  SERVE_HIP(ctx, salt::launch_kv_read(a, cv.bf16, s));
  return SALT_OK;
}

salt_status salt_attend(salt_ctx* ctx, salt_seqs* q, int32_t layer, const void* queries, int64_t ldq, void* out,
                        int64_t ldo, float scale, void* stream) {
  salt_status st = batch_call(ctx, q, layer);
  if (st != SALT_OK) return st;
  if (!std::isfinite(scale) || !(scale > 0.f)) return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "scale must be finite and > 0");
  if (q->T == 0) return SALT_OK;
  const salt_kv* kv = q->kv;
  const int64_t width = (int64_t)kv->cfg.n_heads * kv->cfg.head_dim;
  if ((st = rows_arg(ctx, "q", queries, ldq, width)) != SALT_OK || (st = rows_arg(ctx, "out", out, ldo, width)) != SALT_OK)
    return st;
  const salt::CtxView cv = salt::ctx_view(ctx);
  SERVE_HIP(ctx, hipSetDevice(cv.device));
  const hipStream_t s = (hipStream_t)stream;
  if ((st = enter(ctx, q, s)) != SALT_OK) return st;
  salt::AttArgs a{};
  a.kv = layer_of(kv, layer);
  a.q = queries;
  a.out = out;
  a.ldq = ldq;
  a.ldo = ldo;
  a.pages = q->dev + q->at_page;
  a.order = q->dev + q->at_order;
  a.items = reinterpret_cast<const salt::AttItem*>(q->dev + q->at_item);
  a.joins = reinterpret_cast<const salt::AttJoin*>(q->dev + q->at_join);
  a.part = q->part;
  a.stat = q->stat;
  a.heads = kv->cfg.n_heads;
  a.group = kv->cfg.n_heads / kv->cfg.n_kv_heads;
  std::copy(q->n_kind, q->n_kind + 4, a.n_kind);
  a.n_joins = q->n_joins;
  a.scale = scale;
  SERVE_HIP(ctx, salt::launch_attend(a, cv.bf16, s));
  return SALT_OK;
}

}  // extern "C"
