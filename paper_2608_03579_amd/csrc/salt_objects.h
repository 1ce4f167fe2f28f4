// Objects of the operators around the apply, as the files of the host runtime that work on them share them
// (salt_serve.cpp, salt_decode.cpp), and the checks that their calls begin with.
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <vector>

#include "salt.h"
#include "salt_serve.h"

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

namespace salt {

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline size_t round_up(size_t v, size_t a) { return (v + a - 1) / a * a; }
inline int ceil_div(int a, int b) { return (a + b - 1) / b; }

inline bool is_capturing(hipStream_t s) {
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
inline salt_status enter_stream(salt_ctx* ctx, StreamOrder& o, hipStream_t s) {
  if (o.refuses(s))
    return ctx_fail(ctx, SALT_ERR_BAD_STATE, "work under capture on another stream than the object's last work");
  SERVE_HIP(ctx, o.enter(s));
  return SALT_OK;
}

}  // namespace salt

// ---- KV cache objects --------------------------------------------------------------------
struct salt_kv {
  salt_kv_config cfg{};
  int log2_page = 0;
  char* pool = nullptr;
  size_t codes = 0, scales = 0;       // bytes of one layer's k (or v) codes, and scales
  std::vector<salt_seqs*> seqs;
  char* marks = nullptr;              // gathered weights and positions (salt_kv_track), layer after layer
  std::vector<uint32_t> stamp;        // per page: the last count of `stamps` that met it
  uint32_t stamps = 0;
  salt::StreamOrder order;                  // writes and reads of the pool
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
  salt::StreamOrder order;
  // the batch
  int T = -1;                         // -1: none was set
  int n_refs = 0, n_own_refs = 0;
  int64_t own_tokens = 0;
  bool clash = false;                 // two of its tokens' pages are one page
  int shared = -1;                    // a page holds own tokens twice, or beside a prefix (-1: not looked at yet)
  int n_seqs = 0, max_len = 0;        // the longest sequence that it has
  bool recorded = false;              // a graph holds its launches: grid sizes and places in `dev`
  size_t at_page = 0, at_row = 0, at_count = 0, at_slot = 0, at_order = 0, at_item = 0, at_join = 0;
  size_t at_unit = 0, at_rec = 0, at_back = 0, at_joined = 0, at_place = 0;
  size_t at_prefix = 0;               // in `staging` alone: first page reference and pages in use of each prefix
  int n_domains = 0;
  int n_units = 0, min_q = 0, max_q = 0;   // units of own keys; new tokens of a sequence that has any
  int n_kind[4] = {0, 0, 0, 0}, n_joins = 0;
  std::vector<uint8_t> given;         // per layer: salt_kv_write_marks gave the batch's marks
};

namespace salt {

// A number that no page is stamped with.
inline uint32_t next_stamp(salt_kv* kv) {
  if (++kv->stamps == 0) {
    std::fill(kv->stamp.begin(), kv->stamp.end(), 0u);
    kv->stamps = 1;
  }
  return kv->stamps;
}

// Whether `kv` is a live cache of `ctx` (asked before anything of it is read).
inline salt_status kv_of(salt_ctx* ctx, const salt_kv* kv) {
  if (!kv || !salt::ctx_owns(ctx, kv)) return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "not a cache of this context");
  return SALT_OK;
}
inline salt_status seqs_of(salt_ctx* ctx, const salt_seqs* q) {
  if (!q) return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "null sequences");
  return kv_of(ctx, q->kv);
}

inline KvLayer layer_of(const salt_kv* kv, int layer) {
  KvLayer l{};
  char* p = kv->pool + (size_t)layer * 2 * (kv->codes + kv->scales);
  l.k = reinterpret_cast<uint8_t*>(p);
  l.v = reinterpret_cast<uint8_t*>(p + kv->codes);
  l.ks = reinterpret_cast<float*>(p + 2 * kv->codes);
  l.vs = reinterpret_cast<float*>(p + 2 * kv->codes + kv->scales);
  l.kv_heads = kv->cfg.n_kv_heads;
  l.dim = kv->cfg.head_dim;
  l.log2_page = kv->log2_page;
  l.format = kv->cfg.format;
  if (kv->marks) {
    l.weight = reinterpret_cast<float*>(kv->marks + (size_t)layer * 2 * kv->scales);
    l.place = reinterpret_cast<int32_t*>(kv->marks + (size_t)layer * 2 * kv->scales + kv->scales);
  }
  return l;
}

// Common checks of the calls on a set batch.
inline salt_status batch_call(salt_ctx* ctx, salt_seqs* q, int32_t layer) {
  SERVE_LIVE(ctx);
  const salt_status st = seqs_of(ctx, q);
  if (st != SALT_OK) return st;
  if (q->T < 0) return ctx_fail(ctx, SALT_ERR_BAD_STATE, "no batch was set on the sequences");
  if (layer < 0 || layer >= q->kv->cfg.n_layers)
    return ctx_fail(ctx, SALT_ERR_OUT_OF_RANGE, "layer %d not in [0, %d)", layer, q->kv->cfg.n_layers);
  return SALT_OK;
}
// A row-major operand of whole heads: rows `ld` elements apart (0: dense).
inline salt_status rows_arg(salt_ctx* ctx, const char* what, const void* p, int64_t& ld, int64_t width) {
  if (ld == 0) ld = width;
  if (!p || !aligned16(p)) return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "null or misaligned %s", what);
  if (ld < width || ld % 8 != 0)
    return ctx_fail(ctx, SALT_ERR_INVALID_ARG, "%s rows of %lld elements: need a multiple of 8 and >= %lld", what,
                    (long long)ld, (long long)width);
  return SALT_OK;
}
// The batch's buffers and the pool, on `s`.
inline salt_status enter(salt_ctx* ctx, salt_seqs* q, hipStream_t s) {
  if (q->kv->order.refuses(s))
    return ctx_fail(ctx, SALT_ERR_BAD_STATE, "work under capture on another stream than the cache's last work");
  salt_status st = enter_stream(ctx, q->order, s);
  if (st == SALT_OK) st = enter_stream(ctx, q->kv->order, s);
  if (st == SALT_OK && is_capturing(s)) q->recorded = true;
  return st;
}

}  // namespace salt
