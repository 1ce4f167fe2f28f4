// Host build of salt_decode.cpp and salt_serve.cpp with a stand-in for the HIP runtime and for what they take from a
// context; the launches note their arguments and do nothing.  argv[1]:
//   refusals  every call that has to be refused, with its status, and that nothing was launched.
//   launches  what reaches a launch: copies cut into launches, beams within their buffers at every size, eviction
//             that has nothing to do.
//   capture   work under capture behind another stream's is refused.
//   memory    host memory runs out at the first, second, .. allocation: no exception leaves an entry point, the
//             same call works afterwards, and nothing is leaked.
// Prints the first failure and exits 1, else "ok".
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstdlib>
#include <limits>
#include <new>
#include <utility>
#include <vector>

#include "salt.h"
#include "salt_decode.h"
#include "salt_serve.h"

static long g_left = -1, g_news = 0;
void* operator new(size_t n) {
  if (g_left >= 0 && g_left-- == 0) throw std::bad_alloc();
  ++g_news;
  if (void* p = malloc(n ? n : 1)) return p;
  abort();
}
void operator delete(void* p) noexcept {
  if (p) --g_news, free(p);
}
void operator delete(void* p, size_t) noexcept { operator delete(p); }

static void need(bool ok, const char* what, long a = 0, long b = 0) {
  if (ok) return;
  std::printf("FAIL %s (%ld %ld)\n", what, a, b);
  std::exit(1);
}

constexpr salt_shape kTables[1] = {{64, 64}};
struct salt_ctx {
  std::vector<std::pair<void*, salt::OwnedFree>> owned;
  void* base = nullptr;
};
static int g_launches = 0, g_copies = 0;
static salt::BeamArgs g_beam;
static salt::RotateArgs g_rotate;
static salt::ScoreArgs g_score;
static salt::EvictArgs g_evict;
static std::vector<int>* g_pairs = nullptr;
namespace salt {
salt_status ctx_live(salt_ctx* c) { return c ? SALT_OK : SALT_ERR_INVALID_ARG; }
CtxView ctx_view(const salt_ctx*) { return CtxView{0, 256, 1, 16, 1, kTables}; }
salt_status ctx_fail(salt_ctx*, salt_status s, const char*, ...) { return s; }
salt_status ctx_hip_fail(salt_ctx*, hipError_t, const char*) { return SALT_ERR_HIP; }
bool ctx_own(salt_ctx* c, void* obj, OwnedFree f) {
  try {
    c->owned.emplace_back(obj, f);
  } catch (const std::bad_alloc&) {
    return false;
  }
  return true;
}
bool ctx_owns(const salt_ctx* c, const void* obj) {
  for (const auto& o : c->owned)
    if (o.first == obj) return true;
  return false;
}
bool ctx_disown(salt_ctx* c, void* obj) {
  for (size_t i = 0; i < c->owned.size(); ++i)
    if (c->owned[i].first == obj) {
      c->owned.erase(c->owned.begin() + (long)i);
      return true;
    }
  return false;
}
void*& ctx_base(salt_ctx* c) { return c->base; }
hipError_t launch_base_pin(const BasePinArgs&, int, hipStream_t) { return ++g_launches, hipSuccess; }
hipError_t launch_base_pin_codes(const BasePinArgs&, hipStream_t) { return ++g_launches, hipSuccess; }
hipError_t launch_base_read(const BasePinArgs&, int, hipStream_t) { return ++g_launches, hipSuccess; }
hipError_t launch_base_product(const BaseArgs&, int, int, hipStream_t) { return ++g_launches, hipSuccess; }
hipError_t launch_kv_write(const KvWriteArgs&, int, hipStream_t) { return ++g_launches, hipSuccess; }
hipError_t launch_kv_read(const KvReadArgs&, int, hipStream_t) { return ++g_launches, hipSuccess; }
hipError_t launch_attend(const AttArgs&, int, hipStream_t) { return ++g_launches, hipSuccess; }
hipError_t launch_rotate(const RotateArgs& a, int, int, hipStream_t) { return g_rotate = a, ++g_launches, hipSuccess; }
hipError_t launch_score(const ScoreArgs& a, int, hipStream_t) { return g_score = a, ++g_launches, hipSuccess; }
hipError_t launch_marks(const MarksArgs&, bool, hipStream_t) { return ++g_launches, hipSuccess; }
hipError_t launch_evict(const EvictArgs& a, hipStream_t) { return g_evict = a, ++g_launches, hipSuccess; }
hipError_t launch_beam(const BeamArgs& a, int, hipStream_t) { return g_beam = a, ++g_launches, hipSuccess; }
hipError_t launch_copy(const CopyArgs& a, hipStream_t) {
  ++g_launches;
  g_copies += a.n;
  need(a.n >= 1 && a.n <= kCopyPairs, "pairs of a launch", a.n);
  if (g_pairs)
    for (int i = 0; i < a.n; ++i) g_pairs->insert(g_pairs->end(), {a.src[i], a.dst[i], a.tokens[i]});
  return hipSuccess;
}
}  // namespace salt

alignas(16) static char g_buf[1 << 16];
static float* const F = (float*)g_buf;
static int32_t* const I = (int32_t*)g_buf;

static void close_context(salt_ctx* c) {
  for (const auto& o : c->owned) o.second(o.first);
  delete c;
  need(fake::live == 0, "leaked device memory or events", fake::live);
}

struct World {
  salt_ctx* c = new salt_ctx;
  salt_kv* kv = nullptr;
  salt_seqs* q = nullptr;
  salt_beams* b = nullptr;
  explicit World(bool track = true, int page = 16, int pages = 64) {
    const salt_kv_config cfg{2, 8, 2, 64, page, pages, SALT_KV_E4M3, 0};
    need(salt_kv_create(c, &cfg, &kv) == SALT_OK, "salt_kv_create");
    if (track) need(salt_kv_track(c, kv) == SALT_OK && salt_kv_track(c, kv) == SALT_OK, "salt_kv_track");
    need(salt_seqs_create(c, kv, 4, 8, 64, &q) == SALT_OK, "salt_seqs_create");
    need(salt_beams_create(c, 24, 16, &b) == SALT_OK, "salt_beams_create");
  }
  ~World() { close_context(c); }
  void set(int32_t l0, int32_t l1, const int32_t* pages, int32_t n_dom = 0, int32_t pre_page = 0) {
    const int32_t q_len[2] = {1, 2}, len[2] = {l0, l1}, dom[2] = {0, -1}, pre_len[1] = {9}, pre_off[2] = {0, 1};
    const int32_t n0 = (l0 + 15) / 16, off[3] = {0, n0, n0 + (l1 + 15) / 16};
    const salt_seq_batch batch{2, q_len, len, off, pages, n_dom ? dom : nullptr, n_dom, pre_len, pre_off, &pre_page};
    need(salt_seqs_set(c, q, &batch, nullptr) == SALT_OK, "salt_seqs_set");
  }
};

static int refusals() {
  const double inf = std::numeric_limits<double>::infinity(), freq[128] = {1.0};
  {
    World w;
    const int32_t pages[4] = {0, 1, 2, 3}, twice[4] = {0, 1, 1, 2};
    const int before = g_launches;
    auto is = [&](salt_status got, salt_status want, const char* what, long i = 0) { need(got == want, what, got, i); };
    // before a batch was set
    is(salt_kv_score(w.c, w.q, 0, g_buf, 0, I, 1.f, 0, nullptr), SALT_ERR_BAD_STATE, "score without a batch");
    is(salt_kv_evict(w.c, w.q, 0, 3, 1, nullptr), SALT_ERR_BAD_STATE, "evict without a batch");
    w.set(20, 30, pages);
    is(salt_kv_score(nullptr, w.q, 0, g_buf, 0, I, 1.f, 0, nullptr), SALT_ERR_INVALID_ARG, "null context");
    is(salt_kv_score(w.c, nullptr, 0, g_buf, 0, I, 1.f, 0, nullptr), SALT_ERR_INVALID_ARG, "null sequences");
    for (int l : {-1, 2}) {
      is(salt_kv_score(w.c, w.q, l, g_buf, 0, I, 1.f, 0, nullptr), SALT_ERR_OUT_OF_RANGE, "score layer", l);
      is(salt_kv_evict(w.c, w.q, l, 3, 1, nullptr), SALT_ERR_OUT_OF_RANGE, "evict layer", l);
      is(salt_kv_read_marks(w.c, w.q, l, F, I, nullptr), SALT_ERR_OUT_OF_RANGE, "marks layer", l);
    }
    is(salt_kv_score(w.c, w.q, 0, g_buf + 8, 0, I, 1.f, 0, nullptr), SALT_ERR_INVALID_ARG, "misaligned q");
    is(salt_kv_score(w.c, w.q, 0, nullptr, 0, I, 1.f, 0, nullptr), SALT_ERR_INVALID_ARG, "null q");
    is(salt_kv_score(w.c, w.q, 0, g_buf, 504, I, 1.f, 0, nullptr), SALT_ERR_INVALID_ARG, "short rows");
    is(salt_kv_score(w.c, w.q, 0, g_buf, 516, I, 1.f, 0, nullptr), SALT_ERR_INVALID_ARG, "rows not of 8");
    is(salt_kv_score(w.c, w.q, 0, g_buf, 0, (int32_t*)(g_buf + 2), 1.f, 0, nullptr), SALT_ERR_INVALID_ARG, "misaligned positions");
    is(salt_kv_score(w.c, w.q, 0, g_buf, 0, I, 0.f, 0, nullptr), SALT_ERR_INVALID_ARG, "scale 0");
    is(salt_kv_score(w.c, w.q, 0, g_buf, 0, I, (float)inf, 0, nullptr), SALT_ERR_INVALID_ARG, "scale inf");
    is(salt_kv_score(w.c, w.q, 0, g_buf, 0, I, 1.f, -1, nullptr), SALT_ERR_OUT_OF_RANGE, "window");
    for (auto kr : {std::pair<int, int>{-1, 0}, {3, -1}, {3, 4}})
      is(salt_kv_evict(w.c, w.q, 0, kr.first, kr.second, nullptr), SALT_ERR_OUT_OF_RANGE, "keep and recent", kr.first);
    is(salt_kv_read_marks(w.c, w.q, 0, nullptr, I, nullptr), SALT_ERR_INVALID_ARG, "null marks");
    is(salt_kv_write_marks(w.c, w.q, 0, F, (int32_t*)(g_buf + 4), nullptr), SALT_ERR_INVALID_ARG, "misaligned marks");
    w.set(20, 30, twice);
    is(salt_kv_score(w.c, w.q, 0, g_buf, 0, I, 1.f, 0, nullptr), SALT_ERR_INVALID_ARG, "score of shared pages");
    is(salt_kv_evict(w.c, w.q, 0, 3, 1, nullptr), SALT_ERR_INVALID_ARG, "evict of shared pages");
    is(salt_kv_write_marks(w.c, w.q, 0, F, I, nullptr), SALT_ERR_INVALID_ARG, "marks of shared pages");
    w.set(20, 30, pages, 1, 2);
    is(salt_kv_evict(w.c, w.q, 0, 3, 1, nullptr), SALT_ERR_INVALID_ARG, "a page of a sequence and a domain");
    // rotation
    const salt_rotation ok{4, 2, 64, 32, 0, freq, nullptr, nullptr, 1e-6f, 1.f};
    auto rot = [&](auto change) {
      salt_rotation r = ok;
      change(r);
      return salt_rotate(w.c, &r, 3, I, g_buf, 0, g_buf, 0, g_buf + 4096, 0, g_buf + 4096, 0, nullptr);
    };
    std::vector<double> bad(128, 1.0);
    int k = 0;
    auto no = [&](auto change) { is(rot(change), SALT_ERR_INVALID_ARG, "rotation", k++); };
    no([](salt_rotation& r) { r.n_heads = -1; });
    no([](salt_rotation& r) { r.n_kv_heads = 65537; });
    no([](salt_rotation& r) { r.n_heads = r.n_kv_heads = 0; });
    no([](salt_rotation& r) { r.head_dim = 60; });
    no([](salt_rotation& r) { r.head_dim = 264; });
    no([](salt_rotation& r) { r.head_dim = 0; });
    no([](salt_rotation& r) { r.rot_dim = 0; });
    no([](salt_rotation& r) { r.rot_dim = 72; });
    no([](salt_rotation& r) { r.rot_dim = 12; });
    no([](salt_rotation& r) { r.interleaved = 2; });
    no([](salt_rotation& r) { r.freq = nullptr; });
    no([](salt_rotation& r) { r.q_norm = g_buf + 2; });
    no([](salt_rotation& r) { r.k_norm = g_buf + 8; });
    no([](salt_rotation& r) { r.eps = -1.f; });
    no([](salt_rotation& r) { r.eps = NAN; });
    no([](salt_rotation& r) { r.gain = INFINITY; });
    for (double f : {std::nan(""), inf, 1.1e4, -1.1e4}) {
      bad[15] = f;
      no([&](salt_rotation& r) { r.freq = bad.data(); });
    }
    auto call = [&](int T, const void* p, const void* q, int64_t lq, void* qo, int64_t lqo, const void* kk, int64_t lk) {
      return salt_rotate(w.c, &ok, T, (const int32_t*)p, q, lq, qo, lqo, kk, lk, g_buf + 8192, 0, nullptr);
    };
    char* g = g_buf;
    is(salt_rotate(w.c, nullptr, 1, I, g, 0, g, 0, g, 0, g, 0, nullptr), SALT_ERR_INVALID_ARG, "null rotation");
    is(call(-1, g, g, 0, g, 0, g, 0), SALT_ERR_OUT_OF_RANGE, "T < 0");
    is(call((1 << 20) + 1, g, g, 0, g, 0, g, 0), SALT_ERR_OUT_OF_RANGE, "T > 2^20");
    is(call(1, nullptr, g, 0, g, 0, g, 0), SALT_ERR_INVALID_ARG, "null positions");
    is(call(1, g + 1, g, 0, g, 0, g, 0), SALT_ERR_INVALID_ARG, "misaligned positions");
    is(call(1, g, nullptr, 0, g, 0, g, 0), SALT_ERR_INVALID_ARG, "null q");
    is(call(1, g, g, 0, g + 4, 0, g, 0), SALT_ERR_INVALID_ARG, "misaligned q_out");
    is(call(1, g, g, 248, g, 0, g, 0), SALT_ERR_INVALID_ARG, "short q rows");
    is(call(1, g, g, 0, g, 264, g, 0), SALT_ERR_INVALID_ARG, "in place with other rows");
    is(call(1, g, g, 0, g, 0, nullptr, 0), SALT_ERR_INVALID_ARG, "null k");
    is(call(1, g, g, 0, g, 0, g, 132), SALT_ERR_INVALID_ARG, "k rows not of 8");
    // beams
    auto sel = [&](salt_beams* b, int reqs, int width, int vocab, const void* x, int64_t ld, const float* s, int n, int32_t* t) {
      return salt_beam_select(w.c, b, reqs, width, vocab, x, ld, s, n, F, I, t, nullptr);
    };
    is(sel(nullptr, 1, 1, 8, g, 0, F, 1, I), SALT_ERR_INVALID_ARG, "null beams");
    is(sel((salt_beams*)w.kv, 1, 65, 8, g, 0, F, 1, I), SALT_ERR_OUT_OF_RANGE, "width 65");
    is(sel(w.b, -1, 1, 8, g, 0, F, 1, I), SALT_ERR_OUT_OF_RANGE, "reqs < 0");
    is(sel(w.b, 1, 0, 8, g, 0, F, 1, I), SALT_ERR_OUT_OF_RANGE, "width 0");
    is(sel(w.b, 5, 5, 8, g, 0, F, 1, I), SALT_ERR_OUT_OF_RANGE, "25 rows of 24");
    is(sel(w.b, 1 << 30, 8, 8, g, 0, F, 1, I), SALT_ERR_OUT_OF_RANGE, "2^33 rows");
    for (int n : {0, 17, 64}) is(sel(w.b, 1, 1, 8, g, 0, F, n, I), SALT_ERR_OUT_OF_RANGE, "n_out", n);
    for (int v : {0, (1 << 24) + 8}) is(sel(w.b, 1, 1, v, g, 0, F, 1, I), SALT_ERR_OUT_OF_RANGE, "vocab", v);
    is(sel(w.b, 1, 1, 9, g, 0, F, 1, I), SALT_ERR_INVALID_ARG, "dense rows not of 8");
    is(sel(w.b, 1, 1, 9, g, 8, F, 1, I), SALT_ERR_INVALID_ARG, "rows short of the vocabulary");
    is(sel(w.b, 1, 1, 8, g + 2, 0, F, 1, I), SALT_ERR_INVALID_ARG, "misaligned logits");
    is(sel(w.b, 1, 1, 8, g, 0, nullptr, 1, I), SALT_ERR_INVALID_ARG, "null scores");
    is(sel(w.b, 1, 1, 8, g, 0, F, 1, (int32_t*)(g + 2)), SALT_ERR_INVALID_ARG, "misaligned tokens");
    salt_beams* nb = (salt_beams*)g;
    is(salt_beams_create(w.c, 0, 1, &nb), SALT_ERR_OUT_OF_RANGE, "max_rows 0");
    need(nb == nullptr, "a refused create hands out nothing");
    is(salt_beams_create(w.c, 65537, 1, &nb), SALT_ERR_OUT_OF_RANGE, "max_rows");
    is(salt_beams_create(w.c, 1, 65, &nb), SALT_ERR_OUT_OF_RANGE, "max_out");
    is(salt_beams_create(w.c, 1, 1, nullptr), SALT_ERR_INVALID_ARG, "null out");
    // copies
    auto copy = [&](std::vector<int32_t> s, std::vector<int32_t> d, const int32_t* t = nullptr) {
      return salt_kv_copy(w.c, w.kv, (int)s.size(), s.data(), d.data(), t, nullptr);
    };
    const int32_t t17 = 17, tm = -1;
    is(copy({64}, {0}), SALT_ERR_OUT_OF_RANGE, "source page");
    is(copy({0}, {-1}), SALT_ERR_OUT_OF_RANGE, "target page");
    is(copy({0}, {1}, &t17), SALT_ERR_OUT_OF_RANGE, "tokens of a page");
    is(copy({0}, {1}, &tm), SALT_ERR_OUT_OF_RANGE, "tokens < 0");
    is(copy({0, 1}, {2, 2}), SALT_ERR_INVALID_ARG, "written twice");
    is(copy({0, 1}, {1, 2}), SALT_ERR_INVALID_ARG, "read and written");
    is(copy({5}, {5}), SALT_ERR_INVALID_ARG, "onto itself");
    is(salt_kv_copy(w.c, w.kv, 65, I, I, nullptr, nullptr), SALT_ERR_OUT_OF_RANGE, "more copies than pages");
    is(salt_kv_copy(w.c, w.kv, -1, I, I, nullptr, nullptr), SALT_ERR_INVALID_ARG, "n < 0");
    is(salt_kv_copy(w.c, w.kv, 1, nullptr, I, nullptr, nullptr), SALT_ERR_INVALID_ARG, "null pages");
    is(salt_kv_copy(w.c, nullptr, 0, I, I, nullptr, nullptr), SALT_ERR_INVALID_ARG, "null cache");
    need(g_launches == before, "a refused call was launched", g_launches, before);
  }
  World w(false);
  const int32_t pages[4] = {0, 1, 2, 3};
  w.set(20, 30, pages);
  const int before = g_launches;
  need(salt_kv_score(w.c, w.q, 0, g_buf, 0, I, 1.f, 0, nullptr) == SALT_ERR_BAD_STATE, "score of an untracked cache");
  need(salt_kv_evict(w.c, w.q, 0, 3, 1, nullptr) == SALT_ERR_BAD_STATE, "evict of an untracked cache");
  need(salt_kv_read_marks(w.c, w.q, 0, F, I, nullptr) == SALT_ERR_BAD_STATE, "marks of an untracked cache");
  need(salt_kv_write_marks(w.c, w.q, 0, F, I, nullptr) == SALT_ERR_BAD_STATE, "marks into an untracked cache");
  need(g_launches == before, "a refused call was launched");
  std::printf("ok\n");
  return 0;
}

static int launches() {
  // a sequence's records and its page references' on the device
  {
    World w;
    const int32_t pages[5] = {7, 3, 9, 8, 2};
    w.set(40, 17, pages, 1, 11);
    need(salt_kv_score(w.c, w.q, 1, g_buf, 0, nullptr, 1.f, 0, nullptr) == SALT_OK, "score");
    const salt::BatchView& b = g_score.b;
    need(b.pre_refs == 1 && b.own_refs == 5 && b.n_seqs == 2, "references", b.pre_refs, b.own_refs);
    for (int i = 0; i < 5; ++i) {
      const int count[5] = {16, 16, 8, 16, 1}, row[5] = {0, 16, 32, 40, 56};
      need(b.count[i] == count[i] && b.row[i] == row[i] && b.pages[1 + i] == pages[i], "reference", i);
    }
    need(b.pages[0] == 11, "the prefix' page");
    need(b.rec[0].tok0 == 0 && b.rec[0].q_len == 1 && b.rec[0].len == 40 && b.rec[0].ref0 == 1, "record 0");
    need(b.rec[1].tok0 == 1 && b.rec[1].q_len == 2 && b.rec[1].len == 17 && b.rec[1].ref0 == 4, "record 1");
    need(b.n_units == 2 && b.unit[0] == 0 && b.unit[1] == 1 && b.rec[0].unit0 == 0 && b.rec[1].unit0 == 1, "units");
    need(g_score.joined[0] == -1 && g_score.joined[2] == -1 && g_score.few && !g_score.many, "joins and rows");
    need(g_score.back[0] == 0 && g_score.back[1] == 1 && g_score.back[2] == 0, "tokens behind");
    need(g_score.window == INT32_MAX, "window 0: all");
    int n = g_launches;
    need(salt_kv_evict(w.c, w.q, 0, 40, 0, nullptr) == SALT_OK && salt_kv_evict(w.c, w.q, 0, 0, 0, nullptr) == SALT_OK, "evict");
    need(g_launches == n, "an eviction that changes nothing is no launch");
    need(salt_kv_evict(w.c, w.q, 0, 39, 39, nullptr) == SALT_OK && g_launches == n + 1 && g_evict.max_len == 40, "evict 39");
    // copies: 64 pages' table, in launches of kCopyPairs
    n = g_launches;
    need(salt_kv_copy(w.c, w.kv, 0, nullptr, nullptr, nullptr, nullptr) == SALT_OK && g_launches == n, "no copies");
  }
  {
    World w(true, 16, 2000);
    std::vector<int> seen;
    std::vector<int32_t> src, dst, tok;
    for (int i = 0; i < 900; ++i) src.push_back(i % 7), dst.push_back(100 + i), tok.push_back(i % 17);
    g_pairs = &seen;
    const int n = g_launches;
    need(salt_kv_copy(w.c, w.kv, 900, src.data(), dst.data(), tok.data(), nullptr) == SALT_OK, "900 copies");
    need(salt_kv_copy(w.c, w.kv, 300, src.data(), dst.data(), nullptr, nullptr) == SALT_OK, "300 copies");
    g_pairs = nullptr;
    need(g_launches == n + 4 + 2 && seen.size() == 3 * 1200, "launches of the copies", g_launches - n, (long)seen.size());
    for (int i = 0; i < 1200; ++i) {
      const int j = i < 900 ? i : i - 900;
      need(seen[3 * i] == src[j] && seen[3 * i + 1] == dst[j] && seen[3 * i + 2] == (i < 900 ? tok[j] : 16), "pair", i);
    }
  }
  // beams: the pieces of every call lie in the buffers, and cover the vocabulary in whole runs
  for (int cu : {1, 80, 256, 304})
    for (int64_t rows = 1; rows <= salt::kMaxBeamRows; rows += 1 + rows / 5)
      for (int vocab : {1, 511, 2047, 2048, 4096, 32001, 131072, 200000, 1 << 24}) {
        const int s = salt::beam_splits(rows, vocab, cu);
        need(s >= 1 && s <= salt::kMaxSplits && rows * s <= salt::beam_pieces(rows, cu), "pieces", (long)rows, s);
        need(rows * s <= salt::beam_pieces(salt::kMaxBeamRows, cu), "pieces of fewer rows", (long)rows, s);
        need(s <= (vocab + 511) / 512, "empty pieces", vocab, s);
      }
  World w;
  for (int rows = 1; rows <= 24; ++rows) {
    need(salt_beam_select(w.c, w.b, 1, rows, 130000, g_buf, 130000, F, 16, F, I, I, nullptr) == SALT_OK, "select", rows);
    need((int64_t)rows * g_beam.splits <= salt::beam_pieces(24, 256), "pieces in the buffers", rows, g_beam.splits);
  }
  const int n = g_launches;
  need(salt_beam_select(w.c, w.b, 0, 3, 8, nullptr, 0, nullptr, 1, nullptr, nullptr, nullptr, nullptr) == SALT_OK && g_launches == n, "no requests");
  const double freq[4] = {6.283185307179586476925286766559, 1, 0, -1};
  const salt_rotation r{1, 0, 8, 8, 1, freq, nullptr, nullptr, 0.f, 1.f};
  need(salt_rotate(w.c, &r, 0, nullptr, nullptr, 0, nullptr, 0, nullptr, 0, nullptr, 0, nullptr) == SALT_OK && g_launches == n, "no tokens");
  need(salt_rotate(w.c, &r, 1, I, g_buf, 0, g_buf, 16, nullptr, 0, nullptr, 0, nullptr) == SALT_ERR_INVALID_ARG, "rows in place");
  need(salt_rotate(w.c, &r, 1, I, g_buf, 0, g_buf, 0, nullptr, 0, nullptr, 0, nullptr) == SALT_OK && g_launches == n + 1, "one head");
  need(g_rotate.freq[0] == 1.0 && g_rotate.freq[2] == 0.0 && g_rotate.ldq == 8, "revolutions");
  std::printf("ok\n");
  return 0;
}

static int capture() {
  World w;
  const int32_t pages[4] = {0, 1, 2, 3}, one = 1, two = 2;
  w.set(20, 30, pages);
  hipStream_t a = (hipStream_t)g_buf, b = (hipStream_t)(g_buf + 64);
  need(salt_beam_select(w.c, w.b, 1, 1, 8, g_buf, 0, F, 1, F, I, I, a) == SALT_OK, "select");
  const int n = g_launches;
  fake::capturing = b;
  need(salt_beam_select(w.c, w.b, 1, 1, 8, g_buf, 0, F, 1, F, I, I, b) == SALT_ERR_BAD_STATE, "select under capture");
  need(salt_kv_score(w.c, w.q, 0, g_buf, 0, I, 1.f, 0, b) == SALT_ERR_BAD_STATE, "score under capture");
  need(salt_kv_evict(w.c, w.q, 0, 3, 1, b) == SALT_ERR_BAD_STATE, "evict under capture");
  need(g_launches == n && !fake::spoiled, "refused calls left something");
  fake::capturing = nullptr;
  w.set(20, 30, pages);                                    // (not recorded: it can be set)
  // on the object's own stream it is recorded, and the batch is the graph's from then on
  need(salt_kv_write_marks(w.c, w.q, 0, F, I, b) == SALT_OK, "marks");
  fake::capturing = b;
  need(salt_kv_score(w.c, w.q, 0, g_buf, 0, I, 1.f, 0, b) == SALT_OK && salt_kv_evict(w.c, w.q, 0, 3, 1, b) == SALT_OK &&
           salt_kv_copy(w.c, w.kv, 1, &one, &two, nullptr, b) == SALT_OK && !fake::spoiled, "recorded calls");
  fake::capturing = nullptr;
  const int32_t q_len[1] = {1}, len[1] = {1}, off[2] = {0, 1};
  const salt_seq_batch batch{1, q_len, len, off, pages, nullptr, 0, nullptr, nullptr, nullptr};
  need(salt_seqs_set(w.c, w.q, &batch, b) == SALT_ERR_BAD_STATE, "the batch of a graph");
  std::printf("ok\n");
  return 0;
}

static bool program(long fail) {
  salt_ctx* c = new salt_ctx;
  auto call = [&](const char* what, auto f) {
    for (int again = 0; again < 2; ++again) {
      salt_status st = SALT_OK;
      try {
        st = f();
      } catch (...) {
        need(false, what, fail, -1);
      }
      if (st == SALT_OK) return;
      need(st == SALT_ERR_OUT_OF_MEMORY && g_left < 0 && again == 0, what, fail, st);
    }
  };
  salt_kv* kv = nullptr;
  salt_seqs* q = nullptr;
  salt_beams* b = nullptr;
  const salt_kv_config cfg{2, 8, 2, 64, 16, 9, SALT_KV_E4M3, 0};
  const int32_t q_len[2] = {1, 2}, len[2] = {3, 20}, off[3] = {0, 1, 3}, pages[3] = {0, 1, 2}, src = 0, dst = 8;
  const salt_seq_batch batch{2, q_len, len, off, pages, nullptr, 0, nullptr, nullptr, nullptr};
  const double freq[4] = {1, 1, 1, 1};
  const salt_rotation r{1, 0, 8, 8, 1, freq, nullptr, nullptr, 0.f, 1.f};
  g_left = fail;
  call("salt_kv_create", [&] { return salt_kv_create(c, &cfg, &kv); });
  call("salt_kv_track", [&] { return salt_kv_track(c, kv); });
  call("salt_seqs_create", [&] { return salt_seqs_create(c, kv, 4, 8, 8, &q); });
  call("salt_beams_create", [&] { return salt_beams_create(c, 4, 4, &b); });
  call("salt_seqs_set", [&] { return salt_seqs_set(c, q, &batch, nullptr); });
  call("salt_rotate", [&] { return salt_rotate(c, &r, 1, I, g_buf, 0, g_buf, 0, nullptr, 0, nullptr, 0, nullptr); });
  call("salt_kv_score", [&] { return salt_kv_score(c, q, 1, g_buf, 0, nullptr, 1.f, 0, nullptr); });
  call("salt_kv_evict", [&] { return salt_kv_evict(c, q, 1, 4, 2, nullptr); });
  call("salt_kv_write_marks", [&] { return salt_kv_write_marks(c, q, 1, F, I, nullptr); });
  call("salt_kv_read_marks", [&] { return salt_kv_read_marks(c, q, 1, F, I, nullptr); });
  call("salt_kv_copy", [&] { return salt_kv_copy(c, kv, 1, &src, &dst, nullptr, nullptr); });
  call("salt_beam_select", [&] { return salt_beam_select(c, b, 1, 4, 8, g_buf, 0, F, 4, F, I, I, nullptr); });
  salt_beams_destroy(c, b);
  const bool reached = g_left < 0 && fail >= 0;
  g_left = -1;
  close_context(c);
  return reached;
}

static int memory() {
  program(-1);
  const long before = g_news;
  long n = 0;
  while (program(n)) ++n;
  need(n >= 8, "allocations of the program", n);
  need(g_news == before, "leaked host memory", g_news, before);
  std::printf("ok\n");
  return 0;
}

int main(int argc, char** argv) {
  if (argc == 2 && !strcmp(argv[1], "refusals")) return refusals();
  if (argc == 2 && !strcmp(argv[1], "launches")) return launches();
  if (argc == 2 && !strcmp(argv[1], "capture")) return capture();
  if (argc == 2 && !strcmp(argv[1], "memory")) return memory();
  return 2;
}
