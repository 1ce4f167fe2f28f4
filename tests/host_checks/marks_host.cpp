// Host build of salt_decode.cpp and salt_serve.cpp with a stand-in for the HIP runtime and for what they take from a
// context; the launches note their arguments and do nothing.  argv[1]:
//   written   salt_kv_write starts the marks of the tokens that it writes, where the cache is tracked and the batch's
//             marks of the layer were not given before.
//   shared    a batch with a page of two sequences, or of a sequence and a domain, is refused by the calls that change
//             marks; its pages are looked at when such a call comes, once for a batch, and not by salt_seqs_set.
//   range     evictions of sequences up to 2^19 tokens are launched, of longer ones refused.
// Prints the first failure and exits 1, else "ok".
#include <hip/hip_runtime.h>

#include <cstdarg>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <utility>
#include <vector>

#include "salt.h"
#include "salt_decode.h"
#include "salt_objects.h"
#include "salt_serve.h"

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
static int g_launches = 0;
static salt::KvWriteArgs g_write;
static salt::EvictArgs g_evict;
namespace salt {
salt_status ctx_live(salt_ctx* c) { return c ? SALT_OK : SALT_ERR_INVALID_ARG; }
CtxView ctx_view(const salt_ctx*) { return CtxView{0, 256, 1, 16, 1, kTables}; }
salt_status ctx_fail(salt_ctx*, salt_status s, const char*, ...) { return s; }
salt_status ctx_hip_fail(salt_ctx*, hipError_t, const char*) { return SALT_ERR_HIP; }
bool ctx_own(salt_ctx* c, void* obj, OwnedFree f) { return c->owned.emplace_back(obj, f), true; }
bool ctx_owns(const salt_ctx* c, const void* obj) {
  for (const auto& o : c->owned)
    if (o.first == obj) return true;
  return false;
}
bool ctx_disown(salt_ctx*, void*) { return false; }
void*& ctx_base(salt_ctx* c) { return c->base; }
hipError_t launch_base_pin(const BasePinArgs&, int, hipStream_t) { return ++g_launches, hipSuccess; }
hipError_t launch_base_pin_codes(const BasePinArgs&, hipStream_t) { return ++g_launches, hipSuccess; }
hipError_t launch_base_read(const BasePinArgs&, int, hipStream_t) { return ++g_launches, hipSuccess; }
hipError_t launch_base_product(const BaseArgs&, int, int, hipStream_t) { return ++g_launches, hipSuccess; }
hipError_t launch_kv_write(const KvWriteArgs& a, int, hipStream_t) { return g_write = a, ++g_launches, hipSuccess; }
hipError_t launch_kv_read(const KvReadArgs&, int, hipStream_t) { return ++g_launches, hipSuccess; }
hipError_t launch_attend(const AttArgs&, int, hipStream_t) { return ++g_launches, hipSuccess; }
hipError_t launch_rotate(const RotateArgs&, int, int, hipStream_t) { return ++g_launches, hipSuccess; }
hipError_t launch_score(const ScoreArgs&, int, hipStream_t) { return ++g_launches, hipSuccess; }
hipError_t launch_marks(const MarksArgs&, bool, hipStream_t) { return ++g_launches, hipSuccess; }
hipError_t launch_evict(const EvictArgs& a, hipStream_t) { return g_evict = a, ++g_launches, hipSuccess; }
hipError_t launch_beam(const BeamArgs&, int, hipStream_t) { return ++g_launches, hipSuccess; }
hipError_t launch_copy(const CopyArgs&, hipStream_t) { return ++g_launches, hipSuccess; }
}  // namespace salt

alignas(16) static char g_buf[1 << 16];
static float* const F = (float*)g_buf;
static int32_t* const I = (int32_t*)g_buf;

struct World {
  salt_ctx* c = new salt_ctx;
  salt_kv* kv = nullptr;
  salt_seqs* q = nullptr;
  const long live = fake::live;
  explicit World(bool track, int pages = 64, int max_tokens = 32) {
    const salt_kv_config cfg{2, 8, 2, 64, 16, pages, SALT_KV_E4M3, 0};
    need(salt_kv_create(c, &cfg, &kv) == SALT_OK, "salt_kv_create");
    if (track) need(salt_kv_track(c, kv) == SALT_OK, "salt_kv_track");
    need(salt_seqs_create(c, kv, 6, max_tokens, pages, &q) == SALT_OK, "salt_seqs_create");
  }
  ~World() {
    for (const auto& o : c->owned) o.second(o.first);
    delete c;
    need(fake::live == live, "leaked device memory or events", fake::live, live);
  }
  salt_status set(std::vector<int32_t> q_len, std::vector<int32_t> len, std::vector<int32_t> pages,
                  std::vector<int32_t> prefix = {}, std::vector<int32_t> prefix_pages = {}, std::vector<int32_t> prefix_off = {}) {
    std::vector<int32_t> off(1, 0), dom(len.size(), -1);
    for (int32_t n : len) off.push_back(off.back() + (n + 15) / 16);
    need((size_t)off.back() <= pages.size(), "pages of a batch");
    const salt_seq_batch b{(int32_t)len.size(), q_len.data(), len.data(), off.data(), pages.data(), dom.data(),
                           (int32_t)prefix.size(), prefix.data(), prefix_off.data(), prefix_pages.data()};
    return salt_seqs_set(c, q, &b, nullptr);
  }
  salt_status write(int layer) { return salt_kv_write(c, q, layer, g_buf, 0, g_buf, 0, nullptr); }
};

static int written() {
  World w(true);
  need(w.set({2, 0, 5, 20}, {40, 7, 3, 20}, {0, 1, 2, 3, 4, 5, 6}) == SALT_OK, "set");
  need(w.write(1) == SALT_OK && g_write.place, "a tracked cache's marks start with the write");
  int t = 0;
  for (int p : {38, 39}) need(g_write.place[t] == p && g_write.slot[t] == 2 * 16 + p - 32, "a step's tokens", t, g_write.place[t]), ++t;
  for (int p : {-2, -1, 0, 1, 2}) {
    need(p < 0 ? g_write.slot[t] == -1 : g_write.place[t] == p && g_write.slot[t] == 4 * 16 + p, "behind the first", t, p);
    ++t;
  }
  for (int p = 0; p < 20; ++p, ++t) need(g_write.place[t] == p, "a prompt", t, g_write.place[t]);
  need(t == g_write.T, "tokens", t, g_write.T);
  // marks that were given first stay, in their layer and for this batch
  need(salt_kv_read_marks(w.c, w.q, 0, F, I, nullptr) == SALT_OK && w.write(0) == SALT_OK && g_write.place, "marks read");
  need(salt_kv_write_marks(w.c, w.q, 1, F, I, nullptr) == SALT_OK, "marks given");
  need(w.write(1) == SALT_OK && !g_write.place, "marks that were given");
  need(w.write(0) == SALT_OK && g_write.place, "the other layer");
  need(w.set({1}, {-1}, {}) != SALT_OK && w.write(1) == SALT_OK && !g_write.place, "the batch that stays behind a refused one");
  need(w.set({1}, {41}, {0, 1, 2}) == SALT_OK && w.write(1) == SALT_OK && g_write.place && g_write.place[0] == 40, "the next batch");
  need(w.set({0}, {7}, {3}) == SALT_OK && w.write(0) == SALT_OK, "a batch without new tokens");
  World plain(false);
  need(plain.set({2}, {40}, {0, 1, 2}) == SALT_OK && plain.write(0) == SALT_OK && !g_write.place, "an untracked cache");
  need(salt_kv_track(plain.c, plain.kv) == SALT_OK && plain.write(0) == SALT_OK && g_write.place && g_write.place[1] == 39,
       "tracked behind the batch");
  std::printf("ok\n");
  return 0;
}

static int range() {
  const int most = 1 << 19;
  World w(true, most / 16 + 3);
  std::vector<int32_t> pages;
  for (int i = 0; i < most / 16 + 3; ++i) pages.push_back(i);
  need(w.set({0, 1}, {most, 9}, pages) == SALT_OK && salt_kv_evict(w.c, w.q, 0, most - 1, 5, nullptr) == SALT_OK, "2^19 tokens");
  need(g_evict.max_len == most && g_evict.keep == most - 1, "eviction's arguments", g_evict.max_len, g_evict.keep);
  const int n = g_launches;
  need(w.set({0, 1}, {most + 1, 9}, pages) == SALT_OK, "set");
  for (int keep : {1, 9, most})
    need(salt_kv_evict(w.c, w.q, 0, keep, 0, nullptr) == SALT_ERR_OUT_OF_RANGE, "2^19 + 1 tokens", keep);
  need(salt_kv_evict(w.c, w.q, 0, most + 1, 0, nullptr) == SALT_OK && g_launches == n, "nothing to evict");
  std::printf("ok\n");
  return 0;
}

static uint32_t g_seed = 1;
static int draw(int n) { return (int)((g_seed = g_seed * 1664525u + 1013904223u) >> 8) % n; }

static int shared() {
  int refused = 0;
  for (int round = 0; round < 400; ++round) {
    const int pages = 8 + draw(56);
    World w(round % 2 == 0, pages);
    for (int batch = 0; batch < 4; ++batch) {
      // holders with tables over few pages, some with references behind their last token
      std::vector<int32_t> q_len, len, tab, off{0}, pre, pre_tab, pre_off{0};
      auto holder = [&](std::vector<int32_t>& l, std::vector<int32_t>& t, std::vector<int32_t>& o, int most) {
        const int refs = draw(most + 1);
        l.push_back(refs ? draw(refs * 16 + 1) : 0);
        for (int k = 0; k < refs; ++k) t.push_back(draw(pages));
        o.push_back((int32_t)t.size());
      };
      const int n = 1 + draw(3), nd = draw(3);
      for (int i = 0; i < nd; ++i) holder(pre, pre_tab, pre_off, 2);
      for (int i = 0; i < n; ++i) holder(len, tab, off, 3), q_len.push_back(len.back() ? 1 : 0);
      const salt_seq_batch b{n, q_len.data(), len.data(), off.data(), tab.data(), nullptr, nd, pre.data(), pre_off.data(), pre_tab.data()};
      const uint32_t before = w.kv->stamps;
      need(salt_seqs_set(w.c, w.q, &b, nullptr) == SALT_OK, "set", round, batch);
      need((int)w.q->shared == -1 && w.kv->stamps == before + 1, "pages are looked at by salt_seqs_set", round, batch);
      int seen[64] = {};
      bool want = false;
      for (int i = 0; i < nd; ++i)
        for (int k = 0; k < (pre[i] + 15) / 16; ++k) seen[pre_tab[pre_off[i] + k]] = 1;
      for (int i = 0; i < n; ++i)
        for (int k = 0; k < (len[i] + 15) / 16; ++k) want |= seen[tab[off[i] + k]]++ > 0;
      if (!w.kv->marks) {
        need(salt_kv_evict(w.c, w.q, 0, 1, 1, nullptr) == SALT_ERR_BAD_STATE, "not tracked", round, batch);
        if (batch == 2) need(salt_kv_track(w.c, w.kv) == SALT_OK, "salt_kv_track");     // (behind the batch)
      }
      if (!w.kv->marks) continue;
      need(salt_kv_read_marks(w.c, w.q, 0, F, I, nullptr) == SALT_OK && w.kv->stamps == before + 1, "marks that are read", round, batch);
      // a refused batch, and other work on the cache's stamps, in between
      const int32_t bad = -1, src = 0, dst = 1;
      const salt_seq_batch no{1, &bad, &bad, off.data(), tab.data(), nullptr, 0, nullptr, nullptr, nullptr};
      need(salt_seqs_set(w.c, w.q, &no, nullptr) != SALT_OK, "a refused batch", round, batch);
      need(salt_kv_copy(w.c, w.kv, 1, &src, &dst, nullptr, nullptr) == SALT_OK, "copy", round, batch);
      refused += want;
      uint32_t after = 0;
      for (int again = 0; again < 3; ++again) {
        const salt_status ok = want ? SALT_ERR_INVALID_ARG : SALT_OK;
        need(salt_kv_score(w.c, w.q, 0, g_buf, 0, nullptr, 1.f, 0, nullptr) == ok, "score", round, batch);
        need(salt_kv_evict(w.c, w.q, 1, 1, 1, nullptr) == ok, "evict", round, batch);
        need(salt_kv_write_marks(w.c, w.q, 0, F, I, nullptr) == ok, "marks", round, batch);
        if (again) need(w.kv->stamps == after, "a batch is looked at once", round, batch);
        after = w.kv->stamps;
      }
    }
    if (round == 200) g_seed = 7;
  }
  need(refused > 100 && refused < 700, "batches of either kind", refused);
  // stamps that start again
  World w(true);
  need(w.set({1, 1}, {20, 20}, {0, 1, 2, 3}) == SALT_OK, "set");
  w.kv->stamps = UINT32_MAX;
  for (uint32_t& s : w.kv->stamp) s = 1;
  need(salt_kv_evict(w.c, w.q, 0, 3, 1, nullptr) == SALT_OK && w.kv->stamps == 1, "stamps from the start");
  w.kv->stamps = UINT32_MAX;
  for (uint32_t& s : w.kv->stamp) s = 1;
  need(w.set({1, 1}, {20, 20}, {0, 1, 2, 1}) == SALT_OK && salt_kv_write(w.c, w.q, 0, g_buf, 0, g_buf, 0, nullptr) == SALT_ERR_INVALID_ARG,
       "writes of two sequences into one page");
  w.kv->stamps = UINT32_MAX;
  for (uint32_t& s : w.kv->stamp) s = 1;
  const int32_t src = 5, dst = 6;
  need(salt_kv_copy(w.c, w.kv, 1, &src, &dst, nullptr, nullptr) == SALT_OK, "a copy where stamps start again");
  std::printf("ok\n");
  return 0;
}

int main(int argc, char** argv) {
  if (argc == 2 && !strcmp(argv[1], "written")) return written();
  if (argc == 2 && !strcmp(argv[1], "shared")) return shared();
  if (argc == 2 && !strcmp(argv[1], "range")) return range();
  return 2;
}
