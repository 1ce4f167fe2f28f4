// Host build of salt_decode.cpp and salt_serve.cpp with a stand-in for the HIP runtime and for what they take from a
// context; the launches note their arguments and do nothing.  argv[1]:
//   written   salt_kv_write starts the marks of the tokens that it writes, where the cache is tracked and the batch's
//             marks of the layer were not given before.
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
hipError_t launch_evict(const EvictArgs&, hipStream_t) { return ++g_launches, hipSuccess; }
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

int main(int argc, char** argv) {
  if (argc == 2 && !strcmp(argv[1], "written")) return written();
  return 2;
}
