// Host build of salt_serve.cpp with a stand-in for the HIP runtime and for what it takes from a context; its
// launches do nothing.  argv[1]:
//   capture   a table's first pin on a stream under capture is refused, before and after the context has base
//             weights, without a call that a capture forbids and without a trace; a later pin is recorded.
//   memory    host memory runs out at the first, second, .. allocation of a program that uses every entry point: no
//             exception leaves an entry point, each answers OK or OUT_OF_MEMORY, the same call works
//             afterwards, and nothing is leaked.
// Prints the first failure and exits 1, else "ok".
#include <hip/hip_runtime.h>

#include <cstdarg>
#include <cstdio>
#include <cstdlib>
#include <new>
#include <utility>
#include <vector>

#include "salt.h"
#include "salt_seqs.h"
#include "salt_serve.h"

static long g_left = -1;                    // allocations until the one that fails (-1: none does)
static long g_news = 0;
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

// ---- a context, as salt_serve.h has it ---------------------------------------------
constexpr salt_shape kTables[3] = {{264, 136}, {264, 72}, {264, 8}};
struct salt_ctx {
  std::vector<std::pair<void*, salt::OwnedFree>> owned;
  void* base = nullptr;
};
static int g_launches = 0;
namespace salt {
salt_status ctx_live(salt_ctx* c) { return c ? SALT_OK : SALT_ERR_INVALID_ARG; }
CtxView ctx_view(const salt_ctx*) { return CtxView{0, 256, 1, 16, 3, kTables}; }
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
}  // namespace salt

alignas(16) static char g_buf[1 << 16];

static void close_context(salt_ctx* c) {
  for (const auto& o : c->owned) o.second(o.first);
  delete c;
  need(fake::live == 0, "leaked device memory or events", fake::live);
}

static int capture() {
  salt_ctx* c = new salt_ctx;
  hipStream_t s = (hipStream_t)g_buf;
  for (int pinned = 0; pinned < 2; ++pinned) {
    if (pinned) need(salt_pin_base(c, 0, g_buf, 136, s) == SALT_OK, "pin");
    const long live = fake::live;
    const int launches = g_launches;
    fake::capturing = s;
    for (int t = 1; t < 3; ++t) {
      need(salt_pin_base(c, t, g_buf, 136, s) == SALT_ERR_BAD_STATE, "salt_pin_base under capture", pinned, t);
      need(salt_pin_base_fp8(c, t, g_buf, 264, (const float*)g_buf, s) == SALT_ERR_BAD_STATE, "salt_pin_base_fp8 under capture",
           pinned, t);
    }
    need(!fake::spoiled, "the capture was spoiled", pinned);
    fake::capturing = nullptr;
    need(fake::live == live && g_launches == launches, "a refused pin left something", pinned);
    const int32_t one = 1;
    void* y = g_buf;
    need(salt_read_base(c, 1, g_buf, 136, s) == SALT_ERR_BAD_STATE, "read of a table that was not pinned", pinned);
    need(salt_base_product(c, 1, &one, 1, g_buf, &y, s) == SALT_ERR_BAD_STATE, "product of a table that was not pinned", pinned);
  }
  fake::capturing = s;
  const int launches = g_launches;
  need(salt_pin_base(c, 0, g_buf, 136, s) == SALT_OK && salt_pin_base_fp8(c, 0, g_buf, 264, (const float*)g_buf, s) == SALT_OK,
       "a later pin under capture");
  need(!fake::spoiled && g_launches == launches + 2, "a later pin is recorded");
  fake::capturing = nullptr;
  close_context(c);
  std::printf("ok\n");
  return 0;
}

// Every entry point once, the `fail`-th allocation failing.  Whether there was one.
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
  const salt_kv_config cfg{2, 8, 2, 64, 16, 9, SALT_KV_E4M3, 0};
  const int32_t t0 = 0, q_len[2] = {1, 2}, len[2] = {3, 20}, off[3] = {0, 1, 3}, pages[3] = {0, 1, 2}, dom[2] = {0, 0};
  const int32_t pre_len[1] = {9}, pre_off[2] = {0, 1}, pre_pages[1] = {5};
  const salt_seq_batch b{2, q_len, len, off, pages, dom, 1, pre_len, pre_off, pre_pages};
  void* y = g_buf;
  g_left = fail;
  call("salt_pin_base", [&] { return salt_pin_base(c, 0, g_buf, 136, nullptr); });
  call("salt_pin_base_fp8", [&] { return salt_pin_base_fp8(c, 1, g_buf, 264, (const float*)g_buf, nullptr); });
  call("salt_base_product", [&] { return salt_base_product(c, 1, &t0, 3, g_buf, &y, nullptr); });
  call("salt_kv_create", [&] { return salt_kv_create(c, &cfg, &kv); });
  call("salt_seqs_create", [&] { return salt_seqs_create(c, kv, 4, 8, 8, &q); });
  call("salt_seqs_set", [&] { return salt_seqs_set(c, q, &b, nullptr); });
  call("salt_kv_write", [&] { return salt_kv_write(c, q, 1, g_buf, 0, g_buf, 0, nullptr); });
  call("salt_kv_read", [&] { return salt_kv_read(c, q, 1, SALT_KV_OWN, g_buf, 0, g_buf, 0, nullptr); });
  call("salt_attend", [&] { return salt_attend(c, q, 1, g_buf, 0, g_buf, 0, 1.f, nullptr); });
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
  need(n >= 20, "allocations of the program", n);
  need(g_news == before, "leaked host memory", g_news, before);
  std::printf("ok\n");
  return 0;
}

int main(int argc, char** argv) {
  if (argc == 2 && !strcmp(argv[1], "capture")) return capture();
  if (argc == 2 && !strcmp(argv[1], "memory")) return memory();
  return 2;
}
