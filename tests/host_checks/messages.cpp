// A context's calls answer, and keep their messages, where host memory is out: salt_runtime.cpp built for the host with
// tests/cpu_kernels/hip in place of HIP.  Its kernels are not linked: no call in here launches one.
// Prints the first failure and exits 1, else "ok".
#include <hip/hip_runtime.h>

#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <new>

#include "salt.h"
#include "salt_serve.h"

static bool g_out = false;
void* operator new(size_t n) {
  if (g_out) throw std::bad_alloc();
  if (void* p = malloc(n ? n : 1)) return p;
  abort();
}
void operator delete(void* p) noexcept { free(p); }
void operator delete(void* p, size_t) noexcept { free(p); }

static void need(bool ok, const char* what) {
  if (ok) return;
  g_out = false;
  std::printf("FAIL %s\n", what);
  std::exit(1);
}
namespace salt {
hipError_t kernels_init(int) { return hipSuccess; }
}

int main() {
  const salt_shape table = {64, 64};
  const salt_config cfg = {SALT_BF16, 1, &table, 0, 0, 1, 0, 4, 0, 0};
  salt_ctx* c = nullptr;
  need(salt_create(&cfg, &c) == SALT_OK, "salt_create");
  for (int i = 0; i < 3; ++i) {
    salt_status st = SALT_OK;
    g_out = true;
    try {
      if (i == 0) st = salt_load_residual(c, 1 << 20, 0, nullptr, 0);
      if (i == 1) st = salt::ctx_fail(c, SALT_ERR_OUT_OF_MEMORY, "base weights %0600d", 7);
      if (i == 2) st = salt::ctx_hip_fail(c, hipErrorOutOfMemory, "a call whose name is longer than what a string holds in place");
    } catch (...) {
      need(false, "an exception left the call");
    }
    g_out = false;
    const salt_status want[] = {SALT_ERR_OUT_OF_RANGE, SALT_ERR_OUT_OF_MEMORY, SALT_ERR_HIP};
    const char* say[] = {"1048576", "base weights 000", "a call whose name is longer than what a string holds in place: "};
    need(st == want[i], "status");
    need(strstr(salt_last_error(c), say[i]) && strlen(salt_last_error(c)) < 512, "message");
  }
  // (poisoned now: the message goes into the next one)
  g_out = true;
  need(salt_wait_loads(c) == SALT_ERR_BAD_STATE, "a poisoned context");
  g_out = false;
  need(strstr(salt_last_error(c), "context is poisoned: a call whose name"), "the message of a poisoned context");
  std::printf("ok\n");
}
