// What the rotation and append calls, and attention with scales, answer where the library's own memory runs out: every allocation that libscoot.so makes while a
// call is watched throws, and the call has to return a status all the same.  Run without a GPU (the devices hidden): the
// calls then build an error message, which allocates.  Prints "name status message" per call.
#include <dlfcn.h>
#include <execinfo.h>

#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <new>

#include "scoot.h"

static thread_local bool watched = false;
static thread_local int thrown = 0;

static bool from_library() {
  void* at[12];
  const int n = backtrace(at, 12);
  for (int i = 0; i < n; ++i) {
    Dl_info info;
    if (!dladdr(at[i], &info) || !info.dli_fname) continue;
    if (std::strstr(info.dli_fname, "libscoot")) return true;
    if (!std::strstr(info.dli_fname, "libstdc++") && !std::strstr(info.dli_fname, "rotary_alloc_check")) return false;
  }
  return false;
}
void* operator new(std::size_t size) {
  if (watched) {
    watched = false;
    const bool mine = from_library();
    watched = true;
    if (mine) {
      ++thrown;
      throw std::bad_alloc();
    }
  }
  void* p = std::malloc(size ? size : 1);
  if (!p) throw std::bad_alloc();
  return p;
}
void operator delete(void* p) noexcept { std::free(p); }
void operator delete(void* p, std::size_t) noexcept { std::free(p); }

template <typename F, typename... A>
static void call(void* lib, const char* name, A... args) {
  F* f = (F*)dlsym(lib, name);
  const auto message = (const char* (*)())dlsym(lib, "scoot_last_error");
  void* warm[4];
  backtrace(warm, 4);  // loads what it needs
  watched = true;
  const int rc = f(args...);
  watched = false;
  std::printf("%s %d %d %s\n", name, thrown, rc, message());
  std::fflush(stdout);
  thrown = 0;
}

int main(int argc, char** argv) {
  void* lib = argc > 1 ? dlopen(argv[1], RTLD_NOW) : nullptr;
  if (!lib) return std::fprintf(stderr, "%s\n", dlerror()), 2;
  alignas(64) static char buf[4096];
  int32_t* i = (int32_t*)buf;
  int64_t* s = (int64_t*)buf;
  double* f = (double*)buf;
  float *a = (float*)buf, *b = (float*)(buf + 64);
  const auto append = [&](scoot_kv_type cache, float* ks, float* vs) {
    call<decltype(scoot_kv_append)>(lib, "scoot_kv_append", buf, 4, (int64_t)256, (int64_t)64, buf, (int64_t)256, (int64_t)64, buf, buf, SCOOT_KV_BF16,
                                    (int64_t)4, 2, 64, (int64_t)128, (int64_t)64, (int64_t)128, (int64_t)64, i, s, f, 64, 0, 1.0, buf, buf, cache,
                                    (int64_t)4, 16, 1.0f, 1.0f, ks, vs, nullptr);
  };
  call<decltype(scoot_rotate)>(lib, "scoot_rotate", buf, SCOOT_KV_BF16, (int64_t)4, 2, 64, (int64_t)128, (int64_t)64, i, f, 64, 0, 1.0, 0, buf,
                               (int64_t)128, (int64_t)64, nullptr);
  append(SCOOT_KV_BF16, nullptr, nullptr);
  append(SCOOT_KV_F8, a, b);
  call<decltype(scoot_kv_attention_scaled)>(lib, "scoot_kv_attention_scaled", buf, SCOOT_KV_BF16, (int64_t)4, 4, 2, 64, (int64_t)256, (int64_t)64, buf,
                                            buf, (int64_t)4, 16, i, 4, (int64_t)4, i, i, 2, (int64_t)2, (int64_t)9, 0.1f, 0, a, b, buf, (int64_t)256,
                                            (int64_t)64, nullptr, (uint64_t)0, nullptr);
  return 0;
}
