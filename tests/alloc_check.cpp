// Calls that run out of host memory return an error, leak nothing and leave a
// history as it was: each allocation of each call fails in turn.  Linked with
// coded_check.cpp, whose launchers work on host memory.
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include <new>
#include <vector>

#include "cache.h"

static long g_left = -1;  // allocations that succeed before one fails; -1: all

void *operator new(size_t n) {
  if (g_left == 0) {
    g_left = -1;
    throw std::bad_alloc();
  }
  if (g_left > 0) --g_left;
  void *p = malloc(n ? n : 1);
  if (!p) abort();
  return p;
}
void operator delete(void *p) noexcept { free(p); }
void operator delete(void *p, size_t) noexcept { free(p); }

#define CHECK(x)                                                     \
  do {                                                               \
    if (!(x)) {                                                      \
      fprintf(stderr, "%s:%d: %s (%s)\n", __FILE__, __LINE__, #x, cheb_last_error()); \
      exit(1);                                                       \
    }                                                                \
  } while (0)

// Runs the call until no allocation of it fails; how many did.  check(rc) looks
// at what each run left.
template <class Call, class Check>
static int each(const char *what, Call call, Check check) {
  for (int n = 0;; ++n) {
    g_left = n;
    const int rc = call();
    const bool failed = g_left < 0;
    g_left = -1;
    if (!failed) {
      CHECK(rc == CHEB_OK);
      check(rc);
      return n;
    }
    if (rc != CHEB_E_INVAL || !strstr(cheb_last_error(), "out of host memory")) {
      fprintf(stderr, "%s, allocation %d: %d (%s)\n", what, n, rc, cheb_last_error());
      exit(1);
    }
    check(rc);
  }
}
template <class Call>
static int each(const char *what, Call call) {
  return each(what, call, [](int) {});
}

static void check_ring(int quant) {
  const std::vector<int64_t> sizes = {4096, 4096, 64, 0}, off = {0, 0, 4032, -1};
  cheb_cache *c = nullptr;
  size_t bytes = 0;
  std::vector<int64_t> at(sizes.size());
  int64_t numel = 0;
  if (quant) {
    CHECK(each("layout", [&] {
            return cheb_cache_layout_quant(2, CHEB_F32, quant, sizes.data(), 4, CHEB_LAYOUT_SLOTS,
                                           at.data(), &numel, &bytes);
          }) > 0);
  } else {
    CHECK(each("layout", [&] {
            return cheb_cache_layout(2, CHEB_F32, sizes.data(), 4, at.data(), &numel, nullptr,
                                     &bytes);
          }) > 0);
    CHECK(each("bytes", [&] {
            return cheb_cache_arena_bytes(2, CHEB_F32, sizes.data(), 4, &bytes, nullptr);
          }) > 0);
    CHECK(each("bytes", [&] {
            return cheb_cache_arena_bytes_ex(2, CHEB_F32, sizes.data(), 4, CHEB_LAYOUT_SLOTS,
                                             &bytes);
          }) > 0);
  }
  char *arena = static_cast<char *>(aligned_alloc(256, (bytes + 255) / 256 * 256));
  CHECK(each("create", [&] {
          return quant ? cheb_cache_create_quant(&c, 2, CHEB_F32, quant, sizes.data(), 4,
                                                 CHEB_LAYOUT_SLOTS, arena, bytes)
                       : cheb_cache_create_ex(&c, 2, CHEB_F32, sizes.data(), 4, CHEB_LAYOUT_SLOTS,
                                              arena, bytes);
        }) > 0);
  float *f = static_cast<float *>(aligned_alloc(16, 4096 * 4));
  for (int i = 0; i < 4096; ++i) f[i] = float(i % 7);
  const void *src[4] = {f, f, f, nullptr};
  for (int t = 0; t < 3 && quant; ++t) {
    CHECK(each("push", [&] { return cheb_cache_push(c, double(t), src, nullptr); },
               [&](int rc) {
                 double held[8];
                 int32_t count = 0;
                 CHECK(cheb_cache_history(c, held, &count) == CHEB_OK);
                 CHECK(count == (t < 2 ? t + (rc == CHEB_OK) : 2));
               }) > 0);
  }
  if (quant) {
    const double w[2] = {1.0, 2.0};
    float *y = static_cast<float *>(aligned_alloc(16, 4096 * 4));
    CHECK(each("residual", [&] {
            return cheb_residual_apply(c, w, off.data(), 4096, f, y, nullptr);
          }) > 0);
    free(y);
  }
  CHECK(cheb_cache_destroy(c) == CHEB_OK);
  free(f);
  free(arena);
}

static void check_table() {
  cheb_table *t = nullptr;
  double x[12];
  uint8_t mask[12];
  for (int i = 0; i < 12; ++i) {
    x[i] = 12.0 - i;
    mask[i] = i % 3 == 0;
  }
  CHECK(each("table", [&] {
          return cheb_table_build(&t, 12, 1, 1, 3, 3, x, CHEB_SHORT_FULL);
        }) > 0);
  char path[] = "/tmp/cheb_alloc_check_XXXXXX";
  const int fd = mkstemp(path);
  CHECK(fd >= 0 && cheb_table_save(t, path) == CHEB_OK);
  CHECK(cheb_table_destroy(t) == CHEB_OK);
  CHECK(each("load", [&] { return cheb_table_load(&t, path); }) > 0);
  CHECK(cheb_table_destroy(t) == CHEB_OK);
  remove(path);
  CHECK(each("mask", [&] {
          return cheb_table_build_mask(&t, 12, mask, 3, x, CHEB_SHORT_FULL);
        }) > 0);
  CHECK(cheb_table_destroy(t) == CHEB_OK);
}

int main() {
  check_ring(CHEB_QUANT_MXINT8);
  check_ring(CHEB_QUANT_NONE);
  check_table();
  printf("alloc ok\n");
  return 0;
}
