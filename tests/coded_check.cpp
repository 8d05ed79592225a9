// Histories of 8-bit entries on the host: the ring, the layout of codes and
// scales in the arena, the residual plan and the refusals, with launchers that
// work on host memory.  Every byte they touch lies in an arena of exactly the
// size the library asks for, so AddressSanitizer sees a place out of bounds.
#include <math.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include <random>
#include <vector>

#include "cache.h"

#define CHECK(x)                                                     \
  do {                                                               \
    if (!(x)) {                                                      \
      fprintf(stderr, "%s:%d: %s (%s)\n", __FILE__, __LINE__, #x, cheb_last_error()); \
      exit(1);                                                       \
    }                                                                \
  } while (0)

static int g_stores = 0, g_store_fails = 0, g_residuals = 0;

namespace cheb {

// A code is the element itself (whole, below 128), its group's scale 1.
static char *code_at(const CodedEntry &e, const CodedPlace &p, int64_t i) {
  return const_cast<char *>(e.codes) + size_t(i / kCodedChunk) * p.code_super +
         size_t(i % kCodedChunk);
}
static char *scale_at(const CodedEntry &e, const CodedPlace &p, int64_t i) {
  const int64_t r = i % kCodedChunk;
  return const_cast<char *>(e.scales) + size_t(i / kCodedChunk) * p.scale_super +
         size_t((r >> 12) * 128 + (r >> 5 & 15) * 8 + (r >> 9 & 7));
}

int launch_store(int, int dtype, const CodedEntry &to, const CodedPlace &place, GatherSeg *segs,
                 int n_segs, hipStream_t) {
  if (dtype != CHEB_F32) return fail(CHEB_E_INVAL, "test stores fp32");
  if (g_store_fails > 0) {
    --g_store_fails;
    return fail(CHEB_E_HIP, "refused");
  }
  for (int s = 0; s < n_segs; ++s) {
    if (segs[s].dst_offset % kCodedBlock != 0) return fail(CHEB_E_INVAL, "inside a block");
    const int64_t whole = (segs[s].numel + kCodedBlock - 1) / kCodedBlock * kCodedBlock;
    for (int64_t i = 0; i < whole; ++i) {
      const float v = i < segs[s].numel ? static_cast<const float *>(segs[s].src)[i] : 0.0f;
      *code_at(to, place, segs[s].dst_offset + i) = char(int(v));
      *scale_at(to, place, segs[s].dst_offset + i) = 1;
    }
  }
  ++g_stores;
  return ok();
}

int launch_predict_coded(int, int, const CodedEntry *src, int n, const double *w, int n_out,
                         void *const *out, int64_t numel, const CodedPlace &place, hipStream_t) {
  for (int m = 0; m < n_out; ++m)
    for (int64_t i = 0; i < numel; ++i) {
      double sum = 0;
      for (int k = 0; k < n; ++k)
        sum += w[m * n + k] * double(*code_at(src[k], place, i)) *
               double(*scale_at(src[k], place, i));
      static_cast<float *>(out[m])[i] = float(sum);
    }
  return ok();
}

int launch_residual_coded(int, int n, const CodedEntry *src, const double *w,
                          const int64_t *delta, int n_delta, const ResidualInterval *iv, int n_iv,
                          const float *x_in, float *x_out, const CodedPlace &place, hipStream_t) {
  if (n_iv < 1 || n_iv > kMaxResIntervals || n_delta > residual_max_cover())
    return fail(CHEB_E_INVAL, "residual tables are malformed");
  for (int i = 0; i < n_iv; delta += iv[i].ncover, ++i)
    for (int64_t j = iv[i].vec_begin * 8; j < (iv[i].vec_begin + iv[i].n_vec) * 8; ++j) {
      double sum = x_in ? double(x_in[j]) : 0.0;
      for (int c = 0; c < iv[i].ncover; ++c)
        for (int k = 0; k < n; ++k)
          sum += w[k] * double(*code_at(src[k], place, delta[c] * 8 + j)) *
                 double(*scale_at(src[k], place, delta[c] * 8 + j));
      x_out[j] = float(sum);
    }
  ++g_residuals;
  return ok();
}

}  // namespace cheb

namespace {

std::mt19937 g_rng(2025);

struct Ring {
  cheb_cache *c = nullptr;
  std::vector<int64_t> sizes, offset;
  int64_t numel = 0;
  void *arena = nullptr;
  std::vector<std::vector<std::vector<float>>> steps;

  Ring(int n, int layout, std::vector<int64_t> seg) : sizes(seg), offset(seg.size()) {
    size_t bytes = 0;
    CHECK(cheb_cache_layout_quant(n, CHEB_F32, CHEB_QUANT_MXINT8, sizes.data(),
                                  int(sizes.size()), layout, offset.data(), &numel,
                                  &bytes) == CHEB_OK);
    arena = aligned_alloc(256, (bytes + 255) / 256 * 256);
    CHECK(cheb_cache_create_quant(&c, n, CHEB_F32, CHEB_QUANT_MXINT8, sizes.data(),
                                  int(sizes.size()), layout, arena, bytes) == CHEB_OK);
  }
  ~Ring() {
    cheb_cache_destroy(c);
    free(arena);
  }
  int push(double t) {
    std::vector<std::vector<float>> segs;
    std::vector<const void *> src;
    std::uniform_int_distribution<int> code(-100, 100);
    for (int64_t n : sizes) {
      // 16-byte aligned, as the call asks; a spare element keeps empty ones apart
      segs.emplace_back(size_t(n) + 1);
      for (float &v : segs.back()) v = float(code(g_rng));
    }
    for (auto &s : segs) src.push_back(s.data());
    const int rc = cheb_cache_push(c, t, src.data(), nullptr);
    if (rc == CHEB_OK) steps.push_back(std::move(segs));
    return rc;
  }
  float held(int back, size_t s, int64_t i) const {
    return steps[steps.size() - 1 - size_t(back)][s][size_t(i)];
  }
};

void check_ring(int n, int layout, std::vector<int64_t> sizes) {
  Ring r(n, layout, sizes);
  for (int k = 0; k < n + 2; ++k) CHECK(r.push(double(k)) == CHEB_OK);
  for (size_t s = 0; s < sizes.size(); ++s) CHECK(r.offset[s] % 4096 == 0);
  float *out = static_cast<float *>(aligned_alloc(16, size_t(r.numel) * 4 + 16));
  for (int idx = 0; idx < n; ++idx) {
    CHECK(cheb_cache_read(r.c, idx, out, nullptr) == CHEB_OK);
    for (size_t s = 0; s < sizes.size(); ++s)
      for (int64_t i = 0; i < (sizes[s] + 4095) / 4096 * 4096; ++i)
        CHECK(out[r.offset[s] + i] == (i < sizes[s] ? r.held(n - 1 - idx, s, i) : 0.0f));
  }
  std::vector<double> w(size_t(2 * n));
  for (size_t i = 0; i < w.size(); ++i) w[i] = double(i) - 1.5;
  float *more = static_cast<float *>(aligned_alloc(16, size_t(r.numel) * 4 + 16));
  void *outs[2] = {out, more};
  CHECK(cheb_extrapolate_multi(r.c, w.data(), 2, outs, nullptr) == CHEB_OK);
  for (int m = 0; m < 2; ++m)
    for (size_t s = 0; s < sizes.size(); ++s)
      for (int64_t i = 0; i < sizes[s]; ++i) {
        double sum = 0;
        for (int k = 0; k < n; ++k) sum += w[size_t(m * n + k)] * double(r.held(n - 1 - k, s, i));
        CHECK((m ? more : out)[r.offset[s] + i] == float(sum));
      }
  free(out);
  free(more);
}

void check_residual(int n, int layout, std::vector<int64_t> sizes, std::vector<int64_t> off,
                    int64_t numel, int launches) {
  Ring r(n, layout, sizes);
  for (int k = 0; k < n; ++k) CHECK(r.push(double(k)) == CHEB_OK);
  std::vector<double> w;
  for (int k = 0; k < n; ++k) w.push_back(1.25 * k - 2.0);
  float *x = static_cast<float *>(aligned_alloc(16, size_t(numel) * 4));
  float *y = static_cast<float *>(aligned_alloc(16, size_t(numel) * 4));
  for (int64_t i = 0; i < numel; ++i) x[i] = float(i % 17);
  g_residuals = 0;
  CHECK(cheb_residual_apply(r.c, w.data(), off.data(), numel, x, y, nullptr) == CHEB_OK);
  CHECK(g_residuals == launches);
  for (int64_t j = 0; j < numel; ++j) {
    double sum = x[j];
    for (size_t s = 0; s < sizes.size(); ++s)
      if (off[s] >= 0 && j >= off[s] && j < off[s] + sizes[s])
        for (int k = 0; k < n; ++k) sum += w[size_t(k)] * double(r.held(n - 1 - k, s, j - off[s]));
    CHECK(fabs(double(y[j]) - sum) <= 1e-6 * (1.0 + fabs(sum)));
  }
  // Offsets and sizes are multiples of 8, weights of fp32's range.
  std::vector<int64_t> bad = off;
  bad[0] = 4;
  CHECK(cheb_residual_apply(r.c, w.data(), bad.data(), numel, x, y, nullptr) == CHEB_E_ALIGN);
  CHECK(cheb_residual_apply(r.c, w.data(), off.data(), numel - 4, x, y, nullptr) == CHEB_E_INVAL);
  w[0] = 1e39;
  CHECK(cheb_residual_apply(r.c, w.data(), off.data(), numel, x, y, nullptr) ==
        CHEB_E_NONFINITE);
  free(x);
  free(y);
}

void check_refusals() {
  const int64_t seg[2] = {100, 5000};
  int64_t off[2] = {-1, -1}, numel = -1;
  size_t bytes = 0;
  cheb_cache *c = nullptr;
  const int I8 = CHEB_QUANT_MXINT8, SL = CHEB_LAYOUT_SLOTS;
  CHECK(cheb_cache_layout_quant(2, CHEB_BF16, I8, seg, 2, SL, off, &numel, &bytes) == CHEB_OK);
  CHECK(off[0] == 0 && off[1] == 4096 && numel == 4096 + 8192);
  CHECK(bytes >= 2 * size_t(numel) / 32 * 33 && bytes < 2 * size_t(numel) / 32 * 33 + 1024);
  CHECK(cheb_cache_layout_quant(2, CHEB_BF16, I8, seg, 2, SL, nullptr, nullptr, nullptr) ==
        CHEB_OK);
  CHECK(cheb_cache_layout_quant(2, 9, I8, seg, 2, SL, off, &numel, &bytes) == CHEB_E_DTYPE);
  for (int q : {int(CHEB_QUANT_NONE), 3, -1})
    CHECK(cheb_cache_layout_quant(2, CHEB_BF16, q, seg, 2, SL, off, &numel, &bytes) ==
          CHEB_E_INVAL);
  CHECK(cheb_cache_layout_quant(2, CHEB_BF16, I8, seg, 2, 7, off, &numel, &bytes) ==
        CHEB_E_INVAL);
  for (int n : {0, 9, -1})
    CHECK(cheb_cache_layout_quant(n, CHEB_BF16, I8, seg, 2, SL, off, &numel, &bytes) ==
          CHEB_E_INVAL);
  CHECK(cheb_cache_layout_quant(2, CHEB_BF16, I8, seg, 0, SL, off, &numel, &bytes) ==
        CHEB_E_INVAL);
  CHECK(cheb_cache_layout_quant(2, CHEB_BF16, I8, nullptr, 2, SL, off, &numel, &bytes) ==
        CHEB_E_INVAL);
  for (int64_t n : {int64_t(-1), int64_t(1) << 40, INT64_MAX}) {
    const int64_t one[1] = {n};
    CHECK(cheb_cache_layout_quant(2, CHEB_BF16, I8, one, 1, SL, off, &numel, &bytes) ==
          CHEB_E_INVAL);
  }
  char *arena = static_cast<char *>(aligned_alloc(256, (bytes + 511) / 256 * 256));
  CHECK(cheb_cache_create_quant(nullptr, 2, CHEB_BF16, I8, seg, 2, SL, arena, bytes) ==
        CHEB_E_INVAL);
  CHECK(cheb_cache_create_quant(&c, 2, CHEB_BF16, I8, seg, 2, SL, nullptr, bytes) ==
        CHEB_E_INVAL);
  CHECK(cheb_cache_create_quant(&c, 2, CHEB_BF16, I8, seg, 2, SL, arena + 16, bytes) ==
        CHEB_E_ALIGN);
  CHECK(cheb_cache_create_quant(&c, 2, CHEB_BF16, I8, seg, 2, SL, arena, bytes - 1) ==
        CHEB_E_MISMATCH);
  CHECK(c == nullptr);
  free(arena);

  Ring r(2, SL, {100, 5000});
  int32_t quant = -1;
  CHECK(cheb_cache_quant(r.c, &quant) == CHEB_OK && quant == I8);
  CHECK(cheb_cache_quant(nullptr, &quant) == CHEB_E_INVAL);
  CHECK(cheb_cache_quant(r.c, nullptr) == CHEB_E_INVAL);
  float *out = static_cast<float *>(aligned_alloc(16, size_t(r.numel) * 4 + 64));
  void *p = nullptr;
  const double w[2] = {1.0, 2.0};
  CHECK(cheb_cache_read(r.c, 0, out, nullptr) == CHEB_E_INVAL);          // empty
  CHECK(cheb_extrapolate(r.c, w, out, nullptr) == CHEB_E_NOTREADY);
  CHECK(r.push(0.0) == CHEB_OK && r.push(1.0) == CHEB_OK);
  CHECK(r.push(1.0) == CHEB_E_DUPNODE);
  CHECK(cheb_cache_begin_push(r.c, &p) == CHEB_E_INVAL);
  CHECK(cheb_cache_entry(r.c, 0, &p) == CHEB_E_INVAL);
  CHECK(cheb_cache_geometry(r.c, nullptr, nullptr, nullptr) == CHEB_E_INVAL);
  CHECK(cheb_cache_read(nullptr, 0, out, nullptr) == CHEB_E_INVAL);
  CHECK(cheb_cache_read(r.c, 2, out, nullptr) == CHEB_E_INVAL);
  CHECK(cheb_cache_read(r.c, -1, out, nullptr) == CHEB_E_INVAL);
  CHECK(cheb_cache_read(r.c, 0, nullptr, nullptr) == CHEB_E_INVAL);
  CHECK(cheb_cache_read(r.c, 0, out + 1, nullptr) == CHEB_E_ALIGN);
  CHECK(cheb_cache_read(r.c, 0, r.arena, nullptr) == CHEB_E_INVAL);
  CHECK(cheb_extrapolate(r.c, w, out, nullptr) == CHEB_OK);
  CHECK(cheb_extrapolate(r.c, w, nullptr, nullptr) == CHEB_E_INVAL);
  CHECK(cheb_extrapolate(r.c, w, out + 1, nullptr) == CHEB_E_ALIGN);
  CHECK(cheb_extrapolate(r.c, w, r.arena, nullptr) == CHEB_E_INVAL);
  void *same[2] = {out, out + 4};
  const double ww[4] = {1, 2, 3, 4}, nan[2] = {1.0, NAN};
  CHECK(cheb_extrapolate_multi(r.c, ww, 2, same, nullptr) == CHEB_E_INVAL);
  CHECK(cheb_extrapolate(r.c, nan, out, nullptr) == CHEB_E_NONFINITE);
  // A push that fails leaves the other entry, and no half-written one.
  g_store_fails = 1;
  CHECK(r.push(2.0) == CHEB_E_HIP);
  int32_t count = 0;
  double t[8];
  CHECK(cheb_cache_history(r.c, t, &count) == CHEB_OK && count == 1 && t[0] == 1.0);
  CHECK(cheb_cache_reset(r.c) == CHEB_OK);
  CHECK(cheb_cache_read(r.c, 0, out, nullptr) == CHEB_E_INVAL);
  free(out);

  // A plain cache has the format "none" and is read through the ordinary
  // combination.
  const int64_t one[1] = {64};
  CHECK(cheb_cache_arena_bytes(1, CHEB_F32, one, 1, &bytes, nullptr) == CHEB_OK);
  void *plain = aligned_alloc(256, (bytes + 255) / 256 * 256);
  CHECK(cheb_cache_create(&c, 1, CHEB_F32, one, 1, plain, bytes) == CHEB_OK);
  CHECK(cheb_cache_quant(c, &quant) == CHEB_OK && quant == CHEB_QUANT_NONE);
  CHECK(cheb_cache_begin_push(c, &p) == CHEB_OK);
  CHECK(cheb_cache_read(c, 0, plain, nullptr) == CHEB_E_NOTREADY);
  CHECK(cheb_cache_commit(c, 0.0) == CHEB_OK);
  CHECK(cheb_cache_read(c, 0, plain, nullptr) == CHEB_E_INVAL);
  CHECK(cheb_cache_read(c, 1, plain, nullptr) == CHEB_E_INVAL);
  CHECK(cheb_cache_destroy(c) == CHEB_OK);
  free(plain);
}

}  // namespace

int main() {
  for (int layout : {int(CHEB_LAYOUT_SLOTS), int(CHEB_LAYOUT_INTERLEAVED)}) {
    check_ring(1, layout, {1});
    check_ring(2, layout, {0, 5, 4096});
    check_ring(3, layout, {100, 0, 8192, 32769, 4095});
    check_ring(8, layout, {70000, 3});
    check_ring(2, layout, {0});
    check_residual(2, layout, {4608, 4608, 4608}, {0, 0, 0}, 4608, 1);
    check_residual(3, layout, {5760, 2664, 8424, 8424}, {2664, 0, 0, 0}, 8424, 1);
    check_residual(1, layout, {8}, {0}, 8, 1);
    std::vector<int64_t> sizes, off;
    for (int i = 0; i < 140; ++i) {
      sizes.push_back(40 + 8 * (i % 3));
      off.push_back(8 * (i % 2));
    }
    // five intervals, one of them of all 140 segments: two tables
    check_residual(2, layout, sizes, off, 64, 6);
  }
  check_refusals();
  printf("coded ok\n");
  return 0;
}
