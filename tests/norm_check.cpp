// The norm calls' host side, and rings of plain and 8-bit entries under it, on
// the CPU: a launcher that works on host memory follows every address the
// library gives it, over buffers of exactly the sizes documented, so
// AddressSanitizer sees one out of bounds.  Linked with coded_check.cpp, whose
// launchers of 8-bit entries it uses and whose checks it runs as well.
#include <math.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include <vector>

#include "cache.h"

#define CHECK(x)                                                     \
  do {                                                               \
    if (!(x)) {                                                      \
      fprintf(stderr, "%s:%d: %s (%s)\n", __FILE__, __LINE__, #x, cheb_last_error()); \
      exit(1);                                                       \
    }                                                                \
  } while (0)

int coded_check_main();

static int g_norms = 0;

namespace cheb {

// Element e of source k, fp32 entries; codes as coded_check.cpp stores them.
static double source_at(const NormSources &f, int k, int64_t e) {
  e += f.first;
  if (f.quant == CHEB_QUANT_NONE) {
    const int64_t vec = e / 4, chunk = vec / kChunkVecs;
    const char *p = static_cast<const char *>(f.base[k]) +
                    (chunk * f.super_vecs + vec % kChunkVecs) * 16;
    return double(reinterpret_cast<const float *>(p)[e % 4]);
  }
  const int64_t r = e % kCodedChunk;
  const char *code = f.src[k].codes + size_t(e / kCodedChunk) * f.place.code_super + r;
  const char *scale = f.src[k].scales + size_t(e / kCodedChunk) * f.place.scale_super +
                      ((r >> 12) * 128 + (r >> 5 & 15) * 8 + (r >> 9 & 7));
  return double(*code) * double(*scale);
}

// y = x times gain plus shift: what the rows are made of, without the norm.
int launch_norm(const NormSources &f, const cheb_norm &n, hipStream_t) {
  ++g_norms;
  for (int64_t r = 0; r < n.rows; ++r)
    for (int64_t i = 0; i < n.dim; ++i) {
      const int64_t e = r * n.dim + i;
      double x = n.x_in ? double(static_cast<const float *>(n.x_in)[e]) : 0.0;
      for (int k = 0; k < f.n; ++k) x += f.w[k] * source_at(f, k, e);
      if (n.x_out) static_cast<float *>(n.x_out)[e] = float(x);
      const int64_t g = n.gain || n.shift ? r / n.rows_per_group * n.dim + i : 0;
      if (n.gain) x *= double(n.gain[g]);
      if (n.shift) x += double(n.shift[g]);
      static_cast<float *>(n.y)[e] = float(x);
    }
  return ok();
}


}  // namespace cheb

namespace {

std::vector<float> numbers(int64_t n, int from) {
  std::vector<float> v(static_cast<size_t>(n));
  for (size_t i = 0; i < v.size(); ++i) v[i] = float(int((i * 7 + size_t(from) * 13) % 61) - 30);
  return v;
}

struct Rows {
  std::vector<float> x, x_out, gain, shift, y;
  cheb_norm n;
  Rows(int64_t rows, int64_t dim, int64_t per_group)
      : x(numbers(rows * dim, 3)), x_out(x.size()), y(x.size()) {
    const int64_t groups = (rows + per_group - 1) / per_group;
    gain = numbers(groups * dim, 5);
    shift = numbers(groups * dim, 6);
    memset(&n, 0, sizeof n);
    n.rows = rows;
    n.dim = dim;
    n.eps = 1e-6;
    n.x_in = x.data();
    n.x_out = x_out.data();
    n.gain = gain.data();
    n.shift = shift.data();
    n.rows_per_group = per_group;
    n.y = y.data();
    n.kind = CHEB_NORM_RMS;
    n.x_dtype = CHEB_F32;
    n.out_format = CHEB_F32;
  }
  void check(const std::vector<double> &sum) const {
    for (int64_t e = 0; e < n.rows * n.dim; ++e) {
      const double want = double(x[size_t(e)]) + sum[size_t(e)];
      const int64_t g = e / n.dim / n.rows_per_group * n.dim + e % n.dim;
      CHECK(x_out[size_t(e)] == float(want));
      CHECK(y[size_t(e)] == float(want * double(gain[size_t(g)]) + double(shift[size_t(g)])));
    }
  }
};

// Rows from element `first` of the middle tensor of a ring whose slots have
// gone round.
void check_ring(int n, int quant, int layout, int64_t rows, int64_t dim, int64_t first,
                int64_t per_group) {
  const std::vector<int64_t> sizes = {70, first + rows * dim + 5, 9};
  size_t bytes = 0;
  cheb_cache *c = nullptr;
  char *arena = nullptr;
  if (quant == CHEB_QUANT_NONE) {
    // Entries of a plain ring are recorded by fused pushes (contiguous slots).
    CHECK(layout == CHEB_LAYOUT_SLOTS);
    CHECK(cheb_cache_arena_bytes(n, CHEB_F32, sizes.data(), 3, &bytes, nullptr) == CHEB_OK);
    arena = static_cast<char *>(aligned_alloc(256, (bytes + 255) / 256 * 256));
    CHECK(cheb_cache_create(&c, n, CHEB_F32, sizes.data(), 3, arena, bytes) == CHEB_OK);
  } else {
    CHECK(cheb_cache_layout_quant(n, CHEB_F32, quant, sizes.data(), 3, layout, nullptr, nullptr,
                                  &bytes) == CHEB_OK);
    arena = static_cast<char *>(aligned_alloc(256, (bytes + 255) / 256 * 256));
    CHECK(cheb_cache_create_quant(&c, n, CHEB_F32, quant, sizes.data(), 3, layout, arena, bytes) ==
          CHEB_OK);
  }
  std::vector<std::vector<float>> steps;
  for (int t = 0; t < n + 2; ++t) {
    steps.push_back(numbers(sizes[1], t));
    if (quant == CHEB_QUANT_NONE) {
      void *slot = nullptr;
      int64_t at = 0;
      CHECK(cheb_cache_begin_push(c, &slot) == CHEB_OK);
      CHECK(cheb_cache_segment_offset(c, 1, &at) == CHEB_OK);
      memcpy(static_cast<float *>(slot) + at, steps.back().data(), size_t(sizes[1]) * 4);
      CHECK(cheb_cache_commit(c, double(t)) == CHEB_OK);
    } else {
      const std::vector<float> a = numbers(sizes[0], 90), b = numbers(sizes[2] + 3, 91);
      const void *src[3] = {a.data(), steps.back().data(), b.data()};
      CHECK(cheb_cache_push(c, double(t), src, nullptr) == CHEB_OK);
    }
  }
  std::vector<double> w;
  for (int k = 0; k < n; ++k) w.push_back(0.25 * (k + 1));
  std::vector<double> sum(size_t(rows * dim), 0.0);
  for (int k = 0; k < n; ++k)
    for (size_t e = 0; e < sum.size(); ++e)
      sum[e] += w[size_t(k)] * double(steps[size_t(2 + k)][size_t(first) + e]);
  Rows r(rows, dim, per_group);
  CHECK(cheb_residual_norm(c, w.data(), 1, first, &r.n, nullptr) == CHEB_OK);
  r.check(sum);
  // Past the tensor, and weights that are not of the entries' range.
  CHECK(cheb_residual_norm(c, w.data(), 1, first + 6, &r.n, nullptr) == CHEB_E_INVAL);
  w[0] = 1e39;
  const int rc = cheb_residual_norm(c, w.data(), 1, first, &r.n, nullptr);
  CHECK(rc == (quant == CHEB_QUANT_NONE ? CHEB_OK : CHEB_E_NONFINITE));
  CHECK(cheb_cache_destroy(c) == CHEB_OK);
  free(arena);
}

void check_sources(int n, int64_t rows, int64_t dim, int64_t per_group) {
  std::vector<std::vector<float>> src;
  std::vector<const void *> p;
  std::vector<double> w, sum(size_t(rows * dim), 0.0);
  for (int k = 0; k < n; ++k) {
    src.push_back(numbers(rows * dim, k));
    w.push_back(0.5 * k - 1.0);
    for (size_t e = 0; e < sum.size(); ++e) sum[e] += w.back() * double(src.back()[e]);
  }
  for (auto &s : src) p.push_back(s.data());
  Rows r(rows, dim, per_group);
  CHECK(cheb_add_norm(n ? p.data() : nullptr, n, n ? w.data() : nullptr, CHEB_F32, &r.n,
                      nullptr) == CHEB_OK);
  r.check(sum);
  // One group for rows that do not fill it, and 2^62 rows to a group.
  if (per_group >= rows) {
    r.n.rows_per_group = int64_t(1) << 62;
    CHECK(cheb_add_norm(p.data(), n, w.data(), CHEB_F32, &r.n, nullptr) == CHEB_OK);
  }
}

}  // namespace

int main() {
  if (coded_check_main() != 0) return 1;
  for (int n : {0, 1, 8})
    for (int64_t per_group : {int64_t(1), int64_t(2), int64_t(3), int64_t(7), int64_t(100)}) {
      check_sources(n, 7, 5, per_group);
      check_sources(n, 1, 1, per_group);
    }
  for (int64_t per_group : {int64_t(1), int64_t(4), int64_t(1000)})
    for (int64_t first : {int64_t(0), int64_t(3)}) {
      check_ring(1, CHEB_QUANT_NONE, CHEB_LAYOUT_SLOTS, 3, 33, first, per_group);
      check_ring(3, CHEB_QUANT_NONE, CHEB_LAYOUT_SLOTS, 100, 333, first, per_group);
      for (int layout : {int(CHEB_LAYOUT_SLOTS), int(CHEB_LAYOUT_INTERLEAVED)}) {
        check_ring(1, CHEB_QUANT_MXINT8, layout, 3, 33, first, per_group);
        check_ring(3, CHEB_QUANT_MXINT8, layout, 200, 333, first, per_group);
      }
    }
  CHECK(g_norms > 0);
  printf("norm ok\n");
  return 0;
}
