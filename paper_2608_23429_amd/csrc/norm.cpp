// The residual's addition and the norm that follows it: argument checks and
// sources of cheb_add_norm and cheb_residual_norm.  (Paper, Section 3.1, block
// equation: module outputs are added to the residual stream; Section 3.3: on a
// skipped step their predictions are.)
#include <float.h>
#include <math.h>

#include "cache.h"

using namespace cheb;

namespace {

struct Span {
  uintptr_t at = 0, bytes = 0;
  bool meets(const Span &o) const {
    return bytes && o.bytes && at < o.at + o.bytes && o.at < at + bytes;
  }
};

Span span(const void *p, int64_t bytes) {
  return p ? Span{reinterpret_cast<uintptr_t>(p), uintptr_t(bytes)} : Span{};
}

bool aligned(const void *p, int bytes) {
  return reinterpret_cast<uintptr_t>(p) % uintptr_t(bytes) == 0;
}

int64_t scale_bytes(const cheb_norm &n) {
  if (n.out_format == CHEB_OUT_MXFP8) return n.rows * ((n.dim + 31) / 32);
  return n.out_format == CHEB_OUT_FP8_ROW ? n.rows * 4 : 0;
}

// The counts and choices, which the sources' checks build on.
int check_shape(const cheb_norm *n) {
  if (!n) return fail(CHEB_E_INVAL, "norm is NULL");
  if (n->kind != CHEB_NORM_RMS && n->kind != CHEB_NORM_LAYER)
    return fail(CHEB_E_INVAL, "unknown norm %d", n->kind);
  if (!valid_dtype(n->x_dtype)) return fail(CHEB_E_DTYPE, "unknown dtype %d", n->x_dtype);
  if (!valid_dtype(n->out_format) && n->out_format != CHEB_OUT_MXFP8 &&
      n->out_format != CHEB_OUT_FP8_ROW)
    return fail(CHEB_E_DTYPE, "unknown output format %d", n->out_format);
  if (n->rows < 0 || n->rows >= int64_t(1) << 26)
    return fail(CHEB_E_INVAL, "rows %lld outside 0..2^26 - 1", (long long)n->rows);
  if (n->dim < 1 || n->dim > CHEB_MAX_NORM_DIM)
    return fail(CHEB_E_INVAL, "dim %lld outside 1..%d", (long long)n->dim, CHEB_MAX_NORM_DIM);
  if (n->rows * n->dim >= int64_t(1) << 34) return fail(CHEB_E_INVAL, "too many elements");
  if (!(n->eps >= 0.0) || !isfinite(n->eps))
    return fail(CHEB_E_INVAL, "eps %g must be finite and not negative", n->eps);
  if ((n->gain || n->shift) && n->rows_per_group < 1)
    return fail(CHEB_E_INVAL, "rows_per_group must be at least 1");
  return CHEB_OK;
}

// The buffers; `in` are the sources' places.
int check_buffers(const cheb_norm &n, const Span *in, int n_in) {
  const bool coded = !valid_dtype(n.out_format);
  if (!n.y) return fail(CHEB_E_INVAL, "y is NULL");
  if (coded && !n.y_scale) return fail(CHEB_E_INVAL, "y_scale is NULL");
  if (!coded && n.y_scale)
    return fail(CHEB_E_INVAL, "y_scale is given, but y holds a storage type");
  const int xb = elem_bytes(n.x_dtype), yb = coded ? 1 : elem_bytes(n.out_format);
  if (!aligned(n.x_in, xb) || !aligned(n.x_out, xb) || !aligned(n.y, yb) ||
      !aligned(n.gain, 4) || !aligned(n.shift, 4) ||
      (n.out_format == CHEB_OUT_FP8_ROW && !aligned(n.y_scale, 4)))
    return fail(CHEB_E_ALIGN, "x_in, x_out, y, y_scale, gain or shift is not aligned");
  const int64_t numel = n.rows * n.dim;
  const bool one = n.rows_per_group >= n.rows;
  const int64_t groups =
      n.gain || n.shift ? (one ? 1 : (n.rows - 1) / n.rows_per_group + 1) : 0;
  const Span x = span(n.x_in, numel * xb), mod[2] = {span(n.gain, groups * n.dim * 4),
                                                     span(n.shift, groups * n.dim * 4)};
  const Span out[3] = {span(n.x_out, numel * xb), span(n.y, numel * yb),
                       span(n.y_scale, scale_bytes(n))};
  static const char *const kName[3] = {"x_out", "y", "y_scale"};
  for (int o = 0; o < 3; ++o) {
    if (out[o].meets(x) && !(o == 0 && n.x_out == n.x_in))
      return fail(CHEB_E_INVAL, "%s overlaps x_in", kName[o]);
    if (out[o].meets(mod[0]) || out[o].meets(mod[1]))
      return fail(CHEB_E_INVAL, "%s overlaps gain or shift", kName[o]);
    for (int k = 0; k < n_in; ++k)
      if (out[o].meets(in[k])) return fail(CHEB_E_INVAL, "%s overlaps a source", kName[o]);
    for (int p = 0; p < o; ++p)
      if (out[o].meets(out[p])) return fail(CHEB_E_INVAL, "%s overlaps %s", kName[o], kName[p]);
  }
  return CHEB_OK;
}

}  // namespace

extern "C" {

int cheb_add_norm(const void *const *src, int32_t n_src, const double *w, int32_t dtype,
                  const cheb_norm *norm, void *stream) {
  int rc = check_shape(norm);
  if (rc != CHEB_OK) return rc;
  if (n_src < 0 || n_src > CHEB_MAX_SLOTS)
    return fail(CHEB_E_INVAL, "n_src %d outside 0..%d", n_src, CHEB_MAX_SLOTS);
  if (n_src > 0 && (!src || !w)) return fail(CHEB_E_INVAL, "src or w is NULL");
  if (n_src > 0 && !valid_dtype(dtype)) return fail(CHEB_E_DTYPE, "unknown dtype %d", dtype);
  if (n_src == 0 && !norm->x_in) return fail(CHEB_E_INVAL, "neither sources nor x_in");
  for (int k = 0; k < n_src; ++k)
    if (!isfinite(w[k])) return fail(CHEB_E_NONFINITE, "w[%d] is not finite", k);
  if (norm->rows == 0) return ok();
  NormSources from;
  from.n = n_src;
  if (n_src > 0) from.dtype = dtype;
  Span in[CHEB_MAX_SLOTS];
  for (int k = 0; k < n_src; ++k) {
    if (!src[k]) return fail(CHEB_E_INVAL, "src[%d] is NULL", k);
    if (!aligned(src[k], elem_bytes(dtype)))
      return fail(CHEB_E_ALIGN, "src[%d] is not aligned", k);
    in[k] = span(src[k], norm->rows * norm->dim * elem_bytes(dtype));
    from.base[k] = src[k];
    from.w[k] = w[k];
  }
  rc = check_buffers(*norm, in, n_src);
  if (rc != CHEB_OK) return rc;
  return launch_norm(from, *norm, static_cast<hipStream_t>(stream));
}

int cheb_residual_norm(cheb_cache *c, const double *w, int32_t seg, int64_t first,
                       const cheb_norm *norm, void *stream) {
  if (!c || !w) return fail(CHEB_E_INVAL, "cache or w is NULL");
  int rc = check_shape(norm);
  if (rc != CHEB_OK) return rc;
  if (seg < 0 || size_t(seg) >= c->seg_numel.size())
    return fail(CHEB_E_INVAL, "segment %d out of range", seg);
  if (first < 0 || first > c->seg_numel[size_t(seg)] ||
      norm->rows * norm->dim > c->seg_numel[size_t(seg)] - first)
    return fail(CHEB_E_INVAL, "the rows end past segment %d", seg);
  if (c->push_open) return fail(CHEB_E_NOTREADY, "a fused push is open");
  if (c->count < c->n_slots)
    return fail(CHEB_E_NOTREADY, "history holds %d of %d entries", c->count, c->n_slots);
  for (int32_t k = 0; k < c->n_slots; ++k) {
    if (!isfinite(w[k])) return fail(CHEB_E_NONFINITE, "w[%d] is not finite", k);
    if (c->coded && fabs(w[k]) > double(FLT_MAX))
      return fail(CHEB_E_NONFINITE, "weight %d (%.17g) overflows fp32", k, w[k]);
  }
  if (norm->rows == 0) return ok();
  const Span arena = span(c->arena, int64_t(c->arena_bytes));
  rc = check_buffers(*norm, &arena, 1);
  if (rc != CHEB_OK) return rc;
  NormSources from;
  from.n = c->n_slots;
  from.dtype = c->dtype;
  from.quant = c->quant;
  from.super_vecs = c->super_vecs;
  from.place = c->place;
  from.first = c->seg_offset[size_t(seg)] + first;
  for (int32_t k = 0; k < c->n_slots; ++k) {
    const int32_t slot = c->slot_of_age(k);
    from.w[k] = w[k];
    if (c->coded)
      from.src[k] = {c->place.codes + size_t(slot) * c->place.code_lane,
                     c->place.scales + size_t(slot) * c->place.scale_lane};
    else
      from.base[k] = c->slot_ptr(slot);
  }
  return launch_norm(from, *norm, static_cast<hipStream_t>(stream));
}

}  // extern "C"
