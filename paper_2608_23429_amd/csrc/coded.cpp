// Histories of 8-bit entries: the layout of codes and scales in the arena,
// and what such a ring does in place of a plain one (paper, Section 3.3: the
// history buffer H; the entries' format is this library's).
#include <float.h>
#include <math.h>
#include <string.h>

#include <memory>
#include <new>
#include <vector>

#include "cache.h"

using namespace cheb;

namespace {

constexpr size_t kPlaneAlign = 256;

size_t up(size_t v, size_t to) { return (v + to - 1) / to * to; }

// Where everything lies, from an arena at address 0, and the bytes that takes.
// Slots: a slot's codes, then its scales.  Interleaved: the entries' chunks of
// codes in turn from the first kLaneAlign boundary, then their chunks of
// scales.
struct Layout {
  std::vector<int64_t> offset;
  int64_t slot_numel = 0;
  size_t codes = 0, scales = 0;  // from the region's start
  size_t bytes = 0, slot_stride = 0;
  CodedPlace place;
};

int lay_out(int32_t n_slots, int32_t dtype, int32_t quant, const int64_t *seg_numel,
            int32_t n_segs, int32_t layout, Layout *l) {
  if (!valid_dtype(dtype)) return fail(CHEB_E_DTYPE, "unknown dtype %d", dtype);
  if (quant != CHEB_QUANT_MXINT8 && quant != CHEB_QUANT_MXFP8)
    return fail(CHEB_E_INVAL, "unknown 8-bit format %d", quant);
  if (layout != CHEB_LAYOUT_SLOTS && layout != CHEB_LAYOUT_INTERLEAVED)
    return fail(CHEB_E_INVAL, "unknown layout %d", layout);
  if (n_slots < 1 || n_slots > CHEB_MAX_SLOTS)
    return fail(CHEB_E_INVAL, "n_slots %d outside 1..%d", n_slots, CHEB_MAX_SLOTS);
  if (n_segs < 1) return fail(CHEB_E_INVAL, "n_segs must be at least 1");
  if (!seg_numel) return fail(CHEB_E_INVAL, "seg_numel is NULL");
  l->offset.assign(size_t(n_segs), 0);
  const int64_t most = kMaxVecs * elems_per_vec(dtype);
  int64_t pos = 0;
  for (int32_t s = 0; s < n_segs; ++s) {
    if (seg_numel[s] < 0) return fail(CHEB_E_INVAL, "seg_numel[%d] is negative", s);
    if (seg_numel[s] >= most) return fail(CHEB_E_INVAL, "cache slot too large");
    l->offset[size_t(s)] = pos;
    pos += (seg_numel[s] + kCodedBlock - 1) / kCodedBlock * kCodedBlock;
    if (pos >= most) return fail(CHEB_E_INVAL, "cache slot too large");
  }
  l->slot_numel = pos;
  const size_t n = size_t(n_slots);
  if (layout == CHEB_LAYOUT_SLOTS) {
    const size_t codes = size_t(pos), scales = size_t(pos) / 32;
    l->slot_stride = up(codes + scales, kPlaneAlign);
    l->scales = codes;
    l->place.code_lane = l->place.scale_lane = l->slot_stride;
    l->place.code_super = size_t(kCodedChunk);
    l->place.scale_super = size_t(kCodedChunkScales);
    l->bytes = l->slot_stride * n;
  } else {
    const size_t chunks = (size_t(pos) + size_t(kCodedChunk) - 1) / size_t(kCodedChunk);
    l->scales = chunks * n * size_t(kCodedChunk);
    l->place.code_lane = size_t(kCodedChunk);
    l->place.scale_lane = size_t(kCodedChunkScales);
    l->place.code_super = n * size_t(kCodedChunk);
    l->place.scale_super = n * size_t(kCodedChunkScales);
    l->bytes = l->scales + chunks * n * size_t(kCodedChunkScales) + kLaneAlign;
  }
  return CHEB_OK;
}

CodedEntry entry_of(const cheb_cache *c, int32_t slot) {
  return {c->place.codes + size_t(slot) * c->place.code_lane,
          c->place.scales + size_t(slot) * c->place.scale_lane};
}

int push(const cheb_cache *c, int32_t slot, GatherSeg *segs, int n_segs, hipStream_t stream) {
  return launch_store(c->quant, c->dtype, entry_of(c, slot), c->place, segs, n_segs, stream);
}

int predict(const cheb_cache *c, int32_t skip, int32_t used, const double *w, int32_t n_out,
            void *const *out, hipStream_t stream) {
  CodedEntry src[CHEB_MAX_SLOTS];
  for (int32_t j = 0; j < used; ++j)
    src[j] = entry_of(c, c->slot_of_age(c->count - skip - used + j));
  return launch_predict_coded(c->quant, c->dtype, src, used, w, n_out, out, c->slot_numel,
                              c->place, stream);
}

int residual(const cheb_cache *c, const double *w, const int64_t *delta, int n_delta,
             const ResidualInterval *iv, int n_iv, const float *x_in, float *x_out,
             hipStream_t stream) {
  CodedEntry src[CHEB_MAX_SLOTS];
  for (int32_t k = 0; k < c->n_slots; ++k) {
    if (fabs(w[k]) > double(FLT_MAX))
      return fail(CHEB_E_NONFINITE, "weight %d (%.17g) overflows fp32", k, w[k]);
    src[k] = entry_of(c, c->slot_of_age(k));
  }
  return launch_residual_coded(c->quant, c->n_slots, src, w, delta, n_delta, iv, n_iv, x_in,
                               x_out, c->place, stream);
}

const CodedOps kOps = {push, predict, residual};

}  // namespace

extern "C" {

int cheb_cache_layout_quant(int32_t n_slots, int32_t dtype, int32_t quant,
                            const int64_t *seg_numel, int32_t n_segs, int32_t layout,
                            int64_t *seg_offset, int64_t *slot_numel,
                            size_t *arena_bytes) try {
  Layout l;
  int rc = lay_out(n_slots, dtype, quant, seg_numel, n_segs, layout, &l);
  if (rc != CHEB_OK) return rc;
  if (seg_offset) memcpy(seg_offset, l.offset.data(), sizeof(int64_t) * l.offset.size());
  if (slot_numel) *slot_numel = l.slot_numel;
  if (arena_bytes) *arena_bytes = l.bytes;
  return ok();
} catch (const std::bad_alloc &) {
  return fail(CHEB_E_INVAL, "out of host memory");
}

int cheb_cache_create_quant(cheb_cache **out, int32_t n_slots, int32_t dtype, int32_t quant,
                            const int64_t *seg_numel, int32_t n_segs, int32_t layout, void *arena,
                            size_t arena_bytes) try {
  if (!out) return fail(CHEB_E_INVAL, "out is NULL");
  *out = nullptr;
  Layout l;
  int rc = lay_out(n_slots, dtype, quant, seg_numel, n_segs, layout, &l);
  if (rc != CHEB_OK) return rc;
  if (!arena) return fail(CHEB_E_INVAL, "arena is NULL");
  const uintptr_t a = reinterpret_cast<uintptr_t>(arena);
  if (a % kPlaneAlign != 0) return fail(CHEB_E_ALIGN, "arena is not 256-byte aligned");
  if (arena_bytes < l.bytes)
    return fail(CHEB_E_MISMATCH, "arena holds %zu bytes, the layout needs %zu", arena_bytes,
                l.bytes);
  std::unique_ptr<cheb_cache> c(new cheb_cache());
  c->n_slots = n_slots;
  c->dtype = dtype;
  c->seg_numel.assign(seg_numel, seg_numel + n_segs);
  c->seg_offset = std::move(l.offset);
  c->slot_numel = l.slot_numel;
  c->slot_stride = l.slot_stride;
  c->arena = static_cast<char *>(arena);
  c->arena_bytes = arena_bytes;
  c->layout = layout;
  c->coded = &kOps;
  c->quant = quant;
  c->place = l.place;
  char *region = layout == CHEB_LAYOUT_INTERLEAVED
                     ? reinterpret_cast<char *>(up(a, kLaneAlign))
                     : c->arena;
  c->place.codes = region + l.codes;
  c->place.scales = region + l.scales;
  *out = c.release();
  return ok();
} catch (const std::bad_alloc &) {
  return fail(CHEB_E_INVAL, "out of host memory");
}

int cheb_cache_quant(const cheb_cache *c, int32_t *quant) {
  if (!c || !quant) return fail(CHEB_E_INVAL, "cache or quant is NULL");
  *quant = c->quant;
  return ok();
}

int cheb_cache_read(cheb_cache *c, int32_t idx, void *out, void *stream) {
  if (!c) return fail(CHEB_E_INVAL, "cache is NULL");
  if (c->push_open) return fail(CHEB_E_NOTREADY, "a fused push is open");
  if (idx < 0 || idx >= c->count)
    return fail(CHEB_E_INVAL, "entry %d outside 0..%d", idx, c->count - 1);
  if (c->slot_numel == 0) return ok();
  void *outs[1] = {out};
  const uintptr_t a = reinterpret_cast<uintptr_t>(c->arena), o = reinterpret_cast<uintptr_t>(out);
  if (o < a + c->arena_bytes && a < o + uintptr_t(c->slot_numel) * uintptr_t(elem_bytes(c->dtype)))
    return fail(CHEB_E_INVAL, "out overlaps the cache arena");
  int rc = check_outputs(1, outs, c->slot_numel, c->dtype);
  if (rc != CHEB_OK) return rc;
  // The combination of one entry with weight one: exact.
  const double one = 1.0;
  if (c->coded)
    return c->coded->predict(c, c->count - 1 - idx, 1, &one, 1, outs,
                             static_cast<hipStream_t>(stream));
  const void *src[1] = {c->slot_ptr(c->slot_of_age(idx))};
  return combine_checked(src, 1, &one, 1, outs, c->slot_numel, c->dtype, c->super_vecs, stream);
}

}  // extern "C"
