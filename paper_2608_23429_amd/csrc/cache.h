// The history cache's handle, shared by the host sources that work on it.
#pragma once

#include <vector>

#include "internal.h"

namespace cheb {

// What a ring of 8-bit entries (coded.cpp) does in place of a plain one.
// Arguments are validated by the calls that reach these.
struct CodedOps {
  int (*push)(const cheb_cache *c, int32_t slot, GatherSeg *segs, int n_segs, hipStream_t stream);
  // From the `used` newest entries but for `skip` of them, oldest first.
  int (*predict)(const cheb_cache *c, int32_t skip, int32_t used, const double *w, int32_t n_out,
                 void *const *out, hipStream_t stream);
  // As launch_residual_intervals; delta in vectors of kCodedVec elements.
  int (*residual)(const cheb_cache *c, const double *w, const int64_t *delta, int n_delta,
                  const ResidualInterval *iv, int n_iv, const float *x_in, float *x_out,
                  hipStream_t stream);
};

}  // namespace cheb

struct cheb_cache {
  int32_t n_slots = 0;
  int32_t dtype = CHEB_BF16;
  std::vector<int64_t> seg_numel;
  std::vector<int64_t> seg_offset;
  int64_t slot_numel = 0;
  size_t slot_stride = 0;
  char *arena = nullptr;
  size_t arena_bytes = 0;
  int32_t layout = CHEB_LAYOUT_SLOTS;
  char *region = nullptr;          // interleaved: first lane, on a kLaneAlign boundary
  int64_t super_vecs = cheb::kChunkVecs; // chunk stride of an entry (vectors)
  // 8-bit entries (null: plain ones): their format, and where a slot's codes
  // and scales lie (coded.cpp).
  const cheb::CodedOps *coded = nullptr;
  int32_t quant = CHEB_QUANT_NONE;
  cheb::CodedPlace place;
  // Ring state: `head` is the slot the next entry goes to; the `count` held
  // entries, oldest first, are in slots head - count, ..., head - 1 (mod n).
  double slot_t[CHEB_MAX_SLOTS] = {0};
  int32_t head = 0;
  int32_t count = 0;
  bool push_open = false;

  int32_t slot_of_age(int32_t age) const {
    return ((head - count + age) % n_slots + n_slots) % n_slots;
  }
  // Base of the entry stored in `slot` (its first vector).
  char *slot_ptr(int32_t slot) const {
    return layout == CHEB_LAYOUT_SLOTS ? arena + size_t(slot) * slot_stride
                                       : region + size_t(slot) * cheb::kChunkBytes;
  }
};
