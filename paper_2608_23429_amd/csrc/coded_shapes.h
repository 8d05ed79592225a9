// How launches over 8-bit entries are laid out, by their sizes.  Host
// arithmetic.
#pragma once

#include <stdint.h>

#include <algorithm>

namespace cheb {

// A prediction's tiles: runs of 512 elements each, and whether the tiles that
// share a line of scales go to one XCD.  Measured on MI355X, bf16, entries of
// 264 M and 807 M elements in either layout, 1 to 8 entries and 1 to 4 outputs,
// tiles of 1, 2 and 4 runs:
//  - two runs; one where stores prevail, three outputs or more of three entries
//    or more (6 entries, 3 outputs of 528 M: 969 us, 988 with two runs; 4
//    entries, 4 outputs: 492, 505);
//  - every XCD reading its own copy of a line of scales costs 9% more reads (21%
//    with tiles of one run), and keeping the line's tiles together takes the stores
//    out of their order: that pays for one output of five entries or more (6
//    entries of 807 M: 980 us, 1009 without; 3 entries, 1 output: 201, 198 without;
//    6 entries, 3 outputs: 1007, 969).
struct CodedShape {
  int runs;
  bool lines;
};
constexpr CodedShape coded_shape(int ns, int no) {
  return {no >= 3 && ns >= 3 ? 1 : 2, no == 1 && ns >= 5};
}

// One-wave blocks that share a compute unit (0: no limit).  About 76 KiB of loads
// and stores in flight, between 8 and 20 blocks (one entry, 1 output: 120 us with 20,
// 122 without a limit; 6 entries: 980 with 10, 1003 with 12, 1016 without); a call of
// under 1 MiB a compute unit is over before the queues fill (3 entries of 33 M: 27.4
// us, 28.7 with 12).
inline int coded_blocks(int ns, int no, int out_bytes, int64_t numel, int cus) {
  const int kib = ns + no * out_bytes;  // of 1024 elements
  if (numel / 1024 * kib < int64_t(1024) * cus) return 0;
  const int blocks = std::min(std::max((76 + kib / 2) / kib, 8), 20);
  return coded_shape(ns, no).runs == 1 ? 2 * blocks : blocks;
}

// The waves that share a residual tile; each loads two segments ahead of its
// sums.  One segment is one wave's; a second wave pays from two on (2 segments
// of one entry, 36.9K tiles: 31.8 us, 37.7 with one; but 8 of them 49.7, 55.0 with
// four), four where there is much to read (24 segments of 2 entries, 1152 tiles:
// 8.1 us, 9.4 with two; FLUX-1024, 6 entries: 787, 789 with eight; 10 segments of 6
// entries, 18.4K tiles: 100.6, 104.5 with two, 113.2 with eight), and eight for
// many segments where the tiles are few (56 segments of 6 entries, 1152 tiles:
// 34.7, 36.5 with four; of 3 entries, 2304 tiles: 34.8, 36.7; from 4608 tiles on
// alike).  A limit on the blocks that share a compute unit gains under 1%.
inline int coded_residual_waves(int ns, int ncover, uint32_t tiles) {
  // HIP refuses a grid of 2^32 threads, which 8 waves a tile reach at 2^23.
  if (tiles >= uint32_t(1) << 23 || ncover <= 1) return 1;
  if (ncover <= 4 || (ns == 1 && ncover <= 28)) return 2;
  if (ncover >= 24 && ns >= 2 && tiles <= 4096) return 8;
  return 4;
}

}  // namespace cheb
