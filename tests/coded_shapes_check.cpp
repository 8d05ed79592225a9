// The launch shapes of calls over 8-bit entries, on the CPU: the kernels that
// are built are the ones chosen, and grids stay within HIP's 2^32 - 1 threads
// up to the largest entry and residual.
#include <stdio.h>
#include <stdlib.h>

#include "coded_shapes.h"
#include "internal.h"
#include "shapes.h"

using namespace cheb;

static void fail_with(const char *what, int a, int b, unsigned long long c, int got) {
  fprintf(stderr, "%s: %d, %d, %llu: %d\n", what, a, b, c, got);
  exit(1);
}

int main() {
  // Residuals: a power of two of waves up to 8, one for one segment; the sums'
  // LDS of a block within what it may have.
  const uint32_t most = uint32_t(((int64_t(1) << 31) * 4 / 8 + 63) / 64);  // fp32: 2^31 vectors
  for (int ns = 1; ns <= 8; ++ns)
    for (int ncover = 0; ncover <= 128; ++ncover)
      for (uint32_t tiles : {1u, 255u, 1152u, 2048u, 2049u, 4096u, 4097u, 1u << 20,
                             (1u << 23) - 1, 1u << 23, (1u << 23) + 1, most, 1u << 25}) {
        const int w = coded_residual_waves(ns, ncover, tiles);
        const bool held = w == 1 || w == 2 || w == 4 || w == 8;
        if (!held || uint64_t(tiles) * 64u * uint64_t(w) > UINT32_MAX ||
            (ncover <= 1 && w != 1) || w * 4096 > kMostLds)
          fail_with("residual", ns, ncover, tiles, w);
      }
  if (coded_residual_waves(3, 56, 1152) != 8 || coded_residual_waves(6, 57, 27648) != 4 ||
      coded_residual_waves(1, 8, 1000) != 2 || coded_residual_waves(8, 56, 1u << 23) != 1)
    fail_with("residual rule", 0, 0, 0, 0);
  // Predictions: one or two runs a tile, lines kept together only where a tile
  // is short of one; entries are whole blocks, so tiles come out even.
  for (int ns = 1; ns <= 8; ++ns)
    for (int no = 1; no <= 8; ++no) {
      const CodedShape s = coded_shape(ns, no);
      if ((s.runs != 1 && s.runs != 2) || kCodedBlock % (512 * s.runs) != 0)
        fail_with("prediction", ns, no, 0, s.runs);
      for (int bytes : {2, 4})
        for (int64_t numel : {kCodedBlock, int64_t(1) << 20, int64_t(1) << 30,
                              kMaxVecs * (16 / bytes) / kCodedBlock * kCodedBlock}) {
          const int blocks = coded_blocks(ns, no, bytes, numel, 256);
          if (blocks < 0 || blocks > 64 || (blocks > 0 && blocks < 8))
            fail_with("blocks", ns, no, (unsigned long long)numel, blocks);
          if (uint64_t(numel) / uint64_t(512 * s.runs) * 64u > UINT32_MAX)
            fail_with("grid", ns, no, (unsigned long long)numel, s.runs);
          if (blocks < 32 && lds_share(160 << 10, blocks) * size_t(blocks) > 160u << 10)
            fail_with("lds", ns, no, (unsigned long long)numel, blocks);
        }
    }
  printf("coded_shapes ok\n");
  return 0;
}
