// Device kernels of the 8-bit history for gfx950 (CDNA4, wave64): a full
// step quantised as it is stored, predictions from such entries, and the
// residual update from them.  The entries' format is described with
// cheb_cache_create_quant, their place in the arena in internal.h.
#include <hip/hip_runtime.h>

#include <stdint.h>
#include <string.h>

#include <algorithm>
#include <type_traits>

#include "coded.h"
#include "coded_shapes.h"
#include "internal.h"
#include "tiles.h"

namespace cheb {
namespace {

// ---- full-step push ----------------------------------------------------------

struct StoreArgs {
  const void *src[kGatherSegs];
  uint32_t block[kGatherSegs];  // first block in the entry
  uint64_t numel[kGatherSegs];
  GatherClass cls[kGatherClasses];
  int32_t classes;
  char *codes, *scales;
  uint64_t code_super, scale_super;
};

constexpr int kRuns = int(kCodedBlock) / 512;   // runs of 64 lanes x 8 elements in a block
constexpr int64_t kStoreVec = kCodedBlock / kGatherTileVecs;

// The four waves of a block quantise 4096 elements, two runs of 64 lanes x 8
// each, and share the line of their scales.  The four lanes of a group find its
// largest magnitude by two exchanges; a wave's two scales of a group's place go
// out together.  Bound by HBM, two reads to one write for bf16: FLUX-1024's 76
// tensors (2.45 GB moved) 387 us, 6.3 TB/s, and 24 ragged tensors of 2.3 M
// fp16 elements 28.3 us; one wave with all eight runs takes 384 and 32.6.
constexpr int kWaveRuns = 2;
constexpr int kStoreThreads = 64 * (kRuns / kWaveRuns);

template <class Fmt, class Src, bool kFlat>
__global__ __launch_bounds__(kStoreThreads) void store_kernel(StoreArgs a) {
  uint32_t s = blockIdx.y, tile = blockIdx.x;
  if constexpr (!kFlat) {
    int32_t p = 0;
    for (int32_t q = 1; q < a.classes; ++q)
      if (blockIdx.x >= a.cls[q].block) p = q;
    const GatherClass c = a.cls[p];
    const uint32_t b = blockIdx.x - c.block;
    s = __umulhi(b, c.inverse);  // b / tiles, or one less
    tile = b - s * c.tiles;
    if (tile >= c.tiles) {
      ++s;
      tile -= c.tiles;
    }
    s += uint32_t(c.seg);
  }
  const uint64_t numel = a.numel[s];
  if (uint64_t(tile) * uint64_t(kCodedBlock) >= numel) return;
  const uint32_t lane = threadIdx.x & 63u;
  const uint32_t run = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * uint32_t(kWaveRuns);
  const uint64_t first = uint64_t(tile) * uint64_t(kCodedBlock) + run * 512u;
  const typename Src::E *src = static_cast<const typename Src::E *>(a.src[s]) + first + lane * 8u;
  const uint32_t block = a.block[s] + tile;
  char *codes = a.codes + uint64_t(block >> 3) * a.code_super + (block & 7u) * 4096u +
                run * 512u + lane * 8u;
  char *scales = a.scales + uint64_t(block >> 3) * a.scale_super + (block & 7u) * 128u + run;
  typename Src::Raw v[kWaveRuns];
  if (first + 512u * kWaveRuns <= numel) {
#pragma unroll
    for (int r = 0; r < kWaveRuns; ++r) v[r] = Src::load(src + r * 512);
  } else {
#pragma unroll
    for (int r = 0; r < kWaveRuns; ++r) {
      const uint64_t at = first + uint64_t(r) * 512u + lane * 8u;
      v[r] = Src::load_some(src + r * 512, at < numel ? numel - at : 0u);
    }
  }
  __builtin_amdgcn_sched_barrier(0);
  uint32_t scale = 0;
#pragma unroll
  for (int r = 0; r < kWaveRuns; ++r) {
    const Group g = group_of<Fmt>(Src::magnitude(quad_max(Src::top(v[r]))));
    float x[8];
    Src::values(v[r], x);
    __builtin_nontemporal_store(Fmt::encode(x, g), reinterpret_cast<u32x2 *>(codes + r * 512));
    scale |= g.scale << (r * 8);
  }
  if ((lane & 3u) == 0)
    *reinterpret_cast<uint16_t *>(scales + (lane >> 2) * 8u) = uint16_t(scale);
}

template <class Fmt, class Src>
hipError_t launch_store_typed(const StoreArgs &a, const GatherPlan &plan, hipStream_t s) {
  const dim3 grid = plan.flat ? dim3(plan.widest, uint32_t(plan.segs)) : dim3(plan.blocks);
  const auto kernel = plan.flat ? store_kernel<Fmt, Src, true> : store_kernel<Fmt, Src, false>;
  hipLaunchKernelGGL(kernel, grid, dim3(kStoreThreads), 0, s, a);
  return hipGetLastError();
}

template <class Fmt>
hipError_t launch_store_fmt(int dtype, const StoreArgs &a, const GatherPlan &plan, hipStream_t s) {
  switch (dtype) {
    case CHEB_BF16: return launch_store_typed<Fmt, Bf16Src>(a, plan, s);
    case CHEB_F16: return launch_store_typed<Fmt, F16Src>(a, plan, s);
    default: return launch_store_typed<Fmt, F32Src>(a, plan, s);
  }
}

// ---- residual update ---------------------------------------------------------

constexpr int kCover = 128;

struct CodedPart {
  uint32_t tile;
  uint32_t vec_begin, n_vec;
  int32_t first, ncover;  // its covering segments in the delta table
};

template <int NS>
struct CodedResArgs {
  const char *codes[NS], *scales[NS];
  double w[NS];  // times kDouble kSum
  int64_t delta[kCover];  // vectors of 8, from an entry's start to the segment's residual vector 0
  CodedPart part[kMaxResIntervals];
  int32_t n_part;
  uint32_t code_super, scale_super;
  const float *x_in;  // may be null: zero
  float *x_out;
};

// A tile is a run of 64 residual vectors of 8.  The W waves of a block share it,
// each taking every W-th batch of U covering segments.  Weights and sums are
// fp64, as over plain entries, the waves' sums joined through LDS: x is rounded
// once, whatever the cache's storage type.  Bound by HBM reads: 33 bytes for 32
// elements of each entry and segment.  FLUX-1024, 6 interleaved entries: 788 us,
// 6.5 TB/s (786 with sums in fp32; 56 segments of 1152 tiles, 3 entries: 19.6, 19.1;
// 859 and 21.1 with codes converted to fp64 instead of built).  The lines of
// scales, 1 in 33, are read by 8 tiles, which are kept on one XCD for that, with
// those of the next line (833 and 22.1 where every XCD reads its own).
template <class Fmt, int NS, int W, int U>
__global__ __launch_bounds__(64 * W) void residual_coded_kernel(CodedResArgs<NS> a) {
  const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t lane = threadIdx.x & 63u;
  const uint32_t tile = line_tile<2 * kRuns>(blockIdx.x, gridDim.x);
  int32_t p = 0;
  for (int32_t q = 1; q < a.n_part; ++q)
    if (tile >= a.part[q].tile) p = q;
  const CodedPart part = a.part[p];
  const uint32_t first = (tile - part.tile) * kRun;
  const uint32_t live = std::min(part.n_vec - first, kRun);
  const uint32_t l = std::min(lane, live - 1u);  // idle lanes repeat the last vector
  const uint64_t j0 = uint64_t(part.vec_begin) + first;
  const auto added = [](uint32_t x, double sum) {
    return __float_as_uint(float(fma(sum, 1.0 / Fmt::kSum, double(__uint_as_float(x)))));
  };
  double acc[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) acc[e] = -0.0;  // the sum of nothing: x + -0.0 is x, -0.0 too
  auto take = [&](auto count, int32_t at) {
    constexpr int N = decltype(count)::value;
    u32x2 v[N][NS];
    uint32_t sc[N][NS];
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const uint64_t v0 = uint64_t(a.delta[part.first + at + u]) + j0;
      const uint64_t chunk = v0 >> 12;
      uint32_t r = (uint32_t(v0) & 4095u) + l;
      const bool next = r >= 4096u;  // a run spans at most two chunks
      r &= 4095u;
      const uint32_t co = r * 8u + (next ? a.code_super : 0u);
      const uint32_t so = (r >> 9) * 128u + (r >> 2 & 15u) * 8u + (r >> 6 & 7u) +
                          (next ? a.scale_super : 0u);
#pragma unroll
      for (int k = 0; k < NS; ++k)
        v[u][k] = __builtin_nontemporal_load(
            reinterpret_cast<const u32x2 *>(a.codes[k] + chunk * a.code_super + co));
#pragma unroll
      for (int k = 0; k < NS; ++k)
        sc[u][k] = *reinterpret_cast<const uint8_t *>(a.scales[k] + chunk * a.scale_super + so);
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int u = 0; u < N; ++u)
#pragma unroll
      for (int k = 0; k < NS; ++k) {
        const double unit = a.w[k] * double(__uint_as_float(sc[u][k] << 23));
        double q[8];
        Fmt::doubles(v[u][k], q);
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[e] = fma(unit, q[e], acc[e]);
      }
  };
  int32_t c = int32_t(wave) * U;
  for (; c + U <= part.ncover; c += W * U) take(std::integral_constant<int, U>(), c);
  if constexpr (U > 1) {
    for (; c < part.ncover; ++c) take(std::integral_constant<int, 1>(), c);
  }
  if constexpr (W == 1) {
    if (lane >= live) return;
    const uint64_t o = (j0 + lane) * 8u;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      u32x4 x = {0u, 0u, 0u, 0u}, r;
      if (a.x_in) x = *reinterpret_cast<const u32x4 *>(a.x_in + o + 4 * h);
#pragma unroll
      for (int q = 0; q < 4; ++q)
        r[q] = added(x[q], acc[4 * h + q]);
      *reinterpret_cast<u32x4 *>(a.x_out + o + 4 * h) = r;
    }
  } else {
    // Element e of vector n at [e * 64 + n]: consecutive lanes write
    // consecutive words.
    __shared__ double sums[W][8 * 64];
#pragma unroll
    for (int e = 0; e < 8; ++e) sums[wave][e * 64 + int(lane)] = acc[e];
    __syncthreads();
    for (uint32_t h = threadIdx.x; h < live * 2u; h += 64u * W) {
      const uint64_t o = j0 * 8u + 4u * h;
      const uint32_t at = 4u * (h & 1u) * 64u + (h >> 1);
      u32x4 x = {0u, 0u, 0u, 0u}, r;
      if (a.x_in) x = *reinterpret_cast<const u32x4 *>(a.x_in + o);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        double s = sums[0][at + uint32_t(q) * 64u];
#pragma unroll
        for (int w = 1; w < W; ++w) s += sums[w][at + uint32_t(q) * 64u];
        r[q] = added(x[q], s);
      }
      *reinterpret_cast<u32x4 *>(a.x_out + o) = r;
    }
  }
}

struct CodedResJob {
  const CodedEntry *src;
  const double *w;
  const int64_t *delta;
  int n_delta;
  const ResidualInterval *iv;
  int n_iv;
  const float *x_in;
  float *x_out;
  const CodedPlace *place;
};

template <class Fmt, int NS>
hipError_t launch_residual_ns(const CodedResJob &j, hipStream_t s) {
  CodedResArgs<NS> a;
  memset(&a, 0, sizeof a);
  for (int k = 0; k < NS; ++k) {
    a.codes[k] = j.src[k].codes;
    a.scales[k] = j.src[k].scales;
    a.w[k] = j.w[k] * (Fmt::kDouble * Fmt::kSum);
  }
  memcpy(a.delta, j.delta, sizeof(int64_t) * size_t(j.n_delta));
  a.code_super = uint32_t(j.place->code_super);
  a.scale_super = uint32_t(j.place->scale_super);
  a.x_in = j.x_in;
  a.x_out = j.x_out;
  a.n_part = j.n_iv;
  int ncover = 0;
  uint32_t tiles = 0;
  for (int i = 0, first = 0; i < j.n_iv; first += j.iv[i].ncover, ++i) {
    const uint32_t n_vec = uint32_t(j.iv[i].n_vec);
    a.part[i] = CodedPart{tiles, uint32_t(j.iv[i].vec_begin), n_vec, first, j.iv[i].ncover};
    tiles += run_tiles<1>(n_vec, kRunLg);
    ncover = std::max(ncover, int(j.iv[i].ncover));
  }
  constexpr int U = 2;  // segments ahead of their sums
  const auto launch = [&](auto kernel, int waves) {
    hipLaunchKernelGGL(kernel, dim3(tiles), dim3(64 * waves), 0, s, a);
    return hipGetLastError();
  };
  switch (coded_residual_waves(NS, ncover, tiles)) {
    case 1: return launch(residual_coded_kernel<Fmt, NS, 1, U>, 1);
    case 2: return launch(residual_coded_kernel<Fmt, NS, 2, U>, 2);
    case 4: return launch(residual_coded_kernel<Fmt, NS, 4, U>, 4);
    default: return launch(residual_coded_kernel<Fmt, NS, 8, U>, 8);
  }
}

template <class Fmt>
hipError_t launch_residual_fmt(int n, const CodedResJob &j, hipStream_t s) {
  switch (n) {
    case 1: return launch_residual_ns<Fmt, 1>(j, s);
    case 2: return launch_residual_ns<Fmt, 2>(j, s);
    case 3: return launch_residual_ns<Fmt, 3>(j, s);
    case 4: return launch_residual_ns<Fmt, 4>(j, s);
    case 5: return launch_residual_ns<Fmt, 5>(j, s);
    case 6: return launch_residual_ns<Fmt, 6>(j, s);
    case 7: return launch_residual_ns<Fmt, 7>(j, s);
    default: return launch_residual_ns<Fmt, 8>(j, s);
  }
}

}  // namespace

int launch_store(int quant, int dtype, const CodedEntry &to, const CodedPlace &place,
                 GatherSeg *segs, int n_segs, hipStream_t stream) {
  n_segs = order_segments(segs, n_segs);
  StoreArgs a;
  for (int at = 0; at < n_segs;) {
    // Blocks of 4096 elements: 64 "vectors" of 64.
    const GatherPlan plan = next_gather(segs + at, n_segs - at, kStoreVec, kChunkVecs);
    memset(&a, 0, sizeof a);
    for (int j = 0; j < plan.segs; ++j) {
      a.src[j] = segs[at + j].src;
      a.block[j] = uint32_t(segs[at + j].dst_offset / kCodedBlock);
      a.numel[j] = uint64_t(segs[at + j].numel);
    }
    memcpy(a.cls, plan.cls, sizeof(GatherClass) * size_t(plan.classes));
    a.classes = plan.classes;
    a.codes = const_cast<char *>(to.codes);
    a.scales = const_cast<char *>(to.scales);
    a.code_super = place.code_super;
    a.scale_super = place.scale_super;
    at += plan.segs;
    const hipError_t e = quant == CHEB_QUANT_MXINT8
                             ? launch_store_fmt<Int8Fmt>(dtype, a, plan, stream)
                             : launch_store_fmt<E4m3Fmt>(dtype, a, plan, stream);
    if (e != hipSuccess) return fail(CHEB_E_HIP, "push launch failed: %s", hipGetErrorString(e));
  }
  return ok();
}

int launch_residual_coded(int quant, int n, const CodedEntry *src, const double *w,
                          const int64_t *delta, int n_delta, const ResidualInterval *iv, int n_iv,
                          const float *x_in, float *x_out, const CodedPlace &place,
                          hipStream_t stream) {
  const CodedResJob j{src, w, delta, n_delta, iv, n_iv, x_in, x_out, &place};
  const hipError_t e = quant == CHEB_QUANT_MXINT8 ? launch_residual_fmt<Int8Fmt>(n, j, stream)
                                                  : launch_residual_fmt<E4m3Fmt>(n, j, stream);
  if (e != hipSuccess) return fail(CHEB_E_HIP, "residual launch failed: %s", hipGetErrorString(e));
  return ok();
}

}  // namespace cheb
