// Predictions from 8-bit entries for gfx950 (paper, Section 3.3, forward
// application equation): out_m = sum_k w_mk value_k over every element.
#include <hip/hip_runtime.h>

#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <limits>
#include <type_traits>

#include "coded.h"
#include "coded_shapes.h"
#include "internal.h"
#include "shapes.h"

namespace cheb {
namespace {

template <int NS, int NO, typename W>
struct CodedHist {
  const char *codes[NS], *scales[NS];
  void *o[NO];
  W w[NO][NS];  // times what a code counts of its scale, over `back`
  W back;
  uint64_t code_super, scale_super;
};

// A power of two, 1 for weights of ordinary size, that takes the largest weight
// to where its products with a scale, up to 2^120 for e4m3 and 2^127 for int8,
// stay in the sums' range: else a zero code beside a large one would give NaN,
// and sums that are in range infinity.
template <class Fmt, class W>
W back_of(const double *w, int n) {
  double most = 0.0;
  for (int k = 0; k < n; ++k) most = std::max(most, fabs(double(W(w[k]))));
  const int room = std::numeric_limits<W>::max_exponent - Fmt::kMostScale;
  if (most * Fmt::kUnit < ldexp(1.0, room)) return W(1);
  return W(ldexp(1.0, ilogb(most * Fmt::kUnit) + 1 - room));
}

__device__ __forceinline__ float mad(float a, float b, float c) { return fmaf(a, b, c); }
__device__ __forceinline__ double mad(double a, double b, double c) { return fma(a, b, c); }

// Outputs: kLane elements of a lane, so that a store instruction of a wave
// covers 1 KiB without gaps (fp32 outputs in stores of 32 bytes a lane with gaps
// between them: 84 us for three entries of 66 M elements, 72 so).
struct Bf16Out {
  using W = float;
  static constexpr int kLane = 8, kBytes = 2;
  __device__ __forceinline__ static void store(void *out, uint64_t e, const W (&a)[8]) {
    u32x4 r;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const f32x2 p = {a[2 * q], a[2 * q + 1]};
      r[q] = __builtin_bit_cast(uint32_t, __builtin_convertvector(p, bf16x2));
    }
    __builtin_nontemporal_store(r, reinterpret_cast<u32x4 *>(static_cast<uint16_t *>(out) + e));
  }
};

struct F16Out {
  using W = float;
  static constexpr int kLane = 8, kBytes = 2;
  __device__ __forceinline__ static void store(void *out, uint64_t e, const W (&a)[8]) {
    u32x4 r;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const f32x2 p = {a[2 * q], a[2 * q + 1]};
      r[q] = __builtin_bit_cast(uint32_t, __builtin_convertvector(p, f16x2));
    }
    __builtin_nontemporal_store(r, reinterpret_cast<u32x4 *>(static_cast<uint16_t *>(out) + e));
  }
};

struct F32Out {
  using W = double;
  static constexpr int kLane = 4, kBytes = 4;
  __device__ __forceinline__ static void store(void *out, uint64_t e, const W (&a)[4]) {
    u32x4 r;
#pragma unroll
    for (int q = 0; q < 4; ++q) r[q] = __float_as_uint(float(a[q]));
    __builtin_nontemporal_store(r, reinterpret_cast<u32x4 *>(static_cast<float *>(out) + e));
  }
};

template <int R>
struct ScalesOf;
template <>
struct ScalesOf<1> {
  using Type = uint8_t;
};
template <>
struct ScalesOf<2> {
  using Type = uint16_t;
};

__device__ __forceinline__ u32x2 load_codes(const u32x2 *p) {
  return __builtin_nontemporal_load(p);
}
__device__ __forceinline__ u32x2 load_codes(const uint32_t *p) {
  return u32x2{__builtin_nontemporal_load(p), 0u};
}

// One-wave blocks, each a tile of R runs of 512 elements, kLane of them to a
// lane at a time.  kLines: the tiles that share a line of scales on one XCD.
template <class Fmt, class Out, int NS, int NO, int R, bool kLines>
__global__ __launch_bounds__(64) void predict_coded_kernel(
    CodedHist<NS, NO, typename Out::W> h) {
  using W = typename Out::W;
  using Codes = std::conditional_t<Out::kLane == 8, u32x2, uint32_t>;
  constexpr uint32_t V = Out::kLane, kTile = 512u * R;
  constexpr int P = 8 / int(V);  // parts of a run, with groups of their own
  constexpr uint32_t kChunkTiles = uint32_t(kCodedChunk) / kTile;
  const uint32_t lane = threadIdx.x;
  const uint32_t tile = kLines ? line_tile<8u / R>(blockIdx.x, gridDim.x) : blockIdx.x;
  const uint64_t chunk = tile / kChunkTiles;
  const uint32_t in = tile % kChunkTiles * kTile;
  const uint64_t cb = chunk * h.code_super + in;
  const uint64_t sb = chunk * h.scale_super + (in >> 12) * 128u + (in >> 9 & 7u);
  u32x2 v[R * P][NS];
  uint32_t sc[P][NS];
#pragma unroll
  for (int k = 0; k < NS; ++k)
#pragma unroll
    for (int r = 0; r < R * P; ++r)
      v[r][k] = load_codes(
          reinterpret_cast<const Codes *>(h.codes[k] + cb + (lane * V + uint32_t(r) * 64u * V)));
#pragma unroll
  for (int k = 0; k < NS; ++k)
#pragma unroll
    for (int p = 0; p < P; ++p)
      sc[p][k] = *reinterpret_cast<const typename ScalesOf<R>::Type *>(
          h.scales[k] + sb + (lane * V / 32u + uint32_t(p) * (16u / P)) * 8u);
  __builtin_amdgcn_sched_barrier(0);
  const uint64_t e0 = uint64_t(tile) * kTile + lane * V;
#pragma unroll
  for (int r = 0; r < R * P; ++r) {
    W acc[NO][V];
#pragma unroll
    for (int k = 0; k < NS; ++k) {
      const W scale = W(__uint_as_float((sc[r % P][k] >> (8 * (r / P)) & 255u) << 23));
      const Halves q = Fmt::decode(v[r][k]);
#pragma unroll
      for (int m = 0; m < NO; ++m) {
        const W unit = h.w[m][k] * scale;
#pragma unroll
        for (int e = 0; e < int(V); ++e)
          acc[m][e] = mad(unit, W(q[e]), k == 0 ? W(0) : acc[m][e]);
      }
    }
    if (std::is_same_v<W, double> || h.back != W(1)) {  // fp64: cheaper than the branch
#pragma unroll
      for (int m = 0; m < NO; ++m)
#pragma unroll
        for (int e = 0; e < int(V); ++e) acc[m][e] *= h.back;
    }
#pragma unroll
    for (int m = 0; m < NO; ++m)
      Out::store(h.o[m], e0 + uint64_t(r) * (64u * V), acc[m]);
  }
}

struct Job {
  const CodedEntry *src;
  const double *w;
  void *const *out;
  int64_t numel;
  const CodedPlace *place;
  int cus, lds_per_cu;
  int waves;  // as configured: 0 chosen here, -1 no limit
};

template <class Fmt, class Out, int NS, int NO>
hipError_t launch_ns_no(const Job &j, hipStream_t s) {
  using W = typename Out::W;
  CodedHist<NS, NO, W> h;
  for (int k = 0; k < NS; ++k) {
    h.codes[k] = j.src[k].codes;
    h.scales[k] = j.src[k].scales;
  }
  h.back = back_of<Fmt, W>(j.w, NO * NS);
  for (int m = 0; m < NO; ++m) {
    h.o[m] = j.out[m];
    for (int k = 0; k < NS; ++k)
      h.w[m][k] = W(j.w[m * NS + k] * Fmt::kUnit / double(h.back));
  }
  h.code_super = j.place->code_super;
  h.scale_super = j.place->scale_super;
  constexpr CodedShape kShape = coded_shape(NS, NO);
  constexpr int R = kShape.runs;
  const uint32_t tiles = uint32_t(j.numel / (512 * R));
  const int blocks = j.waves != 0 ? j.waves : coded_blocks(NS, NO, Out::kBytes, j.numel, j.cus);
  hipLaunchKernelGGL((predict_coded_kernel<Fmt, Out, NS, NO, R, kShape.lines>), dim3(tiles),
                     dim3(64), blocks > 2 && blocks < 32 ? lds_share(j.lds_per_cu, blocks) : 0, s,
                     h);
  return hipGetLastError();
}

template <class Fmt, class Out, int NS>
hipError_t launch_ns(int n_out, const Job &j, hipStream_t s) {
  switch (n_out) {
    case 1: return launch_ns_no<Fmt, Out, NS, 1>(j, s);
    case 2: return launch_ns_no<Fmt, Out, NS, 2>(j, s);
    case 3: return launch_ns_no<Fmt, Out, NS, 3>(j, s);
    case 4: return launch_ns_no<Fmt, Out, NS, 4>(j, s);
    case 5: return launch_ns_no<Fmt, Out, NS, 5>(j, s);
    case 6: return launch_ns_no<Fmt, Out, NS, 6>(j, s);
    case 7: return launch_ns_no<Fmt, Out, NS, 7>(j, s);
    default: return launch_ns_no<Fmt, Out, NS, 8>(j, s);
  }
}

template <class Fmt, class Out>
hipError_t launch_out(int n, int n_out, const Job &j, hipStream_t s) {
  switch (n) {
    case 1: return launch_ns<Fmt, Out, 1>(n_out, j, s);
    case 2: return launch_ns<Fmt, Out, 2>(n_out, j, s);
    case 3: return launch_ns<Fmt, Out, 3>(n_out, j, s);
    case 4: return launch_ns<Fmt, Out, 4>(n_out, j, s);
    case 5: return launch_ns<Fmt, Out, 5>(n_out, j, s);
    case 6: return launch_ns<Fmt, Out, 6>(n_out, j, s);
    case 7: return launch_ns<Fmt, Out, 7>(n_out, j, s);
    default: return launch_ns<Fmt, Out, 8>(n_out, j, s);
  }
}

template <class Fmt>
hipError_t launch_fmt(int dtype, int n, int n_out, const Job &j, hipStream_t s) {
  switch (dtype) {
    case CHEB_BF16: return launch_out<Fmt, Bf16Out>(n, n_out, j, s);
    case CHEB_F16: return launch_out<Fmt, F16Out>(n, n_out, j, s);
    default: return launch_out<Fmt, F32Out>(n, n_out, j, s);
  }
}

}  // namespace

int launch_predict_coded(int quant, int dtype, const CodedEntry *src, int n, const double *w,
                         int n_out, void *const *out, int64_t numel, const CodedPlace &place,
                         hipStream_t stream) {
  Job j{src, w, out, numel, &place, 0, 0, launch_shape().waves_per_cu};
  int rc = device_info(&j.cus, &j.lds_per_cu);
  if (rc != CHEB_OK) return rc;
  const hipError_t e = quant == CHEB_QUANT_MXINT8 ? launch_fmt<Int8Fmt>(dtype, n, n_out, j, stream)
                                                  : launch_fmt<E4m3Fmt>(dtype, n, n_out, j, stream);
  if (e != hipSuccess) return fail(CHEB_E_HIP, "prediction launch failed: %s", hipGetErrorString(e));
  return ok();
}

}  // namespace cheb
