// Predictions from 8-bit entries for gfx950 (paper, Section 3.3, forward
// application equation): out_m = sum_k w_mk value_k over every element.
#include <hip/hip_runtime.h>

#include <stdint.h>
#include <string.h>

#include <algorithm>

#include "coded.h"
#include "internal.h"
#include "shapes.h"

namespace cheb {
namespace {

template <int NS, int NO, typename W>
struct CodedHist {
  const char *codes[NS], *scales[NS];
  void *o[NO];
  W w[NO][NS];
  uint64_t code_super, scale_super;
};

__device__ __forceinline__ float mad(float a, float b, float c) { return fmaf(a, b, c); }
__device__ __forceinline__ double mad(double a, double b, double c) { return fma(a, b, c); }

struct Bf16Out {
  using W = float;
  static constexpr int kBytes = 2;
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
  static constexpr int kBytes = 2;
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
  static constexpr int kBytes = 4;
  __device__ __forceinline__ static void store(void *out, uint64_t e, const W (&a)[8]) {
    u32x4 *o = reinterpret_cast<u32x4 *>(static_cast<float *>(out) + e);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      u32x4 r;
#pragma unroll
      for (int q = 0; q < 4; ++q) r[q] = __float_as_uint(float(a[4 * h + q]));
      __builtin_nontemporal_store(r, o + h);
    }
  }
};

// One-wave blocks, each a tile of two runs of 64 lanes x 8 elements.
template <class Fmt, class Out, int NS, int NO>
__global__ __launch_bounds__(64) void predict_coded_kernel(
    CodedHist<NS, NO, typename Out::W> h, uint32_t n_tiles) {
  constexpr int R = 2;
  using W = typename Out::W;
  const uint32_t lane = threadIdx.x;
  // The four tiles that share a line of scales go to one XCD (blocks are
  // dealt to the eight in turn).
  uint32_t tile = blockIdx.x;
  if (tile < (n_tiles & ~31u)) {
    const uint32_t q = tile >> 3;
    tile = ((q & ~3u) << 3) + ((tile & 7u) << 2) + (q & 3u);
  }
  const uint64_t chunk = tile >> 5;         // 32 tiles of 1024 elements
  const uint32_t in = (tile & 31u) * 1024u;
  const uint32_t co = in + lane * 8u;
  const uint32_t so = (in >> 12) * 128u + (lane >> 2) * 8u + (in >> 9 & 7u);
  u32x2 v[R][NS];
  uint32_t sc[NS];
#pragma unroll
  for (int k = 0; k < NS; ++k) {
    sc[k] = *reinterpret_cast<const uint16_t *>(h.scales[k] + chunk * h.scale_super + so);
#pragma unroll
    for (int r = 0; r < R; ++r)
      v[r][k] = __builtin_nontemporal_load(
          reinterpret_cast<const u32x2 *>(h.codes[k] + chunk * h.code_super + co + r * 512));
  }
  __builtin_amdgcn_sched_barrier(0);
  const uint64_t e0 = uint64_t(tile) * 1024u + lane * 8u;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    W acc[NO][8];
#pragma unroll
    for (int k = 0; k < NS; ++k) {
      const W scale = W(__uint_as_float((sc[k] >> (8 * r) & 255u) << 23));
      float q[8];
      Fmt::decode(v[r][k], q);
#pragma unroll
      for (int m = 0; m < NO; ++m) {
        const W unit = h.w[m][k] * scale;
#pragma unroll
        for (int e = 0; e < 8; ++e)
          acc[m][e] = k == 0 ? unit * W(q[e]) : mad(unit, W(q[e]), acc[m][e]);
      }
    }
#pragma unroll
    for (int m = 0; m < NO; ++m) Out::store(h.o[m], e0 + uint64_t(r) * 512u, acc[m]);
  }
}

struct Job {
  const CodedEntry *src;
  const double *w;
  void *const *out;
  int64_t numel;
  const CodedPlace *place;
  int cus, lds_per_cu;
};

template <class Fmt, class Out, int NS, int NO>
hipError_t launch_ns_no(const Job &j, hipStream_t s) {
  using W = typename Out::W;
  CodedHist<NS, NO, W> h;
  for (int k = 0; k < NS; ++k) {
    h.codes[k] = j.src[k].codes;
    h.scales[k] = j.src[k].scales;
  }
  for (int m = 0; m < NO; ++m) {
    h.o[m] = j.out[m];
    for (int k = 0; k < NS; ++k) h.w[m][k] = W(j.w[m * NS + k] * Fmt::kUnit);
  }
  h.code_super = j.place->code_super;
  h.scale_super = j.place->scale_super;
  const uint32_t tiles = uint32_t(j.numel / 1024);
  hipLaunchKernelGGL((predict_coded_kernel<Fmt, Out, NS, NO>), dim3(tiles), dim3(64), 0, s, h,
                     tiles);
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
  Job j{src, w, out, numel, &place, 0, 0};
  int rc = device_info(&j.cus, &j.lds_per_cu);
  if (rc != CHEB_OK) return rc;
  const hipError_t e = quant == CHEB_QUANT_MXINT8 ? launch_fmt<Int8Fmt>(dtype, n, n_out, j, stream)
                                                  : launch_fmt<E4m3Fmt>(dtype, n, n_out, j, stream);
  if (e != hipSuccess) return fail(CHEB_E_HIP, "prediction launch failed: %s", hipGetErrorString(e));
  return ok();
}

}  // namespace cheb
