// The residual's addition and the norm that follows it, for gfx950: see
// cheb_norm for the mathematics.
#include <hip/hip_runtime.h>

#include <stdint.h>
#include <string.h>

#include <algorithm>

#include "coded.h"
#include "internal.h"

namespace cheb {
namespace {

struct NormArgs {
  uint64_t base[CHEB_MAX_SLOTS], scales[CHEB_MAX_SLOTS];
  double w[CHEB_MAX_SLOTS];
  uint64_t first;                    // element of the sources' row 0
  uint64_t super, scale_super;       // bytes from chunk to chunk
  int32_t n;
  int32_t chunked;                   // sources lie in chunks
  const void *x_in;
  void *x_out;
  const float *gain, *shift;
  void *y;
  void *y_scale;
  double eps, inv_dim;
  uint32_t rows, dim, rows_per_group;
  int32_t layer, x_dtype, out_format;
};

// Four elements at any address aligned to one: a load or store of that many
// bytes takes any alignment.
typedef u32x2 __attribute__((aligned(2))) half4_any;
typedef u32x4 __attribute__((aligned(4))) float4_any;
typedef uint32_t __attribute__((aligned(1))) code4_any;

__device__ __forceinline__ float bf16_value(uint32_t h) { return __uint_as_float(h << 16); }
__device__ __forceinline__ float f16_value(uint32_t h) {
  return float(__builtin_bit_cast(_Float16, uint16_t(h)));
}

struct Four {
  float v[4];
};

// The first m (1 to 4) of four elements, zeros for the others.
template <class T>
__device__ __forceinline__ Four load_four(int dtype, const T *p, uint32_t m) {
  Four r;
  if (dtype == CHEB_F32) {
    const float *f = reinterpret_cast<const float *>(p);
    if (m == 4) {
      const u32x4 t = *reinterpret_cast<const float4_any *>(f);
#pragma unroll
      for (int i = 0; i < 4; ++i) r.v[i] = __uint_as_float(t[i]);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) r.v[i] = uint32_t(i) < m ? f[i] : 0.0f;
    }
    return r;
  }
  const uint16_t *h = reinterpret_cast<const uint16_t *>(p);
  uint32_t t[4];
  if (m == 4) {
    const u32x2 u = *reinterpret_cast<const half4_any *>(h);
#pragma unroll
    for (int i = 0; i < 4; ++i) t[i] = u[i >> 1] >> (16 * (i & 1)) & 0xffffu;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) t[i] = uint32_t(i) < m ? h[i] : 0u;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) r.v[i] = dtype == CHEB_BF16 ? bf16_value(t[i]) : f16_value(t[i]);
  return r;
}

__device__ __forceinline__ void store_four(int dtype, void *base, uint64_t at, const Four &x,
                                           uint32_t m) {
  if (dtype == CHEB_F32) {
    float *f = static_cast<float *>(base) + at;
    if (m == 4) {
      u32x4 t;
#pragma unroll
      for (int i = 0; i < 4; ++i) t[i] = __float_as_uint(x.v[i]);
      *reinterpret_cast<float4_any *>(f) = t;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (uint32_t(i) < m) f[i] = x.v[i];
    }
    return;
  }
  uint16_t *h = static_cast<uint16_t *>(base) + at;
  uint32_t t[2];
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    const f32x2 p = {x.v[2 * q], x.v[2 * q + 1]};
    t[q] = dtype == CHEB_BF16
               ? __builtin_bit_cast(uint32_t, __builtin_convertvector(p, bf16x2))
               : __builtin_bit_cast(uint32_t, __builtin_convertvector(p, f16x2));
  }
  if (m == 4) {
    *reinterpret_cast<half4_any *>(h) = u32x2{t[0], t[1]};
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (uint32_t(i) < m) h[i] = uint16_t(t[i >> 1] >> (16 * (i & 1)));
  }
}

// Sources of a storage type: element e at base + e, or in 32 KiB chunks.
template <int DT>
struct PlainSrc {
  static constexpr uint32_t kSize = DT == CHEB_F32 ? 4 : 2;
  static constexpr int kLg = DT == CHEB_F32 ? 13 : 14;  // elements of a chunk
  __device__ __forceinline__ static Four load(const NormArgs &a, int k, uint64_t e, uint32_t m) {
    const char *b = reinterpret_cast<const char *>(a.base[k]);
    if (!a.chunked) return load_four(DT, b + e * kSize, m);
    const uint32_t in = uint32_t(e) & ((1u << kLg) - 1u);
    const char *p = b + (e >> kLg) * a.super + in * kSize;
    if (in + m <= 1u << kLg) return load_four(DT, p, m);
    // across a chunk's end, element by element
    Four r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint64_t f = e + uint64_t(i);
      const char *q = b + (f >> kLg) * a.super + (uint32_t(f) & ((1u << kLg) - 1u)) * kSize;
      r.v[i] = uint32_t(i) < m ? load_four(DT, q, 1).v[0] : 0.0f;
    }
    return r;
  }
};

// 8-bit entries.
template <class Fmt>
struct CodedSrc {
  __device__ __forceinline__ static float scale(const NormArgs &a, int k, uint64_t e) {
    const uint32_t r = uint32_t(e) & uint32_t(kCodedChunk - 1);
    const uint8_t *s = reinterpret_cast<const uint8_t *>(a.scales[k]) +
                       (e >> kCodedChunkLg) * a.scale_super + (r >> 12) * 128u +
                       (r >> 5 & 15u) * 8u + (r >> 9 & 7u);
    return __uint_as_float(uint32_t(*s) << 23);
  }
  __device__ __forceinline__ static const uint8_t *code(const NormArgs &a, int k, uint64_t e) {
    return reinterpret_cast<const uint8_t *>(a.base[k]) + (e >> kCodedChunkLg) * a.super +
           (uint32_t(e) & uint32_t(kCodedChunk - 1));
  }
  __device__ __forceinline__ static Four load(const NormArgs &a, int k, uint64_t e, uint32_t m) {
    Four r;
    float q[8];
    if (m == 4 && (uint32_t(e) & 31u) <= 28u) {
      Fmt::decode(u32x2{*reinterpret_cast<const code4_any *>(code(a, k, e)), 0u}, q);
      const float s = scale(a, k, e) * float(Fmt::kUnit);
#pragma unroll
      for (int i = 0; i < 4; ++i) r.v[i] = q[i] * s;
      return r;
    }
    // across a group's end, or a row's, element by element
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      r.v[i] = 0.0f;
      if (uint32_t(i) < m) {
        Fmt::decode(u32x2{*code(a, k, e + uint64_t(i)), 0u}, q);
        r.v[i] = q[0] * (scale(a, k, e + uint64_t(i)) * float(Fmt::kUnit));
      }
    }
    return r;
  }
};

// Sums and maxima over the L threads of a row; every one gets the result.
template <int L>
struct RowOf {
  static constexpr int kWaves = L > 64 ? L / 64 : 1;

  __device__ __forceinline__ static double sum(double v, double *shared) {
#pragma unroll
    for (int o = 1; o < (L < 64 ? L : 64); o *= 2) v += __shfl_xor(v, o);
    if constexpr (kWaves > 1) {
      if ((threadIdx.x & 63u) == 0) shared[threadIdx.x >> 6] = v;
      __syncthreads();
      v = 0.0;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) v += shared[w];
    }
    return v;
  }

  __device__ __forceinline__ static uint32_t top(uint32_t v, uint32_t *shared) {
#pragma unroll
    for (int o = 1; o < (L < 64 ? L : 64); o *= 2) v = max(v, uint32_t(__shfl_xor(int(v), o)));
    if constexpr (kWaves > 1) {
      if ((threadIdx.x & 63u) == 0) shared[threadIdx.x >> 6] = v;
      __syncthreads();
      v = 0u;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) v = max(v, shared[w]);
    }
    return v;
  }
};

__device__ __forceinline__ uint32_t magnitude_of(const Four &y) {
  uint32_t t = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) t = max(t, __float_as_uint(y.v[i]) & 0x7fffffffu);
  return t;
}

// Codes of y times `factor` (0: codes 0, whatever y holds).
__device__ __forceinline__ void store_codes(void *base, uint64_t at, const Four &y, float factor,
                                            uint32_t m) {
  float v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = factor == 0.0f ? 0.0f : y.v[i] * factor;
  int p = __builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[1], 0, false);
  p = __builtin_amdgcn_cvt_pk_fp8_f32(v[2], v[3], p, true);
  uint8_t *b = static_cast<uint8_t *>(base) + at;
  if (m == 4) {
    *reinterpret_cast<code4_any *>(b) = uint32_t(p);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (uint32_t(i) < m) b[i] = uint8_t(p >> (8 * i));
  }
}

// L threads hold a row, P times four elements each: thread t's i-th four are
// elements (i L + t) * 4 on.
template <class Src, int L, int P>
__global__ __launch_bounds__(L < 256 ? 256 : L) void norm_kernel(NormArgs a) {
  constexpr int kThreads = L < 256 ? 256 : L;
  __shared__ double sums[2][16];
  __shared__ uint32_t tops[16];
  const uint32_t t = threadIdx.x % uint32_t(L);
  const uint32_t row = blockIdx.x * uint32_t(kThreads / L) + threadIdx.x / uint32_t(L);
  if (row >= a.rows) return;  // a whole row's threads; only L < 256, which meets no barrier
  const uint64_t r0 = uint64_t(row) * a.dim;
  uint32_t m[P];  // elements of each four within the row
#pragma unroll
  for (int i = 0; i < P; ++i) {
    const uint32_t e = (uint32_t(i) * L + t) * 4u;
    m[i] = e < a.dim ? (a.dim - e < 4u ? a.dim - e : 4u) : 0u;
  }
  double acc[P][4];
#pragma unroll
  for (int i = 0; i < P; ++i)
#pragma unroll
    for (int q = 0; q < 4; ++q) acc[i][q] = -0.0;  // the sum of nothing: x + -0.0 is x, -0.0 too
  Four x[P], s[P];
#pragma unroll
  for (int i = 0; i < P; ++i) {
    x[i] = Four{{0.0f, 0.0f, 0.0f, 0.0f}};
    const uint64_t e = r0 + (uint32_t(i) * L + t) * 4u;
    if (a.x_in && m[i])
      x[i] = load_four(a.x_dtype,
                       static_cast<const char *>(a.x_in) + e * (a.x_dtype == CHEB_F32 ? 4u : 2u),
                       m[i]);
  }
  for (int k = 0; k < a.n; ++k) {
#pragma unroll
    for (int i = 0; i < P; ++i) {
      s[i] = Four{{0.0f, 0.0f, 0.0f, 0.0f}};
      if (m[i]) s[i] = Src::load(a, k, a.first + r0 + (uint32_t(i) * L + t) * 4u, m[i]);
    }
    const double w = a.w[k];
#pragma unroll
    for (int i = 0; i < P; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q) acc[i][q] = fma(w, double(s[i].v[q]), acc[i][q]);
  }
  double sum = 0.0, squares = 0.0;
#pragma unroll
  for (int i = 0; i < P; ++i) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      x[i].v[q] = float(double(x[i].v[q]) + acc[i][q]);
      if (uint32_t(q) >= m[i]) x[i].v[q] = 0.0f;
      sum += double(x[i].v[q]);
      squares = fma(double(x[i].v[q]), double(x[i].v[q]), squares);
    }
    if (a.x_out && m[i])
      store_four(a.x_dtype, a.x_out, r0 + (uint32_t(i) * L + t) * 4u, x[i], m[i]);
  }
  if (a.layer) {
    const double mean = RowOf<L>::sum(sum, sums[0]) * a.inv_dim;
    squares = 0.0;
#pragma unroll
    for (int i = 0; i < P; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        x[i].v[q] = uint32_t(q) < m[i] ? float(double(x[i].v[q]) - mean) : 0.0f;
        squares = fma(double(x[i].v[q]), double(x[i].v[q]), squares);
      }
  }
  const float r =
      float(1.0 / sqrt(RowOf<L>::sum(squares, sums[1]) * a.inv_dim + a.eps));
  const uint64_t g0 = a.gain || a.shift ? uint64_t(row / a.rows_per_group) * a.dim : 0u;
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < P; ++i) {
    const uint32_t e = (uint32_t(i) * L + t) * 4u;
    Four g = {{1.0f, 1.0f, 1.0f, 1.0f}}, b = {{0.0f, 0.0f, 0.0f, 0.0f}};
    if (a.gain && m[i]) g = load_four(CHEB_F32, a.gain + g0 + e, m[i]);
    if (a.shift && m[i]) b = load_four(CHEB_F32, a.shift + g0 + e, m[i]);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const float y = x[i].v[q] * r;
      x[i].v[q] = a.gain ? y * g.v[q] : y;
      if (a.shift) x[i].v[q] += b.v[q];
      if (uint32_t(q) >= m[i]) x[i].v[q] = 0.0f;
    }
    top = max(top, magnitude_of(x[i]));
  }
  if (a.out_format == CHEB_OUT_MXFP8) {
    const uint32_t width = (a.dim + 31u) / 32u;
#pragma unroll
    for (int i = 0; i < P; ++i) {
      // the eight threads of a group: two exchanges in fours, then the fours
      uint32_t g = quad_max(magnitude_of(x[i]));
      g = max(g, uint32_t(__builtin_amdgcn_mov_dpp(int(g), 0x141, 0xF, 0xF, true)));
      const Group of = group_of<E4m3Fmt>(g);
      const uint32_t e = (uint32_t(i) * L + t) * 4u;
      if (m[i]) store_codes(a.y, r0 + e, x[i], of.factor, m[i]);
      if (m[i] && (t & 7u) == 0)
        static_cast<uint8_t *>(a.y_scale)[uint64_t(row) * width + e / 32u] = uint8_t(of.scale);
    }
    return;
  }
  if (a.out_format == CHEB_OUT_FP8_ROW) {
    const uint32_t bits = RowOf<L>::top(top, tops);
    float scale = 1.0f, factor = 1.0f;
    if (bits >= 0x7f800000u) {
      scale = __uint_as_float(0x7fc00000u);
      factor = 0.0f;
    } else if (bits != 0u) {
      scale = fmaxf(__uint_as_float(bits) / 448.0f, 0x1p-126f);
      factor = 1.0f / scale;
    }
    if (t == 0) static_cast<float *>(a.y_scale)[row] = scale;
#pragma unroll
    for (int i = 0; i < P; ++i)
      if (m[i]) store_codes(a.y, r0 + (uint32_t(i) * L + t) * 4u, x[i], factor, m[i]);
    return;
  }
#pragma unroll
  for (int i = 0; i < P; ++i)
    if (m[i]) store_four(a.out_format, a.y, r0 + (uint32_t(i) * L + t) * 4u, x[i], m[i]);
}

template <class Src, int L, int P>
hipError_t launch_shape(const NormArgs &a, hipStream_t s) {
  constexpr uint32_t kThreads = L < 256 ? 256 : L, kRows = kThreads / L;
  hipLaunchKernelGGL((norm_kernel<Src, L, P>), dim3((a.rows + kRows - 1) / kRows), dim3(kThreads),
                     0, s, a);
  return hipGetLastError();
}

// The fewest threads that hold a row in at most six times four elements each,
// so that a wave's worth of them needs no barrier.
template <class Src>
hipError_t launch_src(const NormArgs &a, hipStream_t s) {
  const uint32_t fours = (a.dim + 3u) / 4u;
  if (fours <= 8) return launch_shape<Src, 8, 1>(a, s);
  if (fours <= 16) return launch_shape<Src, 16, 1>(a, s);
  if (fours <= 32) return launch_shape<Src, 32, 1>(a, s);
  switch ((fours + 63u) / 64u) {
    case 1: return launch_shape<Src, 64, 1>(a, s);
    case 2: return launch_shape<Src, 64, 2>(a, s);
    case 3: return launch_shape<Src, 64, 3>(a, s);
    case 4: return launch_shape<Src, 64, 4>(a, s);
    case 5: return launch_shape<Src, 64, 5>(a, s);
    case 6: return launch_shape<Src, 64, 6>(a, s);
    default: break;
  }
  switch ((fours + 255u) / 256u) {
    case 2: return launch_shape<Src, 256, 2>(a, s);
    case 3: return launch_shape<Src, 256, 3>(a, s);
    case 4: return launch_shape<Src, 256, 4>(a, s);
    case 5:
    case 6: return launch_shape<Src, 256, 6>(a, s);
    case 7:
    case 8: return launch_shape<Src, 1024, 2>(a, s);
    default: return launch_shape<Src, 1024, 4>(a, s);
  }
}

}  // namespace

int launch_norm(const NormSources &from, const cheb_norm &n, hipStream_t stream) {
  NormArgs a;
  memset(&a, 0, sizeof a);
  for (int k = 0; k < from.n; ++k) {
    const bool coded = from.quant != CHEB_QUANT_NONE;
    a.base[k] = reinterpret_cast<uint64_t>(coded ? from.src[k].codes : from.base[k]);
    a.scales[k] = coded ? reinterpret_cast<uint64_t>(from.src[k].scales) : 0u;
    a.w[k] = from.w[k];
  }
  a.first = uint64_t(from.first);
  a.n = from.n;
  a.chunked = from.super_vecs != kChunkVecs;
  a.super = uint64_t(from.super_vecs) * 16u;
  a.x_in = n.x_in;
  a.x_out = n.x_out;
  a.gain = n.gain;
  a.shift = n.shift;
  a.y = n.y;
  a.y_scale = n.y_scale;
  a.eps = n.eps;
  a.inv_dim = 1.0 / double(n.dim);
  a.rows = uint32_t(n.rows);
  a.dim = uint32_t(n.dim);
  a.rows_per_group = uint32_t(std::min<int64_t>(std::max<int64_t>(n.rows_per_group, 1), 1 << 30));
  a.layer = n.kind == CHEB_NORM_LAYER;
  a.x_dtype = n.x_dtype;
  a.out_format = n.out_format;
  hipError_t e;
  if (from.quant != CHEB_QUANT_NONE) {
    a.super = from.place.code_super;
    a.scale_super = from.place.scale_super;
    e = from.quant == CHEB_QUANT_MXINT8 ? launch_src<CodedSrc<Int8Fmt>>(a, stream)
                                        : launch_src<CodedSrc<E4m3Fmt>>(a, stream);
  } else if (from.dtype == CHEB_BF16) {
    e = launch_src<PlainSrc<CHEB_BF16>>(a, stream);
  } else if (from.dtype == CHEB_F16) {
    e = launch_src<PlainSrc<CHEB_F16>>(a, stream);
  } else {
    e = launch_src<PlainSrc<CHEB_F32>>(a, stream);
  }
  if (e != hipSuccess) return fail(CHEB_E_HIP, "norm launch failed: %s", hipGetErrorString(e));
  return ok();
}

}  // namespace cheb
