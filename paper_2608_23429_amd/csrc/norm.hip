// The residual's addition and the norm that follows it, for gfx950: see
// cheb_norm for the mathematics.
#include <hip/hip_runtime.h>

#include <stdint.h>
#include <string.h>

#include <algorithm>
#include <type_traits>

#include "coded.h"
#include "internal.h"

namespace cheb {
namespace {

struct NormArgs {
  uint64_t base[CHEB_MAX_SLOTS], scales[CHEB_MAX_SLOTS];
  double w[CHEB_MAX_SLOTS];
  uint64_t first;                    // element of the sources' row 0
  uint32_t super, scale_super;       // bytes from chunk to chunk
  int32_t n;
  int32_t chunked;                   // sources lie in chunks
  const void *x_in;
  void *x_out;
  const float *gain, *shift;
  void *y;
  void *y_scale;
  double eps, inv_dim;
  uint32_t rows, dim, rows_per_group, group_inverse;
  int32_t layer, x_dtype, out_format;
};

// Four elements at any address aligned to one: a load or store of that many
// bytes takes any alignment.  (The types lose theirs as template arguments, so
// they are named where memory is read or written.)
typedef u32x2 __attribute__((aligned(2))) half4_any;
typedef u32x4 __attribute__((aligned(4))) float4_any;
typedef uint32_t __attribute__((aligned(1))) code4_any;

struct Four {
  float v[4];
};

// Four stored elements as loaded, converted later, so that loads follow one
// another without a wait.
struct Raw {
  uint32_t u[4];
};

__device__ __forceinline__ Raw raw_of(u32x4 t) { return {{t[0], t[1], t[2], t[3]}}; }
__device__ __forceinline__ Raw raw_of(u32x2 t) { return {{t[0], t[1], 0u, 0u}}; }

template <int DT>
struct Stored {
  static constexpr uint32_t kSize = DT == CHEB_F32 ? 4 : 2;

  // kStream: read once, with the non-temporal hint.
  template <bool kStream>
  __device__ __forceinline__ static Raw four(const char *p) {
    if constexpr (DT == CHEB_F32) {
      const float4_any *v = reinterpret_cast<const float4_any *>(p);
      return raw_of(kStream ? __builtin_nontemporal_load(v) : *v);
    } else {
      const half4_any *v = reinterpret_cast<const half4_any *>(p);
      return raw_of(kStream ? __builtin_nontemporal_load(v) : *v);
    }
  }
  // Element q of the four.
  __device__ __forceinline__ static void one(Raw &r, int q, const char *p) {
    if constexpr (DT == CHEB_F32) r.u[q] = *reinterpret_cast<const uint32_t *>(p);
    else r.u[q >> 1] |= uint32_t(*reinterpret_cast<const uint16_t *>(p)) << (16 * (q & 1));
  }
  __device__ __forceinline__ static Four values(const Raw &r) {
    Four x;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      if constexpr (DT == CHEB_F32) {
        x.v[q] = __uint_as_float(r.u[q]);
      } else {
        const uint32_t h = r.u[q >> 1] >> (16 * (q & 1));
        x.v[q] = DT == CHEB_BF16 ? __uint_as_float(h << 16)
                                 : float(__builtin_bit_cast(_Float16, uint16_t(h)));
      }
    }
    return x;
  }
};

// Which elements of a lane's four are the row's own: those from lo up to hi
// (none: hi is 0).
struct Own {
  uint32_t lo, hi;
  __device__ __forceinline__ bool has(uint32_t q) const { return q >= lo && q < hi; }
  __device__ __forceinline__ bool all() const { return lo == 0 && hi == 4; }
};

template <bool kStream>
__device__ __forceinline__ void put(char *to, u32x4 v) {
  float4_any *p = reinterpret_cast<float4_any *>(to);
  if constexpr (kStream) __builtin_nontemporal_store(v, p);
  else *p = v;
}
template <bool kStream>
__device__ __forceinline__ void put(char *to, u32x2 v) {
  half4_any *p = reinterpret_cast<half4_any *>(to);
  if constexpr (kStream) __builtin_nontemporal_store(v, p);
  else *p = v;
}

// kSome: not all or none of a four may be the row's own.
template <int DT, bool kSome, bool kStream = false>
__device__ __forceinline__ void store_four(char *p, const Four &x, const Own &own) {
  if constexpr (DT == CHEB_F32) {
    if (!kSome || own.all()) {
      u32x4 t;
#pragma unroll
      for (int q = 0; q < 4; ++q) t[q] = __float_as_uint(x.v[q]);
      put<kStream>(p, t);
    } else {
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (own.has(uint32_t(q))) reinterpret_cast<float *>(p)[q] = x.v[q];
    }
  } else {
    uint32_t t[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const f32x2 v = {x.v[2 * h], x.v[2 * h + 1]};
      if constexpr (DT == CHEB_BF16)
        t[h] = __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
      else
        t[h] = __builtin_bit_cast(uint32_t, __builtin_convertvector(v, f16x2));
    }
    if (!kSome || own.all()) {
      put<kStream>(p, u32x2{t[0], t[1]});
    } else {
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (own.has(uint32_t(q)))
          reinterpret_cast<uint16_t *>(p)[q] = uint16_t(t[q >> 1] >> (16 * (q & 1)));
    }
  }
}

// How a row's elements fall into fours.
//   kEven  dim is a multiple of four (and so is the sources' first element,
//          where fours must not cross a chunk or a group): every four is the
//          row's own or none of it is.
//   kOdd   contiguous sources of any dim: a row's last four reaches into the next
//          row, and in the last rows, which have none, starts earlier instead.
//   kSplit sources whose fours may cross a chunk or a group, or of fewer than
//          four elements in all: element by element.
enum { kEven, kOdd, kSplit };

// Where a row of the sources starts: `rb` bytes (scales: `rs`) from an entry's
// base, `in` elements into a chunk (0: contiguous sources).
struct RowAt {
  uint64_t rb, rs;
  uint32_t in;
};

// Sources of a storage type: contiguous, or in 32 KiB chunks.
template <int DT>
struct PlainSrc {
  using Type = Stored<DT>;
  using Held = Raw;
  using At = uint32_t;                                      // bytes from the row's base
  static constexpr uint32_t kLg = DT == CHEB_F32 ? 13 : 14;  // elements of a chunk
  static constexpr bool kAnyPlace = true;                    // fours may start at any element
  static constexpr double kSum = 1.0;                        // sums are held as that of their value

  __device__ __forceinline__ static RowAt row(const NormArgs &a, uint64_t e) {
    if (!a.chunked) return {e * Type::kSize, 0u, 0u};
    return {(e >> kLg) * a.super, 0u, uint32_t(e) & ((1u << kLg) - 1u)};
  }
  __device__ __forceinline__ static At at(const NormArgs &a, const RowAt &r, uint32_t el) {
    if (!a.chunked) return el * Type::kSize;
    const uint32_t in = r.in + el;
    return (in >> kLg) * a.super + (in & ((1u << kLg) - 1u)) * Type::kSize;
  }
  __device__ __forceinline__ static Held four(const NormArgs &a, int k, const RowAt &r, At at) {
    return Type::template four<true>(reinterpret_cast<const char *>(a.base[k] + r.rb) + at);
  }
  __device__ __forceinline__ static Held some(const NormArgs &a, int k, const RowAt &r,
                                              uint32_t el, const Own &own) {
    Held h = {{0u, 0u, 0u, 0u}};
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (own.has(uint32_t(q)))
        Type::one(h, q, reinterpret_cast<const char *>(a.base[k] + r.rb) +
                            at(a, r, el + uint32_t(q)));
    return h;
  }
  template <int M>
  __device__ __forceinline__ static void add(double (&sum)[4], double w, const Held &h) {
    const Four x = Type::values(h);
#pragma unroll
    for (int q = 0; q < 4; ++q) sum[q] = fma(w, double(x.v[q]), sum[q]);
  }
};

// 8-bit entries: four codes and their scale (kSplit: scales, a byte each).
// Codes are taken as fp64 numbers, so that one of 2^128 or more, beside fp32's
// largest values, counts; weights come times kDouble kSum.
template <class Fmt>
struct CodedSrc {
  struct Held {
    uint32_t codes, scales;
  };
  struct At {
    uint32_t code, scale;
  };
  static constexpr bool kAnyPlace = false;
  static constexpr double kSum = Fmt::kSum;

  __device__ __forceinline__ static RowAt row(const NormArgs &a, uint64_t e) {
    return {(e >> kCodedChunkLg) * a.super, (e >> kCodedChunkLg) * a.scale_super,
            uint32_t(e) & uint32_t(kCodedChunk - 1)};
  }
  __device__ __forceinline__ static At at(const NormArgs &a, const RowAt &r, uint32_t el) {
    const uint32_t in = r.in + el, chunk = in >> kCodedChunkLg;
    const uint32_t e = in & uint32_t(kCodedChunk - 1);
    return {chunk * a.super + e,
            chunk * a.scale_super + (e >> 12) * 128u + (e >> 5 & 15u) * 8u + (e >> 9 & 7u)};
  }
  __device__ __forceinline__ static Held four(const NormArgs &a, int k, const RowAt &r, At at) {
    return {__builtin_nontemporal_load(
                reinterpret_cast<const code4_any *>(a.base[k] + r.rb + at.code)),
            uint32_t(*reinterpret_cast<const uint8_t *>(a.scales[k] + r.rs + at.scale))};
  }
  __device__ __forceinline__ static Held some(const NormArgs &a, int k, const RowAt &r,
                                              uint32_t el, const Own &own) {
    Held h = {0u, 0u};
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (own.has(uint32_t(q))) {
        const At p = at(a, r, el + uint32_t(q));
        h.codes |= uint32_t(*reinterpret_cast<const uint8_t *>(a.base[k] + r.rb + p.code))
                   << (8 * q);
        h.scales |= uint32_t(*reinterpret_cast<const uint8_t *>(a.scales[k] + r.rs + p.scale))
                    << (8 * q);
      }
    return h;
  }
  template <int M>
  __device__ __forceinline__ static void add(double (&sum)[4], double w, const Held &h) {
    double c[8];
    Fmt::doubles(u32x2{h.codes, 0u}, c);
    double unit = w * double(__uint_as_float(h.scales << 23));
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      if constexpr (M == kSplit)
        unit = w * double(__uint_as_float((h.scales >> (8 * q) & 255u) << 23));
      sum[q] = fma(unit, c[q], sum[q]);
    }
  }
};

template <int CTRL>
__device__ __forceinline__ uint32_t moved(uint32_t v) {
  return uint32_t(__builtin_amdgcn_mov_dpp(int(v), CTRL, 0xF, 0xF, true));
}
template <int CTRL>
__device__ __forceinline__ double moved(double v) {
  const uint64_t b = __builtin_bit_cast(uint64_t, v);
  return __builtin_bit_cast(double, uint64_t(moved<CTRL>(uint32_t(b))) |
                                        uint64_t(moved<CTRL>(uint32_t(b >> 32))) << 32);
}

// Joins the values of the L (up to 64) neighbouring lanes of a row: exchanges
// within fours, eights and sixteens by mirrors (both halves hold one value each
// by then), then across.
template <int L, class T, class Join>
__device__ __forceinline__ T join_lanes(T v, Join join) {
  v = join(v, moved<0xB1>(v));   // 1 0 3 2
  v = join(v, moved<0x4E>(v));   // 2 3 0 1
  v = join(v, moved<0x141>(v));  // mirrored in eights
  if constexpr (L >= 16) v = join(v, moved<0x140>(v));  // in sixteens
  if constexpr (L >= 32) v = join(v, __shfl_xor(v, 16));
  if constexpr (L >= 64) v = join(v, __shfl_xor(v, 32));
  return v;
}

// Codes of y times `factor` (0: codes 0, whatever y holds): exact for a power of
// two, in fp64 for others.  y times the fp64 reciprocal of an fp32 scale, rounded
// to fp32, is the fp32 quotient: no quotient of two such numbers is within 2^-49
// of its size of the middle between two more, and the product is off by 2^-52.
template <bool kSome, class Factor>
__device__ __forceinline__ void store_codes(char *p, const Four &y, Factor factor,
                                            const Own &own) {
  float v[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) v[q] = float(Factor(y.v[q]) * factor);
  if (__builtin_expect(__ballot(factor == Factor(0)) != 0ull, 0)) {
#pragma unroll
    for (int q = 0; q < 4; ++q) v[q] = factor == Factor(0) ? 0.0f : v[q];
  }
  int c = __builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[1], 0, false);
  c = __builtin_amdgcn_cvt_pk_fp8_f32(v[2], v[3], c, true);
  if (!kSome || own.all()) {
    *reinterpret_cast<code4_any *>(p) = uint32_t(c);
  } else {
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (own.has(uint32_t(q))) reinterpret_cast<uint8_t *>(p)[q] = uint8_t(c >> (8 * q));
  }
}

// 1 / sqrt(v): the hardware's first 23 bits or so and a Newton step, which leaves
// far less than fp32 keeps.  (A division and a root in fp64 take ten times the
// instructions, which rows of 64 or 128 elements feel.)
__device__ __forceinline__ double inverse_root(double v) {
  const double r = __builtin_amdgcn_rsq(v);
  const double s = fma(r, fma(-0.5 * v * r, r, 0.5), r);
  return s == s ? s : r;  // of 0 and infinity: the first value
}

template <int DT, int L, int P, int M>
__device__ __forceinline__ void load_x(Raw (&x)[P], const char *p, const uint32_t (&el)[P],
                                       const Own (&own)[P]) {
#pragma unroll
  for (int i = 0; i < P; ++i) {
    if constexpr (M != kSplit) {
      x[i] = Stored<DT>::template four<false>(p + int64_t(int32_t(el[i])) * Stored<DT>::kSize);
    } else {
      x[i] = Raw{{0u, 0u, 0u, 0u}};
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (own[i].has(uint32_t(q)))
          Stored<DT>::one(x[i], q, p + (el[i] + uint32_t(q)) * Stored<DT>::kSize);
    }
  }
}

template <int DT, int P, int M, bool kStream = false>
__device__ __forceinline__ void store_rows(void *to, uint64_t r0, const Four (&x)[P],
                                           const uint32_t (&el)[P], const Own (&own)[P]) {
  char *p = static_cast<char *>(to) + r0 * Stored<DT>::kSize;
#pragma unroll
  for (int i = 0; i < P; ++i)
    if (own[i].hi)
      store_four<DT, M != kEven, kStream>(p + int64_t(int32_t(el[i])) * Stored<DT>::kSize, x[i], own[i]);
}

// sum = x_in + `unit` times the sources' sum, kept where that is asked for.
template <int DT, int P, int M>
__device__ __forceinline__ void add_rows(double (&sum)[P][4], double unit, const Raw (&x0)[P],
                                         void *to, uint64_t r0, const uint32_t (&el)[P],
                                         const Own (&own)[P]) {
  Four x[P];
#pragma unroll
  for (int i = 0; i < P; ++i) {
    x[i] = Stored<DT>::values(x0[i]);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      sum[i][q] = fma(sum[i][q], unit, double(x[i].v[q]));
      x[i].v[q] = float(sum[i][q]);
    }
  }
  if (to) store_rows<DT, P, M, true>(to, r0, x, el, own);
}

// One pass: L threads hold a row in registers, P times four elements each (thread
// t's i-th four is elements (i L + t) * 4 on), so that x is formed, summed and
// normed without being read again; B sources are loaded ahead of their sums.
// Bound by HBM: n sources and x_in read, x_out and y written.  x, its mean and
// squares and the product with the row's factor are fp64, whose sums neither
// overflow nor cancel, so y is rounded to fp32 once before its gain and shift:
// an 8-bit code then flips beside a tie less often than it would by an fp32
// chain.  (All of it in fp32 for 16- and 8-bit sources: 0 to 9% less time; 16384 x
// 1152, one bf16 source, layer norm: 27.8 us for 29.6.)  Sources carry the
// non-temporal hint, and so does x_out, which is read a whole block later; x_in
// may be in a cache still, and y is read next.  Measured on MI355X:
//   8192 x 1152, 6 bf16 entries into MXFP8: 33.0 us, 6.0 TB/s (39.7 without the
//   hints; 6 MXINT8 entries 29.6, MXFP8 27.6); 16384 x 1152, layer norm of 4 fp32
//   entries: 73.9 us, 6.4 TB/s (88); 5003 x 1155 in fp16, a scale a row: 11.3 us.
template <class Src, int L, int P, int B, int M>
__global__ __launch_bounds__(L < 256 ? 256 : L) void norm_kernel(NormArgs a) {
  constexpr int kThreads = L < 256 ? 256 : L, kWaves = L > 64 ? L / 64 : 1;
  __shared__ double sums[kWaves][3];
  __shared__ uint32_t tops[kWaves];
  const uint32_t t = threadIdx.x % uint32_t(L);
  uint32_t row = blockIdx.x * uint32_t(kThreads / L) + threadIdx.x / uint32_t(L);
  if constexpr (L >= 64) row = __builtin_amdgcn_readfirstlane(row);
  if (row >= a.rows) return;  // a whole row's threads; only L < 256, which meets no barrier
  const uint64_t r0 = uint64_t(row) * a.dim;
  uint32_t el[P];  // first element of each four (kOdd: may lie before the row)
  Own own[P];
#pragma unroll
  for (int i = 0; i < P; ++i) {
    const uint32_t e = (uint32_t(i) * L + t) * 4u;
    own[i] = {0u, 4u};
    if (i == P - 1)  // the others end within the row: P is the least that holds it
      own[i].hi = e < a.dim ? (M == kEven || a.dim - e >= 4u ? 4u : a.dim - e) : 0u;
    el[i] = own[i].hi ? e : 0u;
    if (M == kOdd && i == P - 1) {
      // elements from the row's first to the last row's last
      const uint64_t left = uint64_t(a.rows - row) * a.dim;
      if (uint64_t(el[i]) + 4u > left) {
        const uint32_t by = el[i] + 4u - uint32_t(left);
        el[i] -= by;
        own[i].lo = own[i].hi ? by : 0u;
        own[i].hi = own[i].hi ? own[i].hi + by : 0u;
      }
    }
  }
  const RowAt from = Src::row(a, a.first + r0);
  typename Src::At at[P];
  if constexpr (M == kEven) {
#pragma unroll
    for (int i = 0; i < P; ++i) at[i] = Src::at(a, from, el[i]);
  }
  double acc[P][4];
#pragma unroll
  for (int i = 0; i < P; ++i)
#pragma unroll
    for (int q = 0; q < 4; ++q) acc[i][q] = -0.0;  // the sum of nothing: x + -0.0 is x, -0.0 too
  Raw x0[P];
#pragma unroll
  for (int i = 0; i < P; ++i) x0[i] = Raw{{0u, 0u, 0u, 0u}};
  if (a.x_in) {
    const char *p = static_cast<const char *>(a.x_in);
    if (a.x_dtype == CHEB_F32) load_x<CHEB_F32, L, P, M>(x0, p + r0 * 4u, el, own);
    else load_x<CHEB_BF16, L, P, M>(x0, p + r0 * 2u, el, own);
  }
  for (int k = 0; k < a.n; k += B) {
    typename Src::Held s[B][P];
#pragma unroll
    for (int j = 0; j < B; ++j)
      if (k + j < a.n) {
#pragma unroll
        for (int i = 0; i < P; ++i) {
          if constexpr (M == kEven) {
            s[j][i] = Src::four(a, k + j, from, at[i]);
          } else if constexpr (M == kOdd) {
            if constexpr (Src::kAnyPlace)
              s[j][i] = Src::Type::template four<false>(
                  reinterpret_cast<const char *>(a.base[k + j] + from.rb) +
                  int64_t(int32_t(el[i])) * Src::Type::kSize);
          } else {
            uint32_t e = el[i];
            asm volatile("" : "+v"(e));  // places formed anew for each source, not kept for all
            s[j][i] = Src::some(a, k + j, from, e, own[i]);
          }
        }
      }
#pragma unroll
    for (int j = 0; j < B; ++j)
      if (k + j < a.n) {
        const double w = a.w[k + j];
#pragma unroll
        for (int i = 0; i < P; ++i) Src::template add<M>(acc[i], w, s[j][i]);
      }
  }
  if (a.x_dtype == CHEB_F32) add_rows<CHEB_F32, P, M>(acc, 1.0 / Src::kSum, x0, a.x_out, r0, el, own);
  else if (a.x_dtype == CHEB_BF16) add_rows<CHEB_BF16, P, M>(acc, 1.0 / Src::kSum, x0, a.x_out, r0, el, own);
  else add_rows<CHEB_F16, P, M>(acc, 1.0 / Src::kSum, x0, a.x_out, r0, el, own);
  Four x[P];
  constexpr int kLanes = L < 64 ? L : 64;
  const auto add = [](double u, double v) { return u + v; };
  double var = 0.0;
  if (!a.layer) {
    double squares = 0.0;
#pragma unroll
    for (int i = 0; i < P; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const double d = own[i].has(uint32_t(q)) ? acc[i][q] : 0.0;
        squares = fma(d, d, squares);
      }
    squares = join_lanes<kLanes>(squares, add);
    if constexpr (kWaves > 1) {
      if ((threadIdx.x & 63u) == 0) sums[threadIdx.x >> 6][0] = squares;
      __syncthreads();
      squares = 0.0;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) squares += sums[w][0];
    }
    var = squares * a.inv_dim;
  } else {
    // Sums about the row's first element, so that one pass gives the mean and
    // the squares about it: x - x_0 loses nothing in fp64 that matters to x.
    double f = 0.0;
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (uint32_t(q) == own[0].lo) f = acc[0][q];
    double about = __shfl(f, 0, kLanes);
    if constexpr (kWaves > 1) {
      if (threadIdx.x == 0) sums[0][2] = about;
      __syncthreads();
      about = sums[0][2];
    }
    double sum = 0.0, squares = 0.0;
#pragma unroll
    for (int i = 0; i < P; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const double d = own[i].has(uint32_t(q)) ? acc[i][q] - about : 0.0;
        sum += d;
        squares = fma(d, d, squares);
      }
    squares = join_lanes<kLanes>(squares, add);
    sum = join_lanes<kLanes>(sum, add);
    if constexpr (kWaves > 1) {
      if ((threadIdx.x & 63u) == 0) {
        sums[threadIdx.x >> 6][0] = sum;
        sums[threadIdx.x >> 6][1] = squares;
      }
      __syncthreads();
      sum = squares = 0.0;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        sum += sums[w][0];
        squares += sums[w][1];
      }
    }
    const double off = sum * a.inv_dim, mean = about + off;
    var = fma(-off, off, squares * a.inv_dim);
    if (var < 0.0) var = 0.0;  // by rounding; a NaN stays
#pragma unroll
    for (int i = 0; i < P; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q) acc[i][q] -= mean;
  }
  const double r = inverse_root(var + a.eps);
#pragma unroll
  for (int i = 0; i < P; ++i)
#pragma unroll
    for (int q = 0; q < 4; ++q) x[i].v[q] = float(acc[i][q] * r);
  if (a.gain || a.shift) {
    uint32_t group = __umulhi(row, a.group_inverse);  // row / rows_per_group, or one less
    if (row - group * a.rows_per_group >= a.rows_per_group) ++group;
    const uint64_t g0 = uint64_t(group) * a.dim;
    const auto row_of = [&](const float *p, Four (&g)[P]) {
#pragma unroll
      for (int i = 0; i < P; ++i) {
        const float *e = p + g0 + int64_t(int32_t(el[i]));
        if constexpr (M == kEven) {
          g[i] = Stored<CHEB_F32>::values(
              Stored<CHEB_F32>::four<false>(reinterpret_cast<const char *>(e)));
        } else {
#pragma unroll
          for (int q = 0; q < 4; ++q) g[i].v[q] = own[i].has(uint32_t(q)) ? e[q] : 0.0f;
        }
      }
    };
    Four g[P], b[P];
    if (a.gain && a.shift) {
      row_of(a.gain, g);
      row_of(a.shift, b);
#pragma unroll
      for (int i = 0; i < P; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q) x[i].v[q] = fmaf(x[i].v[q], g[i].v[q], b[i].v[q]);
    } else if (a.gain) {
      row_of(a.gain, g);
#pragma unroll
      for (int i = 0; i < P; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q) x[i].v[q] *= g[i].v[q];
    } else {
      row_of(a.shift, b);
#pragma unroll
      for (int i = 0; i < P; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q) x[i].v[q] += b[i].v[q];
    }
  }
  const auto highest = [](uint32_t u, uint32_t v) { return max(u, v); };
  const auto magnitude = [&](int i) {
    uint32_t m = 0;
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (own[i].has(uint32_t(q))) m = max(m, __float_as_uint(x[i].v[q]) & 0x7fffffffu);
    return m;
  };
  char *codes = static_cast<char *>(a.y) + r0;
  if (a.out_format == CHEB_OUT_MXFP8) {
    const uint32_t width = (a.dim + 31u) / 32u;
    uint8_t *scales = static_cast<uint8_t *>(a.y_scale) + uint64_t(row) * width;
#pragma unroll
    for (int i = 0; i < P; ++i) {
      const Group of = group_of<E4m3Fmt>(join_lanes<8>(magnitude(i), highest));
      if (own[i].hi) {
        store_codes<M != kEven>(codes + int64_t(int32_t(el[i])), x[i], of.factor, own[i]);
        if ((t & 7u) == 0) scales[(uint32_t(i) * L + t) / 8u] = uint8_t(of.scale);
      }
    }
  } else if (a.out_format == CHEB_OUT_FP8_ROW) {
    uint32_t bits = 0;
#pragma unroll
    for (int i = 0; i < P; ++i) bits = max(bits, magnitude(i));
    bits = join_lanes<kLanes>(bits, highest);
    if constexpr (kWaves > 1) {
      if ((threadIdx.x & 63u) == 0) tops[threadIdx.x >> 6] = bits;
      __syncthreads();
      bits = 0u;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) bits = max(bits, tops[w]);
    }
    float scale = 1.0f;
    double factor = 1.0;
    if (bits >= 0x7f800000u) {
      scale = __uint_as_float(0x7fc00000u);
      factor = 0.0;
    } else if (bits != 0u) {
      scale = fmaxf(__uint_as_float(bits) / 448.0f, 0x1p-126f);
      factor = 1.0 / double(scale);
    }
    if (t == 0) static_cast<float *>(a.y_scale)[row] = scale;
#pragma unroll
    for (int i = 0; i < P; ++i)
      if (own[i].hi) store_codes<M != kEven>(codes + int64_t(int32_t(el[i])), x[i], factor, own[i]);
  } else if (a.out_format == CHEB_F32) {
    store_rows<CHEB_F32, P, M>(a.y, r0, x, el, own);
  } else if (a.out_format == CHEB_BF16) {
    store_rows<CHEB_BF16, P, M>(a.y, r0, x, el, own);
  } else {
    store_rows<CHEB_F16, P, M>(a.y, r0, x, el, own);
  }
}

template <class Src, int L, int P>
hipError_t launch_shape(const NormArgs &a, hipStream_t s) {
  constexpr uint32_t kThreads = L < 256 ? 256 : L, kRows = kThreads / L;
  constexpr int B = 2;
  const bool placed = a.chunked || !Src::kAnyPlace;  // fours must not cross
  const bool even = a.dim % 4u == 0 && (!placed || a.first % 4u == 0);
  auto kernel = norm_kernel<Src, L, P, B, kEven>;
  if (!even) {
    kernel = norm_kernel<Src, L, P, 1, kSplit>;
    if constexpr (Src::kAnyPlace)
      if (!placed && uint64_t(a.rows) * a.dim >= 4u) kernel = norm_kernel<Src, L, P, B, kOdd>;
  }
  hipLaunchKernelGGL(kernel, dim3((a.rows + kRows - 1) / kRows), dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

// The fewest threads that hold a row in at most six times four elements each, so
// that a wave's worth of them needs no barrier and short rows share a wave, and
// exactly as many fours.  (18.9 M elements of bf16 in rows of 64, 128 and 256:
// 26 to 29 us, 32 to 33 with one four a thread.  Rows of 1028 to 3060 on 128
// threads: 3% less to 5% more, so they take 64 or 256.)
template <class Src>
hipError_t launch_src(const NormArgs &a, hipStream_t s) {
  const uint32_t fours = (a.dim + 3u) / 4u;
  if (fours <= 32) {
    switch ((fours + 7u) / 8u) {
      case 1: return launch_shape<Src, 8, 1>(a, s);
      case 2: return launch_shape<Src, 8, 2>(a, s);
      case 3: return launch_shape<Src, 8, 3>(a, s);
      default: return launch_shape<Src, 8, 4>(a, s);
    }
  }
  if (fours <= 48) return launch_shape<Src, 16, 3>(a, s);
  if (fours <= 64) return launch_shape<Src, 16, 4>(a, s);
  if (fours <= 96) return launch_shape<Src, 32, 3>(a, s);
  if (fours <= 128) return launch_shape<Src, 32, 4>(a, s);
  switch ((fours + 63u) / 64u) {
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
    case 5: return launch_shape<Src, 256, 5>(a, s);
    case 6: return launch_shape<Src, 256, 6>(a, s);
    default: break;
  }
  switch ((fours + 1023u) / 1024u) {
    case 2: return launch_shape<Src, 1024, 2>(a, s);
    case 3: return launch_shape<Src, 1024, 3>(a, s);
    default: return launch_shape<Src, 1024, 4>(a, s);
  }
}

}  // namespace

int launch_norm(const NormSources &from, const cheb_norm &n, hipStream_t stream) {
  NormArgs a;
  memset(&a, 0, sizeof a);
  const double unit = from.quant == CHEB_QUANT_MXINT8  ? Int8Fmt::kDouble * Int8Fmt::kSum
                      : from.quant == CHEB_QUANT_MXFP8 ? E4m3Fmt::kDouble * E4m3Fmt::kSum
                                                       : 1.0;
  for (int k = 0; k < from.n; ++k) {
    const bool coded = from.quant != CHEB_QUANT_NONE;
    a.base[k] = reinterpret_cast<uint64_t>(coded ? from.src[k].codes : from.base[k]);
    a.scales[k] = coded ? reinterpret_cast<uint64_t>(from.src[k].scales) : 0u;
    a.w[k] = from.w[k] * unit;
  }
  a.first = uint64_t(from.first);
  a.n = from.n;
  a.chunked = from.super_vecs != kChunkVecs;
  a.super = uint32_t(from.super_vecs) * 16u;
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
  a.group_inverse = a.rows_per_group == 1 ? UINT32_MAX
                                          : uint32_t((uint64_t(1) << 32) / a.rows_per_group);
  a.layer = n.kind == CHEB_NORM_LAYER;
  a.x_dtype = n.x_dtype;
  a.out_format = n.out_format;
  hipError_t e;
  if (from.quant != CHEB_QUANT_NONE) {
    a.super = uint32_t(from.place.code_super);
    a.scale_super = uint32_t(from.place.scale_super);
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
