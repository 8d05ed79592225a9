// Device code of the 8-bit formats: codes and scales from the values of a
// group, and values from codes.
#pragma once

#include <hip/hip_runtime.h>

#include <stdint.h>
#include <string.h>

namespace cheb {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

// The tile of a block where N neighbouring tiles share a line of scales: they
// go to one XCD, whose L2 then reads the line once (blocks are dealt to the
// eight XCDs in turn; tiles past the last whole 8 N keep their order).
template <uint32_t N>
__device__ __forceinline__ uint32_t line_tile(uint32_t block, uint32_t blocks) {
  if (N == 1 || block >= blocks / (8u * N) * (8u * N)) return block;
  const uint32_t q = block >> 3;
  return (q / N * 8u + (block & 7u)) * N + q % N;
}

// A group's scale byte (2^(scale - 127), 255: NaN) and the factor that takes
// values to codes (0 for a group that is not finite: its codes are 0, and 0
// times the scale's infinity, 255 << 23, is NaN).
struct Group {
  uint32_t scale;
  float factor;
  bool top;  // its largest value may round past the largest code
};

// The largest of four neighbouring lanes' values, by two exchanges.
__device__ __forceinline__ uint32_t quad_max(uint32_t m) {
  m = max(m, uint32_t(__builtin_amdgcn_mov_dpp(int(m), 0xB1, 0xF, 0xF, true)));  // 1 0 3 2
  return max(m, uint32_t(__builtin_amdgcn_mov_dpp(int(m), 0x4E, 0xF, 0xF, true)));  // 2 3 0 1
}

// From the bits of the group's largest magnitude a (fp32): the exponent e, the
// least with a <= L 2^e, is a's own less L's, one more where a's fraction
// exceeds L's.
template <class Fmt>
__device__ __forceinline__ Group group_of(uint32_t a) {
  const int e = int((a + (0x7fffffu - Fmt::kLimitFraction)) >> 23) - 127 - Fmt::kLimitExponent;
  const int kept = min(max(e, -120), 127);
  Group g;
  g.top = e > 127;
  g.scale = uint32_t(kept + 127);
  g.factor = __uint_as_float(uint32_t(127 + Fmt::kShift - kept) << 23);
  if (a >= 0x7f800000u) {
    g.scale = 255u;
    g.factor = 0.0f;
    g.top = true;
  }
  return g;
}

// A lane's eight codes.  decode() gives halves, pairs of exact fp16 numbers,
// which v_fma_mix_f32 takes as they are; a code counts kUnit of its scale times
// its half.  The conversions from integers and fp8 run at a quarter of the rate
// of other instructions and would bound the sums over several entries; these
// take full-rate ones.
struct Halves {
  f16x2 h[4];
  __device__ __forceinline__ float operator[](int i) const { return float(h[i >> 1][i & 1]); }
};

// The same codes as fp64 numbers, for sums of more bits: doubles() builds them
// from their bits, as fp64 conversions run at a quarter of the rate too.  One
// counts kDouble of its scale.  A sum of them is held as kSum of its value:
// weights, below 2^128, go in times kDouble kSum, which keeps products with a
// scale within fp64's range.
__device__ __forceinline__ double high_word(uint32_t w) {
  return __builtin_bit_cast(double, uint64_t(w) << 32);
}

struct Int8Fmt {
  static constexpr uint32_t kLimitFraction = 0x7e0000u;  // 127/64 = 1.984375
  static constexpr int kLimitExponent = 0;
  static constexpr int kShift = 6;        // a code counts 64ths of the scale
  static constexpr double kUnit = 0x1p-6;
  static constexpr int kMostScale = 127;  // 2^127
  static constexpr double kDouble = kUnit, kSum = 1.0;

  // The stored byte is the code plus 128.  Adding 1.5 2^23 + 128 rounds to the
  // nearest whole number, ties to even, and leaves it as the low byte of the
  // sum's bits (x factor is exact: a power of two).
  __device__ __forceinline__ static u32x2 encode(const float (&x)[8], const Group &g) {
    constexpr float kWhole = 0x1.8p23f + 128.0f;
    uint32_t t[8];
    if (__builtin_expect(__ballot(g.top) != 0ull, 0)) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float v = g.factor == 0.0f ? 0.0f : fminf(fmaxf(x[i] * g.factor, -127.0f), 127.0f);
        t[i] = __float_as_uint(v + kWhole);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) t[i] = __float_as_uint(fmaf(x[i], g.factor, kWhole));
    }
    u32x2 r;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t lo = __builtin_amdgcn_perm(t[4 * h + 1], t[4 * h], 0x0c0c0400u);
      const uint32_t hi = __builtin_amdgcn_perm(t[4 * h + 3], t[4 * h + 2], 0x04000c0cu);
      r[h] = lo | hi;
    }
    return r;
  }

  // 0x64 above a byte b is the fp16 number 1024 + b.
  __device__ __forceinline__ static Halves decode(u32x2 v) {
    const f16x2 off = {_Float16(-1152.0f), _Float16(-1152.0f)};
    Halves q;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      q.h[i] = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, v[i >> 1],
                                                               i & 1 ? 0x04030402u : 0x04010400u)) +
               off;
    return q;
  }

  // A byte b eight places up in the high word of 2^12 is the number 4096 + b.
  __device__ __forceinline__ static void doubles(u32x2 v, double (&q)[8]) {
    constexpr uint32_t kByte[4] = {0x07060004u, 0x07060104u, 0x07060204u, 0x07060304u};
#pragma unroll
    for (int i = 0; i < 8; ++i)
      q[i] = high_word(__builtin_amdgcn_perm(0x40b00000u, v[i >> 2], kByte[i & 3])) - 4224.0;
  }
};

struct E4m3Fmt {
  static constexpr uint32_t kLimitFraction = 0x600000u;  // 448 = 1.75 2^8
  static constexpr int kLimitExponent = 8;
  static constexpr int kShift = 0;
  static constexpr double kUnit = 1.0;
  static constexpr int kMostScale = 120;
  static constexpr double kDouble = 0x1p1016, kSum = 0x1p-248;

  __device__ __forceinline__ static u32x2 encode(const float (&x)[8], const Group &g) {
    float v[8];
    if (__builtin_expect(__ballot(g.top) != 0ull, 0)) {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = g.factor == 0.0f ? 0.0f : x[i] * g.factor;
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = x[i] * g.factor;
    }
    u32x2 r;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      int p = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * h], v[4 * h + 1], 0, false);
      p = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * h + 2], v[4 * h + 3], p, true);
      r[h] = uint32_t(p);
    }
    return r;
  }

  // The code's exponent and fraction one place below a half's sign are the
  // fp16 number of 2^-8 its value (exponents are biased by 7 and 15), fp16's
  // small numbers being e4m3's.  Codes are never NaN.  The 2^8 is not left to
  // the weights: with a scale of 2^120 they would overflow.
  __device__ __forceinline__ static Halves decode(u32x2 v) {
    const f16x2 up = {_Float16(256.0f), _Float16(256.0f)};
    Halves q;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t p =
          __builtin_amdgcn_perm(0u, v[i >> 1], i & 1 ? 0x030c020cu : 0x010c000cu);
      q.h[i] = __builtin_bit_cast(f16x2, (p & 0x80008000u) | (p >> 1 & 0x3fff3fffu)) * up;
    }
    return q;
  }

  // The code's exponent and fraction at the end of fp64's exponent are the
  // number of 2^-1016 its value, fp64's small numbers being e4m3's.  The 2^1016
  // is left to the weights (0.9 of the time of a product here).
  __device__ __forceinline__ static void doubles(u32x2 v, double (&q)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int32_t p = int32_t(v[i >> 2] << (24 - 8 * (i & 3)));  // below the code: others' bits
      q[i] = high_word(uint32_t(p >> 7) & 0x80fe0000u);
    }
  }
};

// ---- eight source elements of a lane: their bits' largest magnitude, and
// their values.  load_some() takes the first n of them and zeros.

__device__ __forceinline__ uint32_t top_of_halves(u32x4 v) {
  u16x2 m = __builtin_bit_cast(u16x2, v[0] & 0x7fff7fffu);
#pragma unroll
  for (int q = 1; q < 4; ++q)
    m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, v[q] & 0x7fff7fffu));
  return max(uint32_t(m.x), uint32_t(m.y));
}

__device__ __forceinline__ u32x4 some_halves(const uint16_t *p, uint64_t n) {
  uint16_t t[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) t[i] = uint64_t(i) < n ? p[i] : uint16_t(0);
  u32x4 r;
  memcpy(&r, t, 16);
  return r;
}

struct Bf16Src {
  using E = uint16_t;
  using Raw = u32x4;
  __device__ __forceinline__ static Raw load(const E *p) {
    return __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(p));
  }
  __device__ __forceinline__ static Raw load_some(const E *p, uint64_t n) {
    return some_halves(p, n);
  }
  __device__ __forceinline__ static uint32_t top(const Raw &v) { return top_of_halves(v); }
  __device__ __forceinline__ static uint32_t magnitude(uint32_t t) { return t << 16; }
  __device__ __forceinline__ static void values(const Raw &v, float (&x)[8]) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      x[2 * q] = __uint_as_float(v[q] << 16);
      x[2 * q + 1] = __uint_as_float(v[q] & 0xffff0000u);
    }
  }
};

struct F16Src {
  using E = uint16_t;
  using Raw = u32x4;
  __device__ __forceinline__ static Raw load(const E *p) { return Bf16Src::load(p); }
  __device__ __forceinline__ static Raw load_some(const E *p, uint64_t n) {
    return some_halves(p, n);
  }
  __device__ __forceinline__ static uint32_t top(const Raw &v) { return top_of_halves(v); }
  __device__ __forceinline__ static uint32_t magnitude(uint32_t t) {
    return __float_as_uint(float(__builtin_bit_cast(_Float16, uint16_t(t))));
  }
  __device__ __forceinline__ static void values(const Raw &v, float (&x)[8]) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      x[2 * q] = float(__builtin_bit_cast(_Float16, uint16_t(v[q])));
      x[2 * q + 1] = float(__builtin_bit_cast(_Float16, uint16_t(v[q] >> 16)));
    }
  }
};

struct F32Src {
  using E = float;
  struct Raw {
    u32x4 v[2];
  };
  __device__ __forceinline__ static Raw load(const E *p) {
    const u32x4 *q = reinterpret_cast<const u32x4 *>(p);
    return {{q[0], q[1]}};
  }
  __device__ __forceinline__ static Raw load_some(const E *p, uint64_t n) {
    Raw r;
#pragma unroll
    for (int i = 0; i < 8; ++i) r.v[i >> 2][i & 3] = __float_as_uint(uint64_t(i) < n ? p[i] : 0.0f);
    return r;
  }
  __device__ __forceinline__ static uint32_t top(const Raw &r) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, r.v[i >> 2][i & 3] & 0x7fffffffu);
    return m;
  }
  __device__ __forceinline__ static uint32_t magnitude(uint32_t t) { return t; }
  __device__ __forceinline__ static void values(const Raw &r, float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(r.v[i >> 2][i & 3]);
  }
};

}  // namespace cheb
