// 8-bit rows: the one format that the quantisers, the 8-bit products and the 8-bit broadcast cache share.
//
// A matrix [R, K] is e4m3 bytes (4 exponent bits, 3 mantissa bits, largest value 448, no infinities) in rows of `ld` bytes, zero
// behind column K up to the next multiple of 128, and one scale for 128 columns of a row: an exponent byte b that stands for
// 2^(b - 127).  A value is e4m3 * scale.  Why powers of two: they are what the scaled matrix instruction of gfx950 multiplies by
// itself (its own blocks are 32 columns; four of them get the same byte), so that a scale per block costs the products nothing,
// dividing by one is exact, and a quantised value is one rounding, at most 2^-4 of the value (of 2^-6 times the scale for values below
// that), off.  Against scales of 24 bits the largest value of a block lies in (224, 448] instead of at 448, which costs
// range and no precision.  Why whole 128-byte rows: a K slice of the product kernels is one cache line per row and needs no tail.
//
// Scale of a block: the smallest power of two, 2^-127 at least, for which the largest finite magnitude stays within 448.  Infinities and
// NaNs become NaN and do not count.
#pragma once
#include "mfma_util.hpp"

namespace pab {

typedef __attribute__((ext_vector_type(2))) unsigned u32x2;
typedef __attribute__((ext_vector_type(4))) unsigned u32x4;

// bits of |x|, 0 where x is not finite
__device__ __forceinline__ unsigned finite_bits(float x) {
  const unsigned a = __float_as_uint(x) & 0x7fffffffu;
  return a < 0x7f800000u ? a : 0u;
}

// exponent byte of a block whose largest magnitude has the bits `big`: 448 = 1.75 * 2^8, so the exponent less 8, one more past 1.75
__device__ __forceinline__ int q8_scale_byte(unsigned big) {
  return max((int)(big >> 23) - 8 + ((big & 0x7fffffu) > 0x600000u ? 1 : 0), 0);
}
// 1 / scale = 2^(127 - b), b at most 247
__device__ __forceinline__ float q8_inverse(int b) { return __uint_as_float((unsigned)(254 - b) << 23); }
// scale = 2^(b - 127); the lowest is a subnormal number, 255 stands for NaN
__device__ __forceinline__ float q8_scale(unsigned b) {
  return __uint_as_float(b == 255u ? 0x7fc00000u : b ? b << 23 : 0x00400000u);
}

// four values, already divided by the scale, as e4m3 (rounded to nearest, ties to even)
__device__ __forceinline__ unsigned pack_e4m3(float a, float b, float c, float d) {
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
}
// The largest finite magnitude among a lane's values, as bits, and infinities become NaN: maxima of three without a look at each value (they
// pass over NaNs), and only where that comes out infinite somewhere in the wavefront value by value.
template <int N>
__device__ __forceinline__ unsigned block_max(float (&x)[N][8]) {
  float m = 0.0f;
#pragma unroll
  for (int u = 0; u < N; ++u)
#pragma unroll
    for (int e = 0; e < 8; e += 2) m = fmaxf(fmaxf(m, fabsf(x[u][e])), fabsf(x[u][e + 1]));
  unsigned big = __float_as_uint(m);
  if (__any(big >= 0x7f800000u)) {
    big = 0;
#pragma unroll
    for (int u = 0; u < N; ++u)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        big = max(big, finite_bits(x[u][e]));
        if (!isfinite(x[u][e])) x[u][e] = __uint_as_float(0x7fc00000u);
      }
  }
  return big;
}

// largest of 16 neighbouring lanes, in all of them, by register moves
__device__ __forceinline__ unsigned max16(unsigned v) {
  v = max(v, (unsigned)__builtin_amdgcn_mov_dpp((int)v, 0xB1, 0xF, 0xF, true));    // lane ^ 1
  v = max(v, (unsigned)__builtin_amdgcn_mov_dpp((int)v, 0x4E, 0xF, 0xF, true));    // lane ^ 2
  v = max(v, (unsigned)__builtin_amdgcn_mov_dpp((int)v, 0x141, 0xF, 0xF, true));   // mirrored in half a row: the other four
  return max(v, (unsigned)__builtin_amdgcn_mov_dpp((int)v, 0x140, 0xF, 0xF, true));   // mirrored in the row: the other eight
}

// n / d for n < 2^31 by a high product: with 2^k <= d < 2^(k+1) and m = 2^(32+k) / d rounded up, m is off by less than d / 2^(32+k) of the
// quotient per unit of n, n d <= 2^(32+k) keeps it exact, and m fits 32 bits unless d is a power of two (then half of both; d = 1: n itself)
struct Divisor {
  unsigned d, m, k, one;
};
inline Divisor divisor(unsigned d) {
  if (d <= 1) return {1, 0, 0, ~0u};
  unsigned k = 31 - __builtin_clz(d);
  if ((d & (d - 1)) == 0) return {d, 0x80000000u, k - 1, 0};
  return {d, (unsigned)(((1ULL << (32 + k)) + d - 1) / d), k, 0};
}
__device__ __forceinline__ unsigned quotient(unsigned n, const Divisor &v) { return (__umulhi(n, v.m) + (n & v.one)) >> v.k; }

// eight values of a row from memory, as fp32, and back
__device__ __forceinline__ void load_row8(const bf16_t *p, float (&v)[8]) {
  const bf16x8 t = *reinterpret_cast<const bf16x8 *>(p);
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = (float)t[e];
}
__device__ __forceinline__ void load_row8(const float *p, float (&v)[8]) {
  const f32x4 a = *reinterpret_cast<const f32x4 *>(p), b = *reinterpret_cast<const f32x4 *>(p + 4);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    v[e] = a[e];
    v[4 + e] = b[e];
  }
}
__device__ __forceinline__ void store_row8(bf16_t *p, const float (&v)[8]) {
  bf16x8 t;
#pragma unroll
  for (int e = 0; e < 8; ++e) t[e] = (bf16_t)v[e];
  *reinterpret_cast<bf16x8 *>(p) = t;
}
__device__ __forceinline__ void store_row8(float *p, const float (&v)[8]) {
  *reinterpret_cast<f32x4 *>(p) = f32x4{v[0], v[1], v[2], v[3]};
  *reinterpret_cast<f32x4 *>(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
}

}  // namespace pab
