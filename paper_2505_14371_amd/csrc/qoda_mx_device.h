// Device code of microscaled matrices: scales and codes of a block, and where they lie.
#pragma once

#include "qoda_matrices.h"
#include "qoda_operators_device.h"

namespace qoda {

namespace {

typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
typedef float v2f __attribute__((ext_vector_type(2)));

// The place in 256 bytes of scales of a row (of 64) and a block (of four).
__device__ __forceinline__ int scale_place(int row, int block) {
  return 64 * block + 16 * ((row >> 3) & 3) + 4 * (row & 3) + 2 * (row >> 5) + ((row >> 2) & 1);
}

// The byte of a block's scale, e + 127, from the bits of its largest magnitude.  To nearest e is floor(log2 m) - 2; stochastically one more where m is
// over 1.5 powers of two: 6 is 1.5 times 4.
__device__ __forceinline__ u32 scale_byte(u32 most, bool stochastic) {
  if (most >= 0x7F800000u) return 255u;
  const int e = (int)(most >> 23) - 2 + (stochastic && (most & 0x7FFFFFu) > 0x400000u ? 1 : 0);
  return e > 0 ? (u32)e : 0u;
}
// ... as the conversions take it: 2^e
__device__ __forceinline__ float scale_of(u32 byte) { return __uint_as_float(byte == 0 ? 0x400000u : byte << 23); }

// The bits of the largest magnitude among eight entries (those of a NaN are above infinity's).
template <class T>
__device__ __forceinline__ u32 most_of(const Eight<T> &v) {
  u32 m = 0;
#pragma unroll
  for (int j = 0; j < Eight<T>::kWords; ++j) {
    const u32 w = v.w[j / 4][j % 4];
    if constexpr (sizeof(T) == 4) {
      const u32 a = w & 0x7FFFFFFFu;
      m = m > a ? m : a;
    } else {
      const u32 lo = w << 16 & 0x7FFFFFFFu, hi = w & 0x7FFF0000u;
      m = m > lo ? m : lo;
      m = m > hi ? m : hi;
    }
  }
  return m;
}

// Codes of eight entries to nearest, by the conversion instruction: ties to even, above 6 to 6.
template <class T>
__device__ __forceinline__ u32 codes_nearest(const Eight<T> &v, float scale) {
  u32 r = 0;
  if constexpr (sizeof(T) == 4) {
    float f[8];
    v.get(f);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, f[0], f[1], scale, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, f[2], f[3], scale, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, f[4], f[5], scale, 2);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, f[6], f[7], scale, 3);
  } else {
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(v2bf, (u32)v.w[0][0]), scale, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(v2bf, (u32)v.w[0][1]), scale, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(v2bf, (u32)v.w[0][2]), scale, 2);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(v2bf, (u32)v.w[0][3]), scale, 3);
  }
  return r;
}

// Stochastic codes.  An entry's place among the codes in steps of 2^-22: with v = |x| / 2^e that is v 2^23 below 1, where neighbours are 1/2 apart, and from 1
// on v's own bits (the exponent and one bit of the mantissa are the code), less those of 1/2.  Below 1 the one is between the other and 2^23, and from 1
// on the other way round: the middle one of the three.  What is below a step is cut off, which changes no comparison with a lot: 65536 (v - q) / d >=
// lot + 1/2 is, in the place's lower 22 bits, place >= 64 lot + 32, and then 4 place + 2^24 - 256 lot - 128 has the next code in its upper byte.  Codes and signs
// are put together four at a time.  (An entry at a time 16384 x 8192 of bf16 took 94 us for the transpose.)
__device__ __forceinline__ u32 code_of(u32 x, int to_place, u32 lot) {   // sign in bit 31, code in bits 24 to 26; lot: 256 (65535 - lot) + 128
  const float v = ldexpf(__uint_as_float(x & 0x7FFFFFFFu), to_place);    // times 2^23
  const int low = (int)(u32)v, high = (int)(__float_as_uint(v) - (23u << 23) - 0x3F000000u);
  const int least = low < high ? low : high, most = low < high ? high : low, under = most < 0x800000 ? most : 0x800000;
  const u32 place = (u32)(least > under ? least : under);
  return ((place << 2) + lot & 0x7FFFFFFFu) | (x & 0x80000000u);
}
// ... of the eight entries 8 block .. 8 block + 7 of a row, the bits of fp32 numbers.
__device__ __forceinline__ u32 codes_stochastic(const u32 (&x)[8], u32 byte, u32 row, u32 block, const MxRounding &a) {
  u32 w[4], t[8];
  philox4x32_10(block, row, a.o0, a.o1, a.k0, a.k1, w);
  const int to_place = 150 - (int)byte;
#pragma unroll
  for (int j = 0; j < 8; ++j) t[j] = code_of(x[j], to_place, __builtin_amdgcn_perm(~w[j & 3], 128u, j < 4 ? 0x0C050400u : 0x0C070600u));
  const u32 even = __builtin_amdgcn_perm(t[2], t[0], 0x0C0C0703u) | __builtin_amdgcn_perm(t[6], t[4], 0x07030C0Cu);
  const u32 odd = __builtin_amdgcn_perm(t[3], t[1], 0x0C0C0703u) | __builtin_amdgcn_perm(t[7], t[5], 0x07030C0Cu);
  return (even & 0x07070707u) | (even >> 4 & 0x08080808u) | (odd & 0x07070707u) << 4 | (odd & 0x80808080u);
}

// What eight codes of a block stand for.
__device__ __forceinline__ void values_of(u32 codes, u32 byte, float (&v)[8]) {
  const float scale = scale_of(byte == 255u ? 127u : byte);
  const v2f a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 1),
            c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 3);
  v[0] = a[0], v[1] = a[1], v[2] = b[0], v[3] = b[1], v[4] = c[0], v[5] = c[1], v[6] = d[0], v[7] = d[1];
  if (byte == 255u)
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = __uint_as_float(0x7FC00000u);
}

}  // namespace

}  // namespace qoda
