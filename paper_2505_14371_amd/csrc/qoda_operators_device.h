// Device code that the operators' kernels share: entries of the two types, activations and their derivatives, dropout's lots.
#pragma once

#include "qoda_operators.h"
#include "qoda_philox.h"

namespace qoda {

typedef unsigned short u16;
typedef unsigned int u32;

struct bf16 { u16 bits; };

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(bf16 v) { return __uint_as_float((u32)v.bits << 16); }
// to nearest even; a NaN stays one
__device__ __forceinline__ u32 bf16_bits(float v) {
  const __bf16 b = (__bf16)v;
  return __builtin_bit_cast(u16, b);
}
template <class T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ bf16 from_float<bf16>(float v) { return bf16{(u16)bf16_bits(v)}; }

constexpr float kSlope = 0.2f;   // of leaky_relu
constexpr float kLog2E = 1.4426950408889634f;

// The two factors of 1 - Phi(|z|) = erfc(|z| / sqrt 2) / 2 = q e with e = exp(-z^2 / 2), which is the density's factor too, so that gelu and its slope take
// one exponential and one reciprocal.  q is a polynomial in t = 1 / (1 + c |z|), fitted here (linear programming over 0 <= |z| <= 14.5), without its constant.
//   fp32: nine terms, off by 2e-8 of q at most, and corrected to first order for the rounding of t: dq/d|z| = |z| q - 1 / sqrt(2 pi).  gelu and its slope
//         of normal values are off by 3.4e-8 and 3.8e-8 in the square mean; with fp32's erf and exp they are by 3.9e-8 and 4.1e-8.
//   bf16: seven terms, off by 3e-8 at most (1.3e-7 with fp32's rounding) and by 4e-5 of q e at most: nothing beside the store's rounding, and little in
//         the fp32 sums that dweight and dbias are.
template <class T>
__device__ __forceinline__ void normal_tail(float z, float &q, float &e) {
  e = __builtin_amdgcn_exp2f(z * z * (-0.5f * kLog2E));
  if constexpr (sizeof(T) == 4) {
    constexpr float kC = 0.27f;
    const float a = fminf(fabsf(z), 16.0f), d = __builtin_fmaf(kC, a, 1.0f), t = __builtin_amdgcn_rcpf(d);   // e is 0 from 14.5 on
    q = __builtin_fmaf(0.028961099684238434f, t, -0.12648585438728333f);
    q = __builtin_fmaf(q, t, 0.16978614032268524f);
    q = __builtin_fmaf(q, t, -0.0692107304930687f);
    q = __builtin_fmaf(q, t, 0.10782559961080551f);
    q = __builtin_fmaf(q, t, 0.07204962521791458f);
    q = __builtin_fmaf(q, t, 0.10181060433387756f);
    q = __builtin_fmaf(q, t, 0.10754287242889404f);
    q = __builtin_fmaf(q, t, 0.10772065818309784f) * t;
    const float off = __builtin_fmaf(-d, t, 1.0f) - __builtin_fmaf(kC, a, 1.0f - d) * t;   // by how much of itself t is too small
    q = __builtin_fmaf(__builtin_fmaf(-a, q, 0.39894228040143268f) * off, d * (1.0f / kC), q);
  } else {
    const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.34f, fabsf(z), 1.0f));
    q = __builtin_fmaf(0.04579341039061546f, t, -0.20435094833374023f);
    q = __builtin_fmaf(q, t, 0.270133376121521f);
    q = __builtin_fmaf(q, t, -0.03557766228914261f);
    q = __builtin_fmaf(q, t, 0.15860435366630554f);
    q = __builtin_fmaf(q, t, 0.12934985756874084f);
    q = __builtin_fmaf(q, t, 0.13604764640331268f) * t;
  }
}

// Of a call whose entries are of type T.
template <class T, int ACT>
__device__ __forceinline__ float act(float z) {
  if constexpr (ACT == kActRelu) return z < 0.0f ? 0.0f : z;   // a NaN stays one
  if constexpr (ACT == kActLeakyRelu) return z > 0.0f ? z : kSlope * z;
  if constexpr (ACT == kActGelu) {
    float q, e;
    normal_tail<T>(z, q, e);
    return z * (z < 0.0f ? q * e : __builtin_fmaf(-q, e, 1.0f));
  }
  if constexpr (ACT == kActSilu) return z * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-kLog2E * z));
  return z;
}

template <class T, int ACT>
__device__ __forceinline__ float act_slope(float z) {
  if constexpr (ACT == kActRelu) return z > 0.0f ? 1.0f : 0.0f;
  if constexpr (ACT == kActLeakyRelu) return z > 0.0f ? 1.0f : kSlope;
  if constexpr (ACT == kActGelu) {
    float q, e;
    normal_tail<T>(z, q, e);
    // Phi + z phi: on the left q e - |z| e / sqrt(2 pi), on the right one less what it is at -z
    const float w = __builtin_fmaf(-0.39894228040143268f, fabsf(z), q);
    return z < 0.0f ? w * e : __builtin_fmaf(-w, e, 1.0f);
  }
  if constexpr (ACT == kActSilu) {
    const float s = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-kLog2E * z));
    return s * __builtin_fmaf(z, 1.0f - s, 1.0f);
  }
  return 1.0f;
}

// Dropout of the eight entries 8 block .. 8 block + 7 of a row.  A lot is compared where it lies, in the upper half of a word: lot >= threshold
// is lot << 16 > (threshold << 16) - 1, and what is below the lot does not change that.
__device__ __forceinline__ void drop8(const Drop &d, u32 row, u32 block, float (&v)[8]) {
  u32 w[4];
  philox4x32_10(block, row, d.o0, d.o1, d.k0, d.k1, w);
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = (j < 4 ? w[j & 3] << 16 : w[j & 3]) > d.limit ? v[j] * d.scale : 0.0f;
}

// Eight adjacent entries as they lie in memory, of which the first n exist (the others are read as 0 and not stored).  Words, so that
// they move 16 bytes at a time at any alignment.
typedef u32 v4u __attribute__((ext_vector_type(4)));
template <class T>
struct Eight {
  static constexpr int kWords = sizeof(T) * 2;
  v4u w[kWords / 4];
  // EVEN: n is at least 8 or not positive.  What handles the others costs registers even where it is not taken.
  template <bool EVEN = false>
  __device__ __forceinline__ void load(const T *p, int n) {
    if (EVEN ? n > 0 : n >= 8) {
#pragma unroll
      for (int q = 0; q < kWords / 4; ++q) __builtin_memcpy(&w[q], reinterpret_cast<const char *>(p) + 16 * q, 16);
    } else if constexpr (EVEN) {
#pragma unroll
      for (int q = 0; q < kWords / 4; ++q) w[q] = v4u{0, 0, 0, 0};
    } else {
      u32 e[8] = {};
      if (n > 0) {   // all at once, those beyond the end from the last one's place: a branch for each would wait for each
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const T *q = p + (j < n ? j : n - 1);
          if constexpr (sizeof(T) == 4) e[j] = __float_as_uint(*q);
          else e[j] = q->bits;
        }
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) e[j] = j < n ? e[j] : 0u;
#pragma unroll
      for (int j = 0; j < kWords; ++j) w[j / 4][j % 4] = sizeof(T) == 4 ? e[j] : e[2 * j % 8] | e[(2 * j + 1) % 8] << 16;
    }
  }
  __device__ __forceinline__ void get(float (&v)[8]) const {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if constexpr (sizeof(T) == 4) v[j] = __uint_as_float(w[j / 4][j % 4]);
      else v[j] = __uint_as_float(j & 1 ? w[0][j / 2] & 0xFFFF0000u : w[0][j / 2] << 16);
    }
  }
  __device__ __forceinline__ void set(const float (&v)[8]) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int j = 0; j < 8; ++j) w[j / 4][j % 4] = __float_as_uint(v[j]);
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) w[0][j] = bf16_bits(v[2 * j]) | bf16_bits(v[2 * j + 1]) << 16;
    }
  }
  template <bool EVEN = false>
  __device__ __forceinline__ void store(T *p, int n) const {
    if (EVEN ? n > 0 : n >= 8) {
#pragma unroll
      for (int q = 0; q < kWords / 4; ++q) __builtin_memcpy(reinterpret_cast<char *>(p) + 16 * q, &w[q], 16);
    } else if constexpr (!EVEN) {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (j < n) {
          if constexpr (sizeof(T) == 4) p[j] = __uint_as_float(w[j / 4][j % 4]);
          else p[j].bits = (u16)(w[0][j / 2] >> (16 * (j & 1)));
        }
    }
  }
};
template <bool EVEN = false, class T>
__device__ __forceinline__ void load8(const T *p, int n, float (&v)[8]) {
  Eight<T> r;
  r.template load<EVEN>(p, n);
  r.get(v);
}
template <bool EVEN = false, class T>
__device__ __forceinline__ void store8(T *p, int n, const float (&v)[8]) {
  Eight<T> r;
  r.set(v);
  r.template store<EVEN>(p, n);
}

}  // namespace qoda
