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

// The two factors of 1 - Phi(|z|) = erfc(|z| / sqrt 2) / 2 = q e with e = exp(-z^2 / 2): formula 7.1.26 of Abramowitz and Stegun, erfc(x) =
// (a1 t + ... + a5 t^5) exp(-x^2) with t = 1 / (1 + p x), whose error is at most 1.5e-7 -- that of 1 + erf in fp32.  The exponential is the
// density's too, so the function and its derivative take one exponential and one reciprocal.  (halves and roots of two are in the constants.)
__device__ __forceinline__ void normal_tail(float z, float &q, float &e) {
  const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.3275911f * 0.70710678118654752f, fabsf(z), 1.0f));
  e = __builtin_amdgcn_exp2f(z * z * (-0.5f * kLog2E));
  q = __builtin_fmaf(0.5f * 1.061405429f, t, 0.5f * -1.453152027f);
  q = __builtin_fmaf(q, t, 0.5f * 1.421413741f);
  q = __builtin_fmaf(q, t, 0.5f * -0.284496736f);
  q = __builtin_fmaf(q, t, 0.5f * 0.254829592f) * t;
}

template <int ACT>
__device__ __forceinline__ float act(float z) {
  if constexpr (ACT == kActRelu) return z < 0.0f ? 0.0f : z;   // a NaN stays one
  if constexpr (ACT == kActLeakyRelu) return z > 0.0f ? z : kSlope * z;
  if constexpr (ACT == kActGelu) {
    float q, e;
    normal_tail(z, q, e);
    return z * (0.5f + copysignf(__builtin_fmaf(-q, e, 0.5f), z));   // Phi - 1/2 is odd
  }
  if constexpr (ACT == kActSilu) return z * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-kLog2E * z));
  return z;
}

template <int ACT>
__device__ __forceinline__ float act_slope(float z) {
  if constexpr (ACT == kActRelu) return z > 0.0f ? 1.0f : 0.0f;
  if constexpr (ACT == kActLeakyRelu) return z > 0.0f ? 1.0f : kSlope;
  if constexpr (ACT == kActGelu) {
    float q, e;
    normal_tail(z, q, e);
    // Phi - 1/2 + z phi is odd: 1/2 - q e + |z| e / sqrt(2 pi) on the right
    return 0.5f + copysignf(__builtin_fmaf(e, __builtin_fmaf(fabsf(z), 0.39894228040143268f, -q), 0.5f), z);
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
