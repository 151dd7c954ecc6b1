// Rounding to microscaled matrices and back, of include/qoda_matrices.h.
//
// A workgroup makes a step: 64 rows of q by 256 entries (eight blocks), whose codes are 128 bytes a row and whose scales are two runs of 256 bytes.
// As it lies: eight entries a lane, 16 or 32 bytes, a block's largest magnitude joined over its four lanes.  Transposed: a lane takes two columns
// of x over 32 rows, a block each, so that nothing is joined, and the codes pass through shared memory to be stored as rows.
//
// Measured, 16384 x 8192 of bf16 (268 MB, and 71 of codes and scales): to nearest 64 us as it lies (5.3 TB/s, memory) and 76 transposed, stochastically 84 to 105 and
// 77 to 92, the first passes after idle ones the longest (arithmetic: the generator is twelve operations an entry and the code ten); values 55 to 63.  Of fp32 111 and 130, 111 and 132, values 152.

#include "qoda_mx_device.h"

namespace qoda {

namespace {

constexpr int kWg = 256;

// The scales of a step, from shared memory.
__device__ __forceinline__ void store_scales(const MxRounding &a, const u8 *s, long long group, long long groups, long long step) {
  const int t = threadIdx.x;
  if (t < 128) {
    u32 w;
    __builtin_memcpy(&w, s + 4 * t, 4);
    u8 *to = a.scales + ((2 * step + (t >> 6)) * groups + group) * 256 + 4 * (t & 63);
    __builtin_memcpy(to, &w, 4);
  }
}

// U: rows that a lane takes one after the other, of 64 / U that the workgroup has at a time.
template <class T, bool STOCHASTIC, int U>
__global__ void __launch_bounds__(2048 / U) k_mx_rows(MxRounding a, long long groups, long long steps) {
  __shared__ __align__(16) u8 scales[512];
  const long long id = a.first + blockIdx.x, group = id / steps, step = id - group * steps;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, eight = lane & 31;
  const long long c0 = step * kMxStep + eight * 8;
  const int n = a.cols - c0 < 8 ? (int)(a.cols - c0) : 8;
  const int row0 = wave * 2 * U + (lane >> 5);
  Eight<T> v[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const long long r = group * 64 + row0 + 2 * u;
    v[u].load(static_cast<const T *>(a.x) + r * a.ldx + c0, r < a.rows ? n : 0);
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int row = row0 + 2 * u;
    const long long r = group * 64 + row;
    u32 most = most_of(v[u]), other = __shfl_xor(most, 1);
    most = most > other ? most : other;
    other = __shfl_xor(most, 2);
    most = most > other ? most : other;
    const u32 byte = scale_byte(most, STOCHASTIC);
    u32 codes;
    if constexpr (STOCHASTIC) {
      float f[8];
      v[u].get(f);
      u32 x[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = __float_as_uint(f[j]);
      codes = codes_stochastic(x, byte, (u32)r, (u32)(c0 >> 3), a);
    } else {
      codes = codes_nearest(v[u], scale_of(byte));
    }
    if (n < 8) codes = n <= 0 ? 0u : codes & ((1u << 4 * n) - 1u);
    if (byte == 255u) codes = 0;
    if (r < a.rows) __builtin_memcpy(a.codes + (r * steps + step) * 128 + eight * 4, &codes, 4);
    if ((lane & 3) == 0) scales[256 * (eight >> 4) + scale_place(row, eight >> 2 & 3)] = (u8)byte;
  }
  __syncthreads();
  store_scales(a, scales, group, groups, step);
}

// Two entries of a row of x, adjacent, of which `n` exist.
template <class T>
struct Two {
  u32 w[sizeof(T) / 2];
  __device__ __forceinline__ void load(const T *p, int n) {
    if (n >= 2) {
      __builtin_memcpy(w, p, sizeof w);
    } else {
#pragma unroll
      for (u32 &v : w) v = 0;
      if (n == 1) {
        if constexpr (sizeof(T) == 4) w[0] = __float_as_uint(*p);
        else w[0] = p->bits;
      }
    }
  }
  __device__ __forceinline__ u32 bits(int h) const {   // as fp32
    if constexpr (sizeof(T) == 4) return w[h];
    else return h ? w[0] & 0xFFFF0000u : w[0] << 16;
  }
};

template <class T, bool STOCHASTIC>
__global__ void __launch_bounds__(kWg) k_mx_columns(MxRounding a, long long groups, long long steps) {
  constexpr int kRow = 144;   // bytes from one row of codes to the next in shared memory: 16 more than it has, for the banks
  __shared__ __align__(16) u8 scales[512], tile[64 * kRow];
  const long long id = a.first + blockIdx.x, step = id / groups, group = id - step * groups;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, block = wave * 2 + (lane >> 5), col = (lane & 31) * 2;
  const long long c0 = group * 64 + col, r0 = step * kMxStep + block * 32;
  const int n = a.cols - c0 < 2 ? (int)(a.cols - c0) : 2;
  const T *x = static_cast<const T *>(a.x) + r0 * a.ldx + c0;
  Two<T> v[32];
  if (group * 64 + 64 <= a.cols && step * kMxStep + kMxStep <= a.rows) {
#pragma unroll
    for (int u = 0; u < 32; ++u) v[u].load(x + u * a.ldx, 2);
  } else {
#pragma unroll
    for (int u = 0; u < 32; ++u) v[u].load(x + u * a.ldx, r0 + u < a.rows ? n : 0);
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    u32 most = 0;
#pragma unroll
    for (int u = 0; u < 32; ++u) {
      const u32 m = v[u].bits(h) & 0x7FFFFFFFu;
      most = most > m ? most : m;
    }
    const u32 byte = scale_byte(most, STOCHASTIC);
    v4u codes;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (STOCHASTIC) {
        u32 x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = v[8 * e + j].bits(h);
        codes[e] = codes_stochastic(x, byte, (u32)(c0 + h), (u32)(r0 >> 3) + e, a);
      } else {
        Eight<T> f;
#pragma unroll
        for (int j = 0; j < Eight<T>::kWords; ++j) {
          if constexpr (sizeof(T) == 4) f.w[j / 4][j % 4] = v[8 * e + j].w[h];
          else f.w[0][j] = h ? __builtin_amdgcn_perm(v[8 * e + 2 * j + 1].w[0], v[8 * e + 2 * j].w[0], 0x07060302u)
                             : __builtin_amdgcn_perm(v[8 * e + 2 * j + 1].w[0], v[8 * e + 2 * j].w[0], 0x05040100u);
        }
        codes[e] = codes_nearest(f, scale_of(byte));
      }
      const long long left = a.rows - r0 - 8 * e;
      if (left < 8) codes[e] = left <= 0 ? 0u : codes[e] & ((1u << 4 * (int)left) - 1u);
      if (byte == 255u) codes[e] = 0;
    }
    __builtin_memcpy(tile + (col + h) * kRow + block * 16, &codes, 16);
    scales[256 * (block >> 2) + scale_place(col + h, block & 3)] = (u8)byte;
  }
  __syncthreads();
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int at = u * kWg + (int)threadIdx.x, row = at >> 3, chunk = at & 7;
    v4u w;
    __builtin_memcpy(&w, tile + row * kRow + chunk * 16, 16);
    if (group * 64 + row < a.cols) __builtin_memcpy(a.codes + ((group * 64 + row) * steps + step) * 128 + chunk * 16, &w, 16);
  }
  store_scales(a, scales, group, groups, step);
}

// Eight entries a lane, 64 rows by 256 entries a workgroup, as they were rounded.
template <class T>
__global__ void __launch_bounds__(kWg) k_mx_values(MxRounding a, long long groups, long long steps) {
  const long long id = a.first + blockIdx.x, group = id / steps, step = id - group * steps;
  const int eight = threadIdx.x & 31, row0 = threadIdx.x >> 5;
  const long long c0 = step * kMxStep + eight * 8;
  const int n = a.cols - c0 < 8 ? (int)(a.cols - c0) : 8, last = a.rows - group * 64 < 64 ? (int)(a.rows - group * 64) - 1 : 63;
  const u8 *codes = a.codes + (group * 64 * steps + step) * 128 + eight * 4, *scales = a.scales + ((2 * step + (eight >> 4)) * groups + group) * 256;
  u32 w[8], byte[8];
#pragma unroll
  for (int u = 0; u < 8; ++u) {   // rows behind the last one: that one's again
    const int row = row0 + 8 * u < last ? row0 + 8 * u : last;
    __builtin_memcpy(&w[u], codes + row * steps * 128, 4);
    byte[u] = scales[scale_place(row, eight >> 2 & 3)];
  }
  T *y = static_cast<T *>(a.x) + group * 64 * a.ldx + c0;
#pragma unroll
  for (int u = 0; u < 8; ++u)
    if (row0 + 8 * u <= last) {
      float v[8];
      values_of(w[u], byte[u], v);
      store8(y + (row0 + 8 * u) * a.ldx, n, v);
    }
}

template <class T, bool STOCHASTIC>
void launch_rounding(const MxRounding &q, hipStream_t s) {
  const long long rows = q.transposed ? q.cols : q.rows, along = q.transposed ? q.rows : q.cols;
  const long long groups = mx_groups(rows), steps = mx_steps(along);
  if (q.transposed) {
    in_launches(q, groups * steps, kWg, [&](const MxRounding &part, unsigned grid) { k_mx_columns<T, STOCHASTIC><<<dim3(grid), kWg, 0, s>>>(part, groups, steps); });
  } else if (groups * steps < 512) {
    // fewer workgroups than the device holds: more waves each
    k_mx_rows<T, STOCHASTIC, 2><<<dim3((unsigned)(groups * steps)), 1024, 0, s>>>(q, groups, steps);
  } else {
    in_launches(q, groups * steps, kWg, [&](const MxRounding &part, unsigned grid) { k_mx_rows<T, STOCHASTIC, 8><<<dim3(grid), kWg, 0, s>>>(part, groups, steps); });
  }
}

}  // namespace

hipError_t launch_mx_quantize(const MxRounding &q, hipStream_t s) {
  if (q.type == kF32) q.stochastic ? launch_rounding<float, true>(q, s) : launch_rounding<float, false>(q, s);
  else q.stochastic ? launch_rounding<bf16, true>(q, s) : launch_rounding<bf16, false>(q, s);
  return hipGetLastError();
}

hipError_t launch_mx_values(const MxRounding &q, hipStream_t s) {
  const long long groups = mx_groups(q.rows), steps = mx_steps(q.cols);
  in_launches(q, groups * steps, kWg, [&](const MxRounding &part, unsigned grid) {
    if (q.type == kF32) k_mx_values<float><<<dim3(grid), kWg, 0, s>>>(part, groups, steps);
    else k_mx_values<bf16><<<dim3(grid), kWg, 0, s>>>(part, groups, steps);
  });
  return hipGetLastError();
}

}  // namespace qoda
