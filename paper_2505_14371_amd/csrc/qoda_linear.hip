// Matrix products with what follows them fused into their stores: x w^T, dz w and dz^T x of include/qoda_operators.h.

#include "qoda_operators_device.h"

namespace qoda {

namespace {

constexpr int kTile = 64, kDepth = 16;

// c[i][j], after the sum over l, to where the call wants it.
template <class T>
__device__ __forceinline__ void finish(const Product &p, int i, int j, float c) {
  if (p.form == kProductColumns) {
    float *o = static_cast<float *>(p.out) + (long long)i * p.ldo + j;
    *o = p.accumulate ? *o + c : c;
    return;
  }
  if (p.form == kProductRows) {
    if (p.bias) c = c + p.bias[j];
    if (p.pre) static_cast<T *>(p.pre)[(long long)i * p.ldp + j] = from_float<T>(c);
    c = act_of(p.activation, c);
  } else if (p.pre) {
    c = c * act_slope_of(p.activation, to_float(static_cast<const T *>(p.pre)[(long long)i * p.ldp + j]));
  }
  c = dropped(p.drop, i, j, c);
  if (p.extra) c = to_float(static_cast<const T *>(p.extra)[(long long)i * p.lde + j]) + c;
  static_cast<T *>(p.out)[(long long)i * p.ldo + j] = from_float<T>(c);
}

// A tile of 64 x 64 sums by 256 threads of 4 x 4, 16 deep through shared memory.
template <class T>
__global__ void __launch_bounds__(256) k_product(Product p) {
  __shared__ float as[kDepth][kTile + 4], bs[kDepth][kTile + 4];
  const int tiles_n = (p.n + kTile - 1) / kTile;
  const int i0 = (int)(blockIdx.x / tiles_n) * kTile, j0 = (int)(blockIdx.x % tiles_n) * kTile;
  const int t = threadIdx.x, ti = t / 16, tj = t % 16;
  const T *a = static_cast<const T *>(p.a), *b = static_cast<const T *>(p.b);
  float c[4][4] = {};
  for (int l0 = 0; l0 < p.k; l0 += kDepth) {
    for (int e = t; e < kTile * kDepth; e += 256) {
      const bool rows = p.form != kProductColumns;
      const int i = rows ? e / kDepth : e % kTile, l = rows ? e % kDepth : e / kTile;
      as[l][i] = i0 + i < p.m && l0 + l < p.k ? to_float(a[rows ? (i0 + i) * p.lda + l0 + l : (l0 + l) * p.lda + i0 + i]) : 0.0f;
    }
    for (int e = t; e < kTile * kDepth; e += 256) {
      const bool rows = p.form == kProductRows;
      const int j = rows ? e / kDepth : e % kTile, l = rows ? e % kDepth : e / kTile;
      bs[l][j] = j0 + j < p.n && l0 + l < p.k ? to_float(b[rows ? (j0 + j) * p.ldb + l0 + l : (l0 + l) * p.ldb + j0 + j]) : 0.0f;
    }
    __syncthreads();
    for (int l = 0; l < kDepth; ++l)
#pragma unroll
      for (int x = 0; x < 4; ++x)
#pragma unroll
        for (int y = 0; y < 4; ++y) c[x][y] = __builtin_fmaf(as[l][4 * ti + x], bs[l][4 * tj + y], c[x][y]);
    __syncthreads();
  }
  for (int x = 0; x < 4; ++x)
    for (int y = 0; y < 4; ++y) {
      const int i = i0 + 4 * ti + x, j = j0 + 4 * tj + y;
      if (i < p.m && j < p.n) finish<T>(p, i, j, c[x][y]);
    }
}

// The sums of a's columns (a[l][i]): 64 columns a workgroup, its four waves take rows in turn.
template <class T>
__global__ void __launch_bounds__(256) k_column_sums(Product p) {
  __shared__ float part[4][64];
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const long long i = (long long)blockIdx.x * 64 + lane;
  const T *a = static_cast<const T *>(p.a);
  float s = 0.0f;
  if (i < p.m)
    for (int l = wave; l < p.k; l += 4) s = s + to_float(a[l * p.lda + i]);
  part[wave][lane] = s;
  __syncthreads();
  if (wave == 0 && i < p.m) {
    s = (part[0][lane] + part[1][lane]) + (part[2][lane] + part[3][lane]);
    p.sums[i] = p.accumulate ? p.sums[i] + s : s;
  }
}

}  // namespace

size_t product_scratch(const Product &) { return 0; }

hipError_t launch_product(const Product &p, hipStream_t s) {
  const long long tiles = (long long)((p.m + kTile - 1) / kTile) * ((p.n + kTile - 1) / kTile);
  if (tiles > 0x7fffffffll) return hipErrorInvalidValue;
  if (tiles > 0) {
    if (p.type == kF32) k_product<float><<<dim3((unsigned)tiles), 256, 0, s>>>(p);
    else k_product<bf16><<<dim3((unsigned)tiles), 256, 0, s>>>(p);
  }
  if (p.sums) {
    if (p.type == kF32) k_column_sums<float><<<dim3((p.m + 63) / 64), 256, 0, s>>>(p);
    else k_column_sums<bf16><<<dim3((p.m + 63) / 64), 256, 0, s>>>(p);
  }
  return hipGetLastError();
}

}  // namespace qoda
