// Group normalisation with an activation, channels last, and its gradient (include/qoda_operators.h).

#include "qoda_operators_device.h"

namespace qoda {

namespace {

// The sum over the workgroup's 256 threads, in all of them.
__device__ float block_sum(float v, float *red) {
  __syncthreads();
  red[threadIdx.x] = v;
  __syncthreads();
  for (int h = 128; h > 0; h /= 2) {
    if (threadIdx.x < h) red[threadIdx.x] = red[threadIdx.x] + red[threadIdx.x + h];
    __syncthreads();
  }
  return red[0];
}

// A workgroup for each (sample, group): the mean, then the squares about it, then the values.
template <class T>
__global__ void __launch_bounds__(256) k_norm(GroupNorm g) {
  __shared__ float red[256];
  const long long n = blockIdx.x / g.groups, gr = blockIdx.x % g.groups, per = g.channels / g.groups, total = per * g.positions;
  const T *x = static_cast<const T *>(g.x) + n * g.x_sample + gr * per;
  T *y = static_cast<T *>(g.out) + n * g.out_sample + gr * per;
  float s = 0.0f;
  for (long long q = threadIdx.x; q < total; q += 256) s = s + to_float(x[q / per * g.x_pos + q % per]);
  const float mean = block_sum(s, red) / (float)total;
  s = 0.0f;
  for (long long q = threadIdx.x; q < total; q += 256) {
    const float d = to_float(x[q / per * g.x_pos + q % per]) - mean;
    s = __builtin_fmaf(d, d, s);
  }
  const float rstd = 1.0f / sqrtf(block_sum(s, red) / (float)total + g.eps);
  if (threadIdx.x == 0) g.mean[blockIdx.x] = mean, g.rstd[blockIdx.x] = rstd;
  for (long long q = threadIdx.x; q < total; q += 256) {
    const long long c = q % per, at = gr * per + c;
    const float h = (to_float(x[q / per * g.x_pos + c]) - mean) * rstd;
    const float v = __builtin_fmaf(h, g.weight ? g.weight[at] : 1.0f, g.bias ? g.bias[at] : 0.0f);
    y[q / per * g.out_pos + c] = from_float<T>(act_of(g.activation, v));
  }
}

// The gradient before the activation, and the normalised value, of entry c of a group's position.
template <class T>
__device__ __forceinline__ void through(const GroupNorm &g, long long n, long long p, long long c, float mean, float rstd, float &dh, float &h) {
  h = (to_float(static_cast<const T *>(g.x)[n * g.x_sample + p * g.x_pos + c]) - mean) * rstd;
  dh = to_float(static_cast<const T *>(g.dy)[n * g.dy_sample + p * g.dy_pos + c]);
  if (g.activation != kActNone)
    dh = dh * act_slope_of(g.activation, __builtin_fmaf(h, g.weight ? g.weight[c] : 1.0f, g.bias ? g.bias[c] : 0.0f));
}

template <class T>
__global__ void __launch_bounds__(256) k_norm_grad(GroupNorm g) {
  __shared__ float red[256];
  const long long n = blockIdx.x / g.groups, gr = blockIdx.x % g.groups, per = g.channels / g.groups, total = per * g.positions;
  const float mean = g.mean[blockIdx.x], rstd = g.rstd[blockIdx.x];
  float s1 = 0.0f, s2 = 0.0f;
  for (long long q = threadIdx.x; q < total; q += 256) {
    const long long c = gr * per + q % per;
    float dh, h;
    through<T>(g, n, q / per, c, mean, rstd, dh, h);
    const float u = g.weight ? dh * g.weight[c] : dh;
    s1 = s1 + u;
    s2 = __builtin_fmaf(u, h, s2);
  }
  const float m1 = block_sum(s1, red) / (float)total, m2 = block_sum(s2, red) / (float)total;
  for (long long q = threadIdx.x; q < total; q += 256) {
    const long long c = gr * per + q % per, p = q / per;
    float dh, h;
    through<T>(g, n, p, c, mean, rstd, dh, h);
    const float u = g.weight ? dh * g.weight[c] : dh;
    float v = __builtin_fmaf(-h, m2, u - m1) * rstd;
    if (g.extra) v = to_float(static_cast<const T *>(g.extra)[n * g.extra_sample + p * g.extra_pos + c]) + v;
    static_cast<T *>(g.out)[n * g.out_sample + p * g.out_pos + c] = from_float<T>(v);
  }
}

// dweight and dbias: 64 channels a workgroup, its four waves take positions in turn.  Before k_norm_grad, which may write where
// the residual is but leaves x and dy alone.
template <class T>
__global__ void __launch_bounds__(256) k_norm_channels(GroupNorm g) {
  __shared__ float part[2][4][64];
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const long long c = (long long)blockIdx.x * 64 + lane;
  float sw = 0.0f, sb = 0.0f;
  if (c < g.channels) {
    const long long gr = c / (g.channels / g.groups);
    for (long long q = wave; q < g.samples * g.positions; q += 4) {
      const long long n = q / g.positions;
      float dh, h;
      through<T>(g, n, q % g.positions, c, g.mean[n * g.groups + gr], g.rstd[n * g.groups + gr], dh, h);
      sw = __builtin_fmaf(dh, h, sw);
      sb = sb + dh;
    }
  }
  part[0][wave][lane] = sw, part[1][wave][lane] = sb;
  __syncthreads();
  if (wave < 2 && c < g.channels) {
    const float v = (part[wave][0][lane] + part[wave][1][lane]) + (part[wave][2][lane] + part[wave][3][lane]);
    float *o = wave == 0 ? g.dweight : g.dbias;
    if (o) o[c] = g.accumulate ? o[c] + v : v;
  }
}

}  // namespace

size_t group_norm_scratch(const GroupNorm &, bool) { return 0; }

hipError_t launch_group_norm(const GroupNorm &g, hipStream_t s) {
  const dim3 grid((unsigned)(g.samples * g.groups));
  if (g.type == kF32) k_norm<float><<<grid, 256, 0, s>>>(g);
  else k_norm<bf16><<<grid, 256, 0, s>>>(g);
  return hipGetLastError();
}

hipError_t launch_group_norm_grad(const GroupNorm &g, hipStream_t s) {
  if (g.dweight || g.dbias) {
    const dim3 grid((unsigned)((g.channels + 63) / 64));
    if (g.type == kF32) k_norm_channels<float><<<grid, 256, 0, s>>>(g);
    else k_norm_channels<bf16><<<grid, 256, 0, s>>>(g);
  }
  const dim3 grid((unsigned)(g.samples * g.groups));
  if (grid.x && g.positions) {
    if (g.type == kF32) k_norm_grad<float><<<grid, 256, 0, s>>>(g);
    else k_norm_grad<bf16><<<grid, 256, 0, s>>>(g);
  }
  return hipGetLastError();
}

}  // namespace qoda
