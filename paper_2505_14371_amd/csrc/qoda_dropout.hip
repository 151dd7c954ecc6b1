// Dropout and its gradient, with the activation and the residual beside it (include/qoda_operators.h).

#include "qoda_operators_device.h"

namespace qoda {

namespace {

// A thread takes the eight entries of one block of lots at a time.
template <class T, int ACT, bool GRAD>
__global__ void __launch_bounds__(256) k_entries(Entries e) {
  const long long blocks = (e.cols + 7) / 8, total = e.rows * blocks;
  const T *x = static_cast<const T *>(e.x), *extra = static_cast<const T *>(e.extra);
  T *y = static_cast<T *>(e.y);
  for (long long q = (long long)blockIdx.x * 256 + threadIdx.x; q < total; q += (long long)gridDim.x * 256) {
    const long long row = q / blocks, c0 = (q - row * blocks) * 8;
    const u32 kept = e.drop.threshold ? kept_bits(e.drop, (u32)row, (u32)(c0 / 8)) : 0xFFu;
    const float scale = e.drop.threshold ? e.drop.scale : 1.0f;
    for (int j = 0; j < 8 && c0 + j < e.cols; ++j) {
      float v = to_float(x[row * e.ldx + c0 + j]);
      const float o = extra ? to_float(extra[row * e.lde + c0 + j]) : 0.0f;
      if (GRAD) v = ACT == kActNone ? v : v * act_slope<ACT>(o);
      else v = act<ACT>(v);
      v = kept >> j & 1 ? v * scale : 0.0f;
      if (!GRAD && extra) v = o + v;
      y[row * e.ldy + c0 + j] = from_float<T>(v);
    }
  }
}

template <class T, int ACT>
void launch(const Entries &e, unsigned grid, hipStream_t s) {
  if (e.gradient) k_entries<T, ACT, true><<<dim3(grid), 256, 0, s>>>(e);
  else k_entries<T, ACT, false><<<dim3(grid), 256, 0, s>>>(e);
}

template <class T>
void launch(const Entries &e, unsigned grid, hipStream_t s) {
  switch (e.activation) {
    case kActRelu: return launch<T, kActRelu>(e, grid, s);
    case kActLeakyRelu: return launch<T, kActLeakyRelu>(e, grid, s);
    case kActGelu: return launch<T, kActGelu>(e, grid, s);
    case kActSilu: return launch<T, kActSilu>(e, grid, s);
    default: return launch<T, kActNone>(e, grid, s);
  }
}

}  // namespace

hipError_t launch_entries(const Entries &e, hipStream_t s) {
  const long long blocks = e.rows * ((e.cols + 7) / 8), groups = (blocks + 255) / 256;
  const unsigned grid = (unsigned)(groups < 65536 ? groups : 65536);
  if (e.type == kF32) launch<float>(e, grid, s);
  else launch<bf16>(e, grid, s);
  return hipGetLastError();
}

}  // namespace qoda
