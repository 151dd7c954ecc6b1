// Dropout and its gradient, with the activation and the residual beside it (include/qoda_operators.h).
//
// One pass, bound by memory with arithmetic close behind: 268 M entries of bf16 through gelu's slope 307 us, 5.2 TB/s (288 without the lots, which are ten
// rounds of the generator for eight entries, a third of the arithmetic).  It hides behind the loads as long as these are whole words and several on
// their way (entry by entry 812 us, as structures of 16-bit entries, which the compiler loads in parts, 353).

#include <type_traits>

#include "qoda_operators_device.h"

namespace qoda {

namespace {

// Whole-number division of 32-bit numbers by one that a launch knows, as a product (Granlund and Montgomery 1994).
struct Divisor {
  u32 d, magic, shift1, shift2;
};
Divisor divisor(u32 d) {
  int l = 0;
  while (l < 32 && (1ull << l) < d) ++l;
  return {d, (u32)(((1ull << l) - d) * (1ull << 32) / d + 1), l > 0 ? 1u : 0u, l > 0 ? (u32)(l - 1) : 0u};
}
__device__ __forceinline__ u32 divide(u32 v, const Divisor &d) {
  const u32 t = __umulhi(d.magic, v);
  return (t + ((v - t) >> d.shift1)) >> d.shift2;
}

constexpr int kEach = 4;   // blocks of eight entries a thread: so many loads on their way while the first block's lots are drawn

// A thread takes blocks of eight entries, which share one draw of lots: 16 bytes of bf16.
template <class T, int ACT, bool GRAD, bool EXTRA, bool DROP, bool EVEN>
__global__ void __launch_bounds__(256) k_entries(Entries e, Divisor blocks) {
  // the workgroup's first block by a 64-bit division, the others from it in 32 bits
  const long long total = e.rows * blocks.d, q0 = (e.first + blockIdx.x) * (256 * kEach);
  const long long row0 = q0 / blocks.d;
  const u32 col0 = (u32)(q0 - row0 * blocks.d);
  const T *x = static_cast<const T *>(e.x), *extra = static_cast<const T *>(e.extra);
  Eight<T> mine[kEach], other[kEach];
  long long row[kEach];
  u32 block[kEach];
  int n[kEach];
#pragma unroll
  for (int u = 0; u < kEach; ++u) {
    const u32 at = col0 + u * 256 + threadIdx.x, r = divide(at, blocks);
    row[u] = row0 + r;
    block[u] = at - r * blocks.d;
    n[u] = q0 + u * 256 + threadIdx.x < total ? (int)(e.cols - (long long)block[u] * 8) : 0;
    if (n[u] > 0) {
      mine[u].template load<EVEN>(x + row[u] * e.ldx + (long long)block[u] * 8, n[u]);
      if (EXTRA) other[u].template load<EVEN>(extra + row[u] * e.lde + (long long)block[u] * 8, n[u]);
    }
  }
#pragma unroll
  for (int u = 0; u < kEach; ++u)
    if (n[u] > 0) {
      float v[8], o[8];
      mine[u].get(v);
      if (EXTRA) other[u].get(o);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = !GRAD ? act<T, ACT>(v[j]) : EXTRA ? v[j] * act_slope<T, ACT>(o[j]) : v[j];
      if (DROP) drop8(e.drop, (u32)row[u], block[u], v);
      if (!GRAD && EXTRA)
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = o[j] + v[j];
      store8<EVEN>(static_cast<T *>(e.y) + row[u] * e.ldy + (long long)block[u] * 8, n[u], v);
    }
}

template <class T, int ACT, bool GRAD, bool EXTRA>
void launch(const Entries &e, unsigned grid, const Divisor &d, hipStream_t s) {
  const auto run = [&](auto even) {
    if (e.drop.threshold) k_entries<T, ACT, GRAD, EXTRA, true, decltype(even)::value><<<dim3(grid), 256, 0, s>>>(e, d);
    else k_entries<T, ACT, GRAD, EXTRA, false, decltype(even)::value><<<dim3(grid), 256, 0, s>>>(e, d);
  };
  if (e.cols % 8 == 0) run(std::true_type());
  else run(std::false_type());
}

template <class T, int ACT>
void launch(const Entries &e, unsigned grid, const Divisor &d, hipStream_t s) {
  if (e.gradient) launch<T, ACT, true, ACT != kActNone>(e, grid, d, s);
  else if (e.extra) launch<T, ACT, false, true>(e, grid, d, s);
  else launch<T, ACT, false, false>(e, grid, d, s);
}

template <class T>
void launch(const Entries &e, unsigned grid, const Divisor &d, hipStream_t s) {
  switch (e.activation) {
    case kActRelu: return launch<T, kActRelu>(e, grid, d, s);
    case kActLeakyRelu: return launch<T, kActLeakyRelu>(e, grid, d, s);
    case kActGelu: return launch<T, kActGelu>(e, grid, d, s);
    case kActSilu: return launch<T, kActSilu>(e, grid, d, s);
    default: return launch<T, kActNone>(e, grid, d, s);
  }
}

}  // namespace

hipError_t launch_entries(const Entries &e, hipStream_t s) {
  const u32 blocks = (u32)((e.cols + 7) / 8);
  const long long groups = (e.rows * blocks + 256 * kEach - 1) / (256 * kEach);
  in_launches(e, groups, 256, [&](const Entries &part, unsigned grid) {
    if (e.type == kF32) launch<float>(part, grid, divisor(blocks), s);
    else launch<bf16>(part, grid, divisor(blocks), s);
  });
  return hipGetLastError();
}

}  // namespace qoda
