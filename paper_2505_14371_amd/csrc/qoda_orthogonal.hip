// Orthogonalisation of updates by Newton-Schulz products, of include/qoda_matrices.h: X <- a X + (b A + c A A) X with A = X X^T.
//
// Small singular values grow by a in every step, and so do the errors of what they came from: sums of fp16 or bf16 products would leave them wrong in the
// second digit.  A number is therefore a pair of fp16 numbers, high + low, of 22 bits, and a product three matrix instructions: high high, high low and
// low high, summed in fp32.  Matrices are scaled by powers of two that the polynomial's bound on the singular values allows, so that the low parts are
// no subnormal numbers where they matter: a number is held to 2^-22 of itself or 2^-41 of the bound.  Polynomials whose bound may be far above the numbers that are there (a
// small or 0, or b s^3 and c s^5 growing) are taken by norm: in every step X and A are divided by what their norms are (at k_start_scales), which
// takes longer: five steps of 8192 x 2048 2447 us, of 16 times 2100 x 410 1004, of 61 x 37 173.
//
// The work is done on X [m][n] with m <= n (g, or its transpose).  Every product is of rows with rows: X is kept beside its transpose, and A and
// B = b A + c A A are symmetric, so that half of their tiles are computed and stored twice.  In memory 32 high parts of a row are followed by their low
// parts, 128 bytes, which is a step along l in shared memory, as in qoda_linear.hip.  Sides are filled up to multiples of 32 with zeros.
//
// Measured, five steps: 8192 x 2048 of fp32 1484 to 1550 us, of which A 4 times 98 and its join 16, the squares of 2048 8 times 38, the four products with X 178 each (375
// TFLOP/s of numbers, 1130 of halves: the library's product of halves reaches 1154) and the start 55; 16 of 2100 x 410 471 to 523; 61 x 37 of bf16 19, all in one
// launch.  Error against 64 bits of 8192 x 2048: 2.8e-6 (fp32 products 3.0e-6).

#include <cmath>

#include "qoda_matrices.h"
#include "qoda_product_device.h"

namespace qoda {

namespace {

typedef _Float16 v8h __attribute__((ext_vector_type(8)));

constexpr int kWg = 256;

__host__ __device__ inline long long up32(long long v) { return (v + 31) & ~31ll; }

// Eight adjacent entries of a row of pairs, from column j (a multiple of 8) on; ld: entries of a row.
__device__ __forceinline__ char *pair_place(void *base, long long ld, long long i, int j) {
  return static_cast<char *>(base) + i * ld * 4 + (j >> 5) * 128 + (j & 31) * 2;
}
__device__ __forceinline__ void store_pairs(char *p, const float (&v)[8]) {
  v8h hi, lo;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    hi[e] = (_Float16)v[e];
    lo[e] = (_Float16)(v[e] - (float)hi[e]);
  }
  __builtin_memcpy(p, &hi, 16);
  __builtin_memcpy(p + 64, &lo, 16);
}
__device__ __forceinline__ void load_pairs(const char *p, float (&v)[8]) {
  v8h hi, lo;
  __builtin_memcpy(&hi, p, 16);
  __builtin_memcpy(&lo, p + 64, 16);
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = (float)hi[e] + (float)lo[e];
}

// The sums of squares of a matrix in parts, each by a workgroup, in 64 bits.
template <class T>
__global__ void __launch_bounds__(kWg) k_squares(Orthogonal o) {
  __shared__ double part[kWg / 64];
  const long long id = o.first + blockIdx.x, matrix = id / o.parts;
  const int p = (int)(id - matrix * o.parts);
  const T *g = static_cast<const T *>(o.g) + matrix * o.g_matrix;
  const long long eights = (o.cols + 7) / 8, total = o.rows * eights;
  double sum = 0.0;
  for (long long q = (long long)p * kWg + threadIdx.x; q < total; q += (long long)o.parts * kWg) {
    const long long r = q / eights, c = (q - r * eights) * 8;
    float v[8];
    load8(g + r * o.g_row + c, o.cols - c < 8 ? (int)(o.cols - c) : 8, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) sum = sum + (double)v[e] * (double)v[e];
  }
#pragma unroll
  for (int d = 1; d < 64; d *= 2) sum = sum + __shfl_xor(sum, d);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = sum;
  __syncthreads();
  if (threadIdx.x == 0) o.squares[id] = (part[0] + part[1]) + (part[2] + part[3]);
}

// |g| of a matrix, from the parts' sums in their order.
__device__ __forceinline__ double norm_of(const double *squares, int parts, long long matrix) {
  double sum = 0.0;
  for (int p = (int)(threadIdx.x & 63); p < parts; p += 64) sum = sum + squares[matrix * parts + p];
#pragma unroll
  for (int d = 1; d < 64; d *= 2) sum = sum + __shfl_xor(sum, d);
  return sqrt(sum);
}

// X_0, scaled, and its transpose from g: 64 x 64 entries a workgroup, by way of shared memory.  STEPS false: nothing else is to be done, and x receives X_0.
template <class T, bool STEPS>
__global__ void __launch_bounds__(kWg) k_start(Orthogonal o, long long tiles_r, long long tiles_c) {
  __shared__ float tile[64][65];
  const long long id = o.first + blockIdx.x, each = tiles_r * tiles_c, matrix = id / each, in = id - matrix * each;
  const long long r0 = in / tiles_c * 64, c0 = (in - in / tiles_c * tiles_c) * 64;
  const double inverse = 1.0 / (norm_of(o.squares, o.parts, matrix) + o.eps) * (STEPS ? (double)o.scale : 1.0);
  const T *g = static_cast<const T *>(o.g) + matrix * o.g_matrix;
  const int t = threadIdx.x, chunk = (t & 7) * 8;
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int row = u * 32 + (t >> 3);
    const long long r = r0 + row, c = c0 + chunk;
    float v[8];
    load8(g + r * o.g_row + c, r < o.rows ? (o.cols - c < 8 ? (int)(o.cols - c) : 8) : 0, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (float)((double)v[e] * inverse);
    if constexpr (STEPS) {
      if (r >= o.rows || c + 7 >= o.cols)
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (r >= o.rows || c + e >= o.cols) v[e] = 0.0f;   // filled up, also where the inverse is no number
      const long long pad_r = up32(o.rows), pad_c = up32(o.cols);
      char *rows_of = static_cast<char *>(o.transposed ? o.xt : o.xs) + matrix * o.m * o.n * 4;
      if (r < pad_r && c < pad_c) store_pairs(pair_place(rows_of, pad_c, r, (int)c), v);
#pragma unroll
      for (int e = 0; e < 8; ++e) tile[row][chunk + e] = v[e];
    } else if (r < o.rows && c < o.cols) {
      store8(static_cast<T *>(o.x) + matrix * o.x_matrix + r * o.x_row + c, o.cols - c < 8 ? (int)(o.cols - c) : 8, v);
    }
  }
  if constexpr (STEPS) {
    __syncthreads();
    char *columns_of = static_cast<char *>(o.transposed ? o.xs : o.xt) + matrix * o.m * o.n * 4;
    const long long pad_r = up32(o.rows), pad_c = up32(o.cols);
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int row = u * 32 + (t >> 3);
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = tile[chunk + e][row];
      if (c0 + row < pad_c && r0 + chunk < pad_r) store_pairs(pair_place(columns_of, pad_r, c0 + row, (int)(r0 + chunk)), v);
    }
  }
}

// Of a step by norm: with n = |X|, Y = X / n, A' = Y Y^T, q = |A'| and A" = A' / q the next X is  n a Y + n^3 B' Y,  B' = q b A" + n^2 q^2 c A" A".  Y and A" are made from fp32 matrices by
// k_start, so that what is held as pairs is near its bound whatever X's size, and |B'| <= |q b| + |n^2 q^2 c|, which a power of two brings below 2^15.  At first X = X_0.  A wave a matrix.
__global__ void __launch_bounds__(kWg) k_start_scales(Orthogonal o, const double *squares_of_a, int parts_of_a, bool first) {
  const long long matrix = (o.first + blockIdx.x) * (kWg / 64) + threadIdx.x / 64;
  if (matrix >= o.matrices) return;
  double n = norm_of(o.squares, o.parts, matrix);
  const double q = norm_of(squares_of_a, parts_of_a, matrix);
  if ((threadIdx.x & 63) != 0) return;
  if (first) n = n / (n + o.eps);
  const double b = o.b * q, c = o.c * (n * n * q * q), size = fabs(b) + fabs(c);
  const int e = size > 0.0 && size < 1e300 ? 14 - ilogb(size) : 0;
  float *s = o.scales + 4 * matrix;
  s[0] = (float)ldexp(c, e), s[1] = (float)ldexp(b, e);
  s[2] = (float)ldexp(n * n * n, -e), s[3] = (float)(n * o.a);
}

// What becomes of eight sums adjacent in a row: v = sums * factor + what E and E2 have there * extra and extra2, which is then stored as T's or as pairs.
struct Place {
  const PairProduct &p;
  long long matrix;
  const float *scales = nullptr;   // the matrix's own
  __device__ __forceinline__ void add(const void *e, float extra, int i, int j, float (&v)[8]) const {
    float was[8];
    load_pairs(pair_place(const_cast<char *>(static_cast<const char *>(e) + matrix * p.m * p.n * 4), p.n, i, j), was);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = __builtin_fmaf(was[e], extra, v[e]);
  }
  __device__ __forceinline__ void finish(int i, int j, float (&v)[8]) const {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = v[e] * p.factor;
    if (scales) {   // one after the other: their product may be no normal number
      float was[8] = {};
      add(p.e, p.extra, i, j, was);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = __builtin_fmaf(was[e], scales[1], v[e] * scales[0]);
      return;
    }
    if (p.e) add(p.e, p.extra, i, j, v);
    if (p.e2) add(p.e2, p.extra2, i, j, v);
  }
  template <class T>
  __device__ __forceinline__ void plain(long long i, long long j, const float (&v)[8]) const {
    if (i < p.x_rows && j < p.x_cols) store8(static_cast<T *>(p.x) + matrix * p.x_matrix + i * p.x_row + j, p.x_cols - j < 8 ? (int)(p.x_cols - j) : 8, v);
  }
  // row i of the result from column j on
  __device__ __forceinline__ void row(int i, int j, const float (&v)[8]) const {
    if (p.x) {
      if (!p.x_transposed) p.type == kF32 ? plain<float>(i, j, v) : plain<bf16>(i, j, v);
    } else {
      store_pairs(pair_place(static_cast<char *>(p.out) + matrix * p.m * p.n * 4, p.n, i, j), v);
    }
  }
  // row j of its transpose, from column i on
  __device__ __forceinline__ void column(int i, int j, const float (&v)[8]) const {
    if (p.x) {
      if (p.x_transposed) p.type == kF32 ? plain<float>(j, i, v) : plain<bf16>(j, i, v);
    } else {
      store_pairs(pair_place(static_cast<char *>(p.out_t) + matrix * p.m * p.n * 4, p.m, j, i), v);
    }
  }
  __device__ __forceinline__ bool columns_wanted() const { return p.x ? p.x_transposed != 0 : p.out_t != nullptr; }
};

// Tile `at` of a symmetric product: those with tm <= tn, column by column.
__device__ __forceinline__ void upper_tile(int at, int &tm, int &tn) {
  int n = (int)((sqrtf(8.0f * (float)at + 1.0f) - 1.0f) * 0.5f);
  while ((long long)n * (n + 1) / 2 > at) --n;
  while ((long long)(n + 1) * (n + 2) / 2 <= at) ++n;
  tn = n, tm = at - (int)((long long)n * (n + 1) / 2);
}

__device__ __forceinline__ v4f multiply_halves(v4u b, v4u a, v4f c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, b), __builtin_bit_cast(v8h, a), c, 0, 0, 0);
}

// c = a b^T of matrices of pairs, [m][k] and [n][k].  S: steps in shared memory, of which one is multiplied and the others are on their way.
template <int BM, int BN, int WM, int WN, int S>
__global__ void __launch_bounds__(64 * WM * WN, 2) k_pair_product(PairProduct p, int tiles_m, int tiles_n, int steps_each) {
  constexpr int WG = 64 * WM * WN, FM = BM / WM / 16, FN = BN / WN / 32, kSide = BM / WM < 64 ? BM / WM : 64, kRow = kSide + 4;
  typedef Operand<bf16, true, 0, BM, WG, true> A;   // entries of 16 bits: 32 high parts and their 32 low parts are a step
  typedef Operand<bf16, true, 1, BN, WG, true> B;
  constexpr int kTiles = S * (BM + BN) * kStepBytes;
  static_assert(WM * WN * 32 * kRow * 4 <= kTiles, "the transposing end fits");
  __shared__ __align__(16) char shared[kTiles];

  const int each = p.symmetric ? tiles_m * (tiles_m + 1) / 2 : tiles_m * tiles_n;
  const long long id = xcd_run(p.first + blockIdx.x, p.matrices * each);   // an XCD has whole matrices, or runs of a matrix's tiles
  const int matrix = __builtin_amdgcn_readfirstlane((int)(id / each)), in = (int)(id - (long long)matrix * each);
  int tm, tn;
  if (p.symmetric) upper_tile(in, tm, tn);
  else band_tile(in, tiles_m, tiles_n, tm, tn);
  tm = __builtin_amdgcn_readfirstlane(tm), tn = __builtin_amdgcn_readfirstlane(tn);
  const int i0 = tm * BM, j0 = tn * BN;
  const int all = (int)(p.k / 32), step0 = (int)blockIdx.y * steps_each, steps = all - step0 < steps_each ? all - step0 : steps_each;
  A a;
  B b;
  a.start(static_cast<const char *>(p.a) + (long long)matrix * p.m * p.k * 4, p.k * 2, i0, (int)p.m, step0 * 64, steps * 64);
  b.start(static_cast<const char *>(p.b) + (long long)matrix * p.n * p.k * 4, p.k * 2, j0, (int)p.n, step0 * 64, steps * 64);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), wm = wave / WN * (BM / WM), wn = wave % WN * (BN / WN);

  v4f c[FM][2 * FN];
#pragma unroll
  for (int x = 0; x < FM; ++x)
#pragma unroll
    for (int y = 0; y < 2 * FN; ++y) c[x][y] = v4f{0, 0, 0, 0};

  const lds_ptr base = (lds_ptr)shared;
  constexpr u32 kBuffer = (BM + BN) * kStepBytes;
  u32 now = 0;   // the buffer of the step that is multiplied
  typedef v4u PiecesA[FM];
  typedef v4u PiecesB[2 * FN];
  u32 key_a = A::lane_key(wm), key_b = B::lane_key(wn);
  const auto read_a = [&](PiecesA &f, u32 from, int s) {
    asm volatile("" : "+v"(key_a));   // made anew each time, as in k_product
#pragma unroll
    for (int x = 0; x < FM; ++x) f[x] = A::piece(base + from, key_a, wm, x * 16, 0, s);
  };
  const auto read_b = [&](PiecesB &f, u32 from, int s) {
    asm volatile("" : "+v"(key_b));
#pragma unroll
    for (int y = 0; y < 2 * FN; ++y) f[y] = B::piece(base + from + BM * kStepBytes, key_b, wn, y / 2 * 32, y & 1, s);
  };
  const auto multiply_all = [&](const PiecesA &fa, const PiecesB &fb) {
#pragma unroll
    for (int x = 0; x < FM; ++x)
#pragma unroll
      for (int y = 0; y < 2 * FN; ++y) c[x][y] = multiply_halves(fb[y], fa[x], c[x][y]);
  };
  const auto request = [&](int t, u32 to) {
    a.direct(t * 64, base + to);
    b.direct(t * 64, base + to + BM * kStepBytes);
  };
  // One block without branches around what is read and multiplied: behind the last step the next one's pieces are read all the same, from what the buffer
  // holds, and not used.  (With branches the compiler kept copies of the sums.)
  PiecesA a_hi, a_lo;
  PiecesB b_hi, b_lo;
  constexpr int kLoads = A::kMine + B::kMine;
  const auto behind = [&](int t) { return steps - 1 - t < S - 2 ? steps - 1 - t : S - 2; };   // steps behind step t that are on their way
#pragma unroll
  for (int t = 0; t < S; ++t)
    if (t < steps) request(t, t * kBuffer);
  arrived_but<kLoads, S - 2>(behind(0));
  read_a(a_hi, 0, 0);
  read_b(b_hi, 0, 0);
  for (int t = 0; t < steps; ++t) {
    read_b(b_lo, now, 1);
    read_a(a_lo, now, 1);
    multiply_all(a_hi, b_hi);
    arrived_but<kLoads, S - 2>(behind(t + 1));   // the next step is there, and nobody reads this one any more
    if (t + S < steps) request(t + S, now);
    now = now == (S - 1) * kBuffer ? 0 : now + kBuffer;
    multiply_all(a_hi, b_lo);
    read_a(a_hi, now, 0);
    multiply_all(a_lo, b_hi);
    read_b(b_hi, now, 0);
    __builtin_amdgcn_sched_barrier(0);
  }

  const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
  const auto row = [&](int x) { return i0 + wm + x * 16 + i; };
  const auto column = [&](int y) { return j0 + wn + y * 32 + g * 8; };
  const auto sums = [&](int x, int y, float (&v)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = c[x][2 * y + e / 4][e & 3];
  };
  if (p.partial) {
    float *to = p.partial + ((long long)blockIdx.y * p.matrices + matrix) * p.m * p.n;
#pragma unroll
    for (int x = 0; x < FM; ++x)
#pragma unroll
      for (int y = 0; y < FN; ++y)
        if (row(x) < p.m && column(y) < p.n) {
          float v[8];
          sums(x, y, v);
          store8<true>(to + (long long)row(x) * p.n + column(y), 8, v);
        }
    return;
  }
  const Place place{p, matrix};
  const bool columns = place.columns_wanted() && !(p.symmetric && tm == tn);
  const lds_ptr mine = base + wave * 32 * kRow * 4;
  __syncthreads();   // the tiles' memory is taken for the transposed result, a wave's own part of it
#pragma unroll
  for (int y = 0; y < FN; ++y)
#pragma unroll
    for (int x0 = 0; x0 < FM; x0 += kSide / 16) {
#pragma unroll
      for (int x = 0; x < kSide / 16; ++x) {
        float v[8];
        sums(x0 + x, y, v);
        if (row(x0 + x) < p.m && column(y) < p.n) {
          place.finish(row(x0 + x), column(y), v);
          place.row(row(x0 + x), column(y), v);
        }
        if (columns)
#pragma unroll
          for (int e = 0; e < 8; ++e) *LDS(float, mine + ((g * 8 + e) * kRow + x * 16 + i) * 4) = v[e];
      }
      if (columns) {
        __builtin_amdgcn_wave_barrier();
        constexpr int kChunks = kSide / 8;
#pragma unroll
        for (int u = 0; u < 32 * kChunks / 64; ++u) {
          const int at = u * 64 + lane, jj = at / kChunks, ii = at % kChunks * 8;
          float v[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = *LDS(float, mine + (jj * kRow + ii + e) * 4);
          const int ci = i0 + wm + x0 * 16 + ii, cj = j0 + wn + y * 32 + jj;
          if (ci < p.m && cj < p.n) place.column(ci, cj, v);
        }
        __builtin_amdgcn_wave_barrier();
      }
    }
}

// The splits' sums added up in their order, and finished: N x N entries a workgroup, N * 4 threads.  Of a symmetric product the entries of tiles above the diagonal and on
// it are there, of the product's own tiles; the join's, which are taken whole, lie inside those where N divides their side.
template <int N>
__global__ void __launch_bounds__(N * 4) k_pair_join(PairProduct p, int splits) {
  __shared__ float tile[N][N + 1];
  const long long tiles_m = (p.m + N - 1) / N, tiles_n = (p.n + N - 1) / N, each = p.symmetric ? tiles_m * (tiles_m + 1) / 2 : tiles_m * tiles_n;
  const long long id = p.first + blockIdx.x, matrix = id / each;
  const int in = (int)(id - matrix * each);
  int tm, tn;
  if (p.symmetric) upper_tile(in, tm, tn);
  else tm = (int)(in / tiles_n), tn = (int)(in - tm * tiles_n);
  const Place place{p, matrix, p.scales ? p.scales + 4 * matrix : nullptr};
  const bool columns = place.columns_wanted() && !(p.symmetric && tm == tn);
  const int t = threadIdx.x, chunk = t % (N / 8) * 8;
#pragma unroll
  for (int u = 0; u < N / 32; ++u) {
    const int row = u * 32 + t / (N / 8), i = tm * N + row, j = tn * N + chunk;
    float c[8] = {};
    if (i < p.m && j < p.n) {
      const float *from = p.partial + matrix * p.m * p.n + (long long)i * p.n + j;
      const long long far = p.matrices * p.m * p.n;
      for (int s = 0; s < splits; s += 4) {   // four on their way
        Eight<float> part[4];
#pragma unroll
        for (int q = 0; q < 4; ++q)
          if (s + q < splits) part[q].load<true>(from + (s + q) * far, 8);
#pragma unroll
        for (int q = 0; q < 4; ++q)
          if (s + q < splits) {
            float v[8];
            part[q].get(v);
#pragma unroll
            for (int e = 0; e < 8; ++e) c[e] = c[e] + v[e];
          }
      }
      place.finish(i, j, c);
      place.row(i, j, c);
    }
    if (columns)
#pragma unroll
      for (int e = 0; e < 8; ++e) tile[row][chunk + e] = c[e];
  }
  if (!columns) return;
  __syncthreads();
#pragma unroll
  for (int u = 0; u < N / 32; ++u) {
    const int row = u * 32 + t / (N / 8);
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = tile[chunk + e][row];
    const int i = tm * N + chunk, j = tn * N + row;
    if (i < p.m && j < p.n) place.column(i, j, v);
  }
}

// Matrices that fit into a workgroup's shared memory with their transpose, A and B: all steps in one launch, a workgroup a matrix.  Rows of pairs as above,
// 16 bytes further apart than they are long, so that the 16 rows of a read lie in different banks.  A wave takes every eighth pair of a product's pieces of 16 x 16,
// adjacent ones, which share an operand: what bounds a step is reads of shared memory, the time from one to the sum, and the barriers.  Pieces of X are
// computed both ways round, from the same operands, which costs less than turning them.
constexpr int kSmallWaves = 8, kSmallWg = 64 * kSmallWaves;

struct SmallPlaces {   // bytes
  int x_row, a_row, xt, a, b, all;   // rows of X, and of the others
  __host__ __device__ SmallPlaces(int m, int n) {
    x_row = n * 4 + 16, a_row = m * 4 + 16;
    xt = m * x_row, a = xt + n * a_row, b = a + m * a_row, all = b + m * a_row;
  }
};

typedef _Float16 v4h __attribute__((ext_vector_type(4)));
__device__ __forceinline__ lds_ptr small_place(lds_ptr m, int row_bytes, int i, int j) { return m + i * row_bytes + (j >> 5) * 128 + (j & 31) * 2; }
__device__ __forceinline__ void small_store(lds_ptr p, v4f v) {
  v4h hi, lo;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    hi[e] = (_Float16)v[e];
    lo[e] = (_Float16)(v[e] - (float)hi[e]);
  }
  *LDS(v4h, p) = hi;
  *LDS(v4h, p + 64) = lo;
}
__device__ __forceinline__ v4f small_load(lds_ptr p) {
  const v4h hi = *LDS(v4h, p), lo = *LDS(v4h, p + 64);
  v4f v;
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = (float)hi[e] + (float)lo[e];
  return v;
}

// A wave's pairs of pieces of a product of rows with rows, `across` pieces (an even number) in a row of the result.
template <int P>
struct SmallPairs {
  int mine, ia[P], ib[P];
  __device__ __forceinline__ SmallPairs(int wave, int pairs, int across) {
    mine = (pairs - wave + kSmallWaves - 1) / kSmallWaves;
#pragma unroll
    for (int u = 0; u < P; ++u) {
      const int q = 2 * (u * kSmallWaves + wave), row = q / across;
      ia[u] = __builtin_amdgcn_readfirstlane(row * 16), ib[u] = __builtin_amdgcn_readfirstlane((q - row * across) * 16);
    }
  }
};
// Pieces (ia, ib) and (ia, ib + 16).  c: lane 16 g + i has the sums of a's row i with b's rows 4 g .. 4 g + 3; d, TURNED: of b's row i with a's.
template <bool TURNED>
__device__ __forceinline__ void small_sums(lds_ptr a, int ia, lds_ptr b, int ib, int row_bytes, int steps, v4f (&c)[2], v4f (&d)[2]) {
  const int lane = threadIdx.x & 63, key = (lane & 15) * row_bytes + (lane >> 4) * 16;
  lds_ptr pa = a + (ia * row_bytes + key), pb = b + (ib * row_bytes + key);
#pragma unroll
  for (int h = 0; h < 2; ++h) c[h] = d[h] = v4f{0, 0, 0, 0};
#pragma unroll 1
  for (int k = 0; k < steps; ++k, pa += 128, pb += 128) {
    const v4u ah = *LDS(v4u, pa), al = *LDS(v4u, pa + 64);
    v4u bh[2], bl[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) bh[h] = *LDS(v4u, pb + h * 16 * row_bytes), bl[h] = *LDS(v4u, pb + h * 16 * row_bytes + 64);
#pragma unroll
    for (int part = 0; part < 3; ++part)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const v4u fa = part == 2 ? al : ah, fb = part == 1 ? bl[h] : bh[h];
        c[h] = multiply_halves(fb, fa, c[h]);
        if constexpr (TURNED) d[h] = multiply_halves(fa, fb, d[h]);
      }
  }
}

// P: pairs of pieces of X that a wave has.
template <class T, int P, int BYTES>
__global__ void __launch_bounds__(kSmallWg) k_small(SmallOrthogonal s) {
  __shared__ __align__(16) char shared[BYTES];
  __shared__ double part[kSmallWaves];
  const Orthogonal &o = s.o;
  const long long matrix = s.first + blockIdx.x;
  const int m = (int)o.m, n = (int)o.n, rows = (int)o.rows, cols = (int)o.cols, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
  const SmallPlaces at(m, n);
  const lds_ptr xs = (lds_ptr)shared, xt = xs + at.xt, a = xs + at.a, b = xs + at.b;
  const T *from = static_cast<const T *>(o.g) + matrix * o.g_matrix;
  float v[8 * P];   // rows cols <= m n = 512 pairs, 8 P of them
  double sum = 0.0;
#pragma unroll
  for (int u = 0; u < 8 * P; ++u) {
    const int q = u * kSmallWg + (int)threadIdx.x, r = q / cols;
    v[u] = q < rows * cols ? to_float(from[(long long)r * o.g_row + (q - r * cols)]) : 0.0f;
  }
  for (int q = threadIdx.x; q < at.a / 16; q += kSmallWg) *LDS(v4u, xs + q * 16) = v4u{0, 0, 0, 0};
#pragma unroll
  for (int u = 0; u < 8 * P; ++u) sum = sum + (double)v[u] * (double)v[u];
#pragma unroll
  for (int d = 1; d < 64; d *= 2) sum = sum + __shfl_xor(sum, d);
  if (lane == 0) part[wave] = sum;
  __syncthreads();
  sum = 0.0;
#pragma unroll
  for (int w = 0; w < kSmallWaves; ++w) sum = sum + part[w];
  const double inverse = 1.0 / (sqrt(sum) + o.eps) * (double)o.scale;
#pragma unroll
  for (int u = 0; u < 8 * P; ++u) {
    const int q = u * kSmallWg + (int)threadIdx.x, r = q / cols, c = q - r * cols, xi = o.transposed ? c : r, xj = o.transposed ? r : c;
    if (q < rows * cols) {
      const float x = (float)((double)v[u] * inverse);
      const _Float16 hi = (_Float16)x, lo = (_Float16)(x - (float)hi);
      const lds_ptr p = small_place(xs, at.x_row, xi, xj), pt = small_place(xt, at.a_row, xj, xi);
      *LDS(_Float16, p) = hi, *LDS(_Float16, p + 64) = lo;
      *LDS(_Float16, pt) = hi, *LDS(_Float16, pt + 64) = lo;
    }
  }
  __syncthreads();
  const SmallPairs<P> square(wave, m / 16 * (m / 16) / 2, m / 16), wide(wave, m / 16 * (n / 16) / 2, n / 16);
  for (int k = 0; k < o.steps; ++k) {
    const StepFactors f = s.f[k];
#pragma unroll
    for (int u = 0; u < P; ++u)
      if (u < square.mine) {
        v4f c[2], d[2];
        const int ia = square.ia[u], ib = square.ib[u];
        small_sums<false>(xs, ia, xs, ib, at.x_row, n / 32, c, d);
#pragma unroll
        for (int h = 0; h < 2; ++h) small_store(small_place(a, at.a_row, ia + i, ib + 16 * h + 4 * g), c[h] * f.a);
      }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < P; ++u)
      if (u < square.mine) {
        v4f c[2], d[2];
        const int ia = square.ia[u], ib = square.ib[u];
        small_sums<false>(a, ia, a, ib, at.a_row, m / 32, c, d);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const v4f was = small_load(small_place(a, at.a_row, ia + i, ib + 16 * h + 4 * g));
          small_store(small_place(b, at.a_row, ia + i, ib + 16 * h + 4 * g), c[h] * f.b + was * f.b_extra);
        }
      }
    __syncthreads();
    v4f c[P][2], d[P][2];
#pragma unroll
    for (int u = 0; u < P; ++u)
      if (u < wide.mine) {
        const int ia = wide.ia[u], ib = wide.ib[u];
        small_sums<true>(b, ia, xt, ib, at.a_row, m / 32, c[u], d[u]);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          c[u][h] = c[u][h] * f.x + small_load(small_place(xs, at.x_row, ia + i, ib + 16 * h + 4 * g)) * f.x_extra;
          d[u][h] = d[u][h] * f.x + small_load(small_place(xt, at.a_row, ib + 16 * h + i, ia + 4 * g)) * f.x_extra;
        }
      }
    const bool last = k + 1 == o.steps;
    if (!last) __syncthreads();   // nobody reads X's transpose any more
    T *to = static_cast<T *>(o.x) + matrix * o.x_matrix;
#pragma unroll
    for (int u = 0; u < P; ++u)
      if (u < wide.mine)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int ia = wide.ia[u], ib = wide.ib[u] + 16 * h;
          if (!last) {
            small_store(small_place(xs, at.x_row, ia + i, ib + 4 * g), c[u][h]);
            small_store(small_place(xt, at.a_row, ib + i, ia + 4 * g), d[u][h]);
          } else {
            const int r = (o.transposed ? ib : ia) + i, c0 = (o.transposed ? ia : ib) + 4 * g;
            const v4f x = o.transposed ? d[u][h] : c[u][h];
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (r < rows && c0 + e < cols) to[(long long)r * o.x_row + c0 + e] = from_float<T>(x[e]);
          }
        }
    if (!last) __syncthreads();
  }
}

constexpr int kMostSmall = 163840 - 128;   // bytes of shared memory, less the sums'

// How many pairs of pieces of X a wave has where the matrices go into shared memory, otherwise 0.
int small_pairs(const Orthogonal &o) {
  if (o.by_norm || o.steps < 1 || o.steps > kMostSmallSteps || o.m > 1024 || o.n > 1024 || SmallPlaces((int)o.m, (int)o.n).all > kMostSmall) return 0;
  const int pairs = (int)(o.m * o.n / 512);
  return pairs <= kSmallWaves ? 1 : pairs <= 2 * kSmallWaves ? 2 : pairs <= 5 * kSmallWaves ? 5 : 0;
}

constexpr int kCus = 256;

enum Tile { kTile64Ahead, kTile64, kTile96Ahead, kTile128, kTile256 };
struct Cut {
  Tile tile;
  int side, splits, steps_each;
  double us;   // estimated
};

long long tiles_of(const PairProduct &p, int side) {
  const long long a = (p.m + side - 1) / side, b = (p.n + side - 1) / side;
  return (p.symmetric ? a * (a + 1) / 2 : a * b) * p.matrices;
}

// The cut with the least estimated time, from what was measured: a tile's rate (products of numbers) without its end, the least time of a step, a tile's start, what the
// ends read and write at the rate of memory (half of it is hidden where a CU holds several workgroups), and the join of splits.  Tiles of 64 with a third step on
// its way take 0.3 us a step where a CU has one of them (1024 x 1024 over 1024, symmetric: 12.6 us; 17.8 with two steps), but where it has more than two they
// have less room (2048 x 8192 over 2048: 235 us, 227); tiles of 96 fill the device once where those of 64 are more (2048 x 2048 over 2048, symmetric: 36 us, 39).
// Measured and estimated, us: 2048 x 8192 over 2048 by 256 182 and 186, by 128 195 and 211; 16 times 416 x 2112 over 416 by 64 71 and 71; 2048 x 2048 over 8192,
// symmetric, in 7 parts of 256 115 and 103.
struct Kind {
  Tile tile;
  int side, a_cu;
  double rate, least;
};
constexpr Kind kKinds[] = {{kTile64Ahead, 64, 2, 310e12, 0.3}, {kTile64, 64, 4, 310e12, 0.5}, {kTile96Ahead, 96, 1, 400e12, 0.55}, {kTile128, 128, 2, 370e12, 0.6}, {kTile256, 256, 1, 480e12, 1.7}};

Cut cut_of(const PairProduct &p) {
  const int steps = (int)(p.k / 32);
  Cut best = {};
  double least = 0.0;
  const double entries = (double)p.matrices * p.m * p.n * (p.symmetric ? 0.5 : 1.0), end = entries * (p.symmetric ? 8.0 : 12.0) / 5e6;
  for (const Kind &c : kKinds) {
    const long long tiles = tiles_of(p, c.side), room = (long long)c.a_cu * kCus;
    if ((c.tile == kTile64Ahead || c.tile == kTile96Ahead) && tiles > room) continue;
    for (int splits = 1; splits == 1 || (splits <= 16 && splits * 4 <= steps && tiles * splits <= room); ++splits) {
      const int each = (steps + splits - 1) / splits;
      const double one = 2.0 * c.side * c.side * 32.0 / (c.rate / kCus) * 1e6;
      long long left = tiles * splits;
      double us = 0.0;
      while (left > 0) {
        const long long now = left < room ? left : room, rounds = left / now;
        const double step = (double)((now + kCus - 1) / kCus) * one;
        us += (double)rounds * (3.0 + each * (step > c.least ? step : c.least));
        left -= rounds * now;
      }
      us += splits > 1 ? 5.0 + (double)splits * entries * 8.0 / 4e6 + end : c.a_cu == 1 ? end : 0.5 * end;
      if (least == 0.0 || us < least) least = us, best = {c.tile, c.side, splits, each, us};
    }
  }
  best.splits = (steps + best.steps_each - 1) / best.steps_each;
  return best;
}

template <int SIDE, int WM, int WN, int S>
void launch_tiles(const PairProduct &p, const Cut &c, hipStream_t s) {
  const int tm = (int)((p.m + SIDE - 1) / SIDE), tn = (int)((p.n + SIDE - 1) / SIDE);
  in_launches(p, tiles_of(p, SIDE), 64 * WM * WN, [&](const PairProduct &part, unsigned x) {
    k_pair_product<SIDE, SIDE, WM, WN, S><<<dim3(x, (unsigned)c.splits), 64 * WM * WN, 0, s>>>(part, tm, tn, c.steps_each);
  });
}

template <int N>
void launch_join(const PairProduct &p, const Cut &c, hipStream_t s) {
  in_launches(p, tiles_of(p, N), N * 4, [&](const PairProduct &part, unsigned x) { k_pair_join<N><<<dim3(x), N * 4, 0, s>>>(part, c.splits); });
}

void launch_pairs(PairProduct p, const Cut &c, float *partial, hipStream_t s) {
  const bool joined = c.splits > 1 || p.scales;
  p.partial = joined ? partial : nullptr;
  switch (c.tile) {
    case kTile64Ahead: launch_tiles<64, 2, 2, 3>(p, c, s); break;
    case kTile64: launch_tiles<64, 2, 2, 2>(p, c, s); break;
    case kTile96Ahead: launch_tiles<96, 2, 3, 3>(p, c, s); break;
    case kTile128: launch_tiles<128, 2, 2, 2>(p, c, s); break;
    case kTile256: launch_tiles<256, 2, 4, 2>(p, c, s); break;
  }
  if (joined) c.side % 64 == 0 ? launch_join<64>(p, c, s) : launch_join<32>(p, c, s);
}

// The three products of a step, without their operands' places.
PairProduct shape_of(const Orthogonal &o, int which) {
  PairProduct p = {};
  p.matrices = o.matrices;
  p.m = o.m, p.n = which == 2 ? o.n : o.m, p.k = which == 0 ? o.n : o.m;
  p.symmetric = which == 1 || (which == 0 && !o.by_norm);   // by norm A is an fp32 matrix, whose tiles are stored once
  return p;
}

// Two steps can be taken at once, from step k on: with A of X and B = b A + c A A the next step's A is (a + B) A (a + B) = N B + a^2 A, N = B A + 2 a A, and
// both steps are X <- a^2 X + R X with R = B' B + a B' + a B, B' of that A.  Three symmetric products of [m][m] in the place of A from X and one of
// B X: 9 of 26 m^3 less where n = 4 m.  A's rounding errors then count (a + b s^2 + ..)^2 times, 12 times where singular values are small, beside those of X itself.
// For fp32 the last two steps are taken so, whose errors no later step multiplies; for bf16, whose store rounds 2^13 times as much, all but the first.
struct Cuts {   // of a step's products
  Cut c[3];
  explicit Cuts(const Orthogonal &o) {
    for (int w = 0; w < 3; ++w) c[w] = cut_of(shape_of(o, w));
  }
  bool two_at_once(const Orthogonal &o, int k) const {
    if (o.by_norm || o.steps - k < 2 || (o.type == kF32 ? o.steps - k != 2 : k == 0 || (o.steps - k) % 2 != 0)) return false;
    return c[0].us + c[2].us > 3.0 * (c[1].us + 1.5);
  }
};

// How many workgroups sum up the squares of a matrix.
int norm_parts(long long rows, long long cols) {
  const long long eights = rows * ((cols + 7) / 8), parts = (eights + kWg * 8 - 1) / (kWg * 8);
  return (int)(parts < 1 ? 1 : parts > 1024 ? 1024 : parts);
}

struct Layout {   // of the workspace, in bytes
  size_t squares, squares_a, scales, xs, xt[2], a, b, c, d, x, partial, all;
};
Layout layout_of(const Orthogonal &o) {
  Layout l = {};
  size_t at = 0;
  const auto take = [&](size_t bytes) {
    const size_t here = at;
    at += (bytes + 255) & ~(size_t)255;
    return here;
  };
  if (small_pairs(o)) return l;
  l.squares = take(sizeof(double) * (size_t)o.matrices * o.parts);
  if (o.steps > 0) {
    const size_t wide = (size_t)o.matrices * o.m * o.n * 4, square = (size_t)o.matrices * o.m * o.m * 4;
    l.xs = take(wide), l.xt[0] = take(wide);
    if (!o.by_norm) l.xt[1] = take(wide);
    l.a = take(square), l.b = take(square);
    if (o.by_norm) {
      const long long x = o.rows * o.cols, a = o.m * o.m;
      l.squares_a = take(sizeof(double) * (size_t)o.matrices * norm_parts(o.m, o.m));
      l.scales = take(sizeof(float) * 4 * (size_t)o.matrices);
      l.x = take(sizeof(float) * (size_t)o.matrices * (x > a ? x : a));
    }
    const Cuts cuts(o);
    if (o.steps > 1 && cuts.two_at_once(o, o.steps - 2)) l.c = take(square), l.d = take(square);
    size_t most = 0;
    for (int w = 0; w < 3; ++w) {
      const PairProduct p = shape_of(o, w);
      const Cut &c = cuts.c[w];
      const size_t bytes = c.splits > 1 || (o.by_norm && w > 0) ? (size_t)c.splits * p.matrices * p.m * p.n * 4 : 0;
      most = bytes > most ? bytes : most;
    }
    l.partial = take(most);
  }
  l.all = at;
  return l;
}

// The largest |a s + b s^3 + c s^5| for s in [0, most].
double largest(double a, double b, double c, double most) {
  const auto at = [&](double s) { return std::fabs(s * (a + s * s * (b + s * s * c))); };
  double v = at(most);
  const double d = 9.0 * b * b - 20.0 * a * c;   // of the slope a + 3 b u + 5 c u^2, u = s^2
  if (!(d >= 0.0)) return v;
  // its roots, without a difference of numbers that are nearly the same: next to c = 0 that would lose the one near -a / (3 b)
  const double q = -0.5 * (3.0 * b + std::copysign(std::sqrt(d), b));
  for (const double u : {q / (5.0 * c), a / q})   // infinite or no number where there is none
    if (u > 0.0 && u < most * most) v = std::fmax(v, at(std::sqrt(u)));
  return v;
}
// ... and |b u + c u^2| for u in [0, most].
double largest_inner(double b, double c, double most) {
  const auto at = [&](double u) { return std::fabs(u * (b + c * u)); };
  double v = at(most);
  if (c != 0.0 && -b / (2.0 * c) > 0.0 && -b / (2.0 * c) < most) v = std::fmax(v, at(-b / (2.0 * c)));
  return v;
}

constexpr double kLeast = 1.0 / (1ll << 40), kMost = (double)(1ll << 40);

// The largest power of two whose product with numbers of this size fp16 holds, with room for their rounding.
int exponent_for(double size) { return (int)std::floor(std::log2(60000.0 / std::fmax(size, kLeast))); }

}  // namespace

bool orthogonal_bounded(double a, double b, double c, int steps) {
  double s = 1.0;
  for (int k = 0; k < steps; ++k) {
    if (largest_inner(b, c, s * s) > kMost) return false;
    s = largest(a, b, c, s);
    if (!(s <= kMost)) return false;
  }
  return true;
}

// Whether the bound may be more than a few times what small singular values come to, |a| a step: pairs then lose digits of fp32's 24 (a matrix of 2^24 entries has some 2^-12
// of its norm in each, 2^29 times what a pair is held to).  Polynomials that bring singular values towards 1 stay below |a|.
bool orthogonal_by_norm(double a, double b, double c, int steps) {
  constexpr double kTimes = 4.0, kSmall = 1.0 / (1 << 20);
  double s = 1.0, small = 1.0;
  for (int k = 0; k < steps; ++k) {
    if (std::fabs(a) < kLeast || largest_inner(b, c, s * s) > kTimes * std::fabs(a)) return true;
    s = largest(a, b, c, s), small *= std::fabs(a);
    if (k + 1 < steps && (s > kTimes * small || s < kSmall)) return true;
  }
  return false;
}

void orthogonal_sides(Orthogonal *o) {
  o->transposed = o->rows > o->cols;
  o->m = up32(o->transposed ? o->cols : o->rows), o->n = up32(o->transposed ? o->rows : o->cols);
  o->parts = norm_parts(o->rows, o->cols);
}

namespace {

void launch_start(const Orthogonal &o, hipStream_t s) {
  in_launches(o, o.matrices * o.parts, kWg, [&](const Orthogonal &part, unsigned x) {
    if (o.type == kF32) k_squares<float><<<dim3(x), kWg, 0, s>>>(part);
    else k_squares<bf16><<<dim3(x), kWg, 0, s>>>(part);
  });
  const long long tr = (o.rows + 63) / 64, tc = (o.cols + 63) / 64;
  in_launches(o, o.matrices * tr * tc, kWg, [&](const Orthogonal &part, unsigned x) {
    if (o.steps == 0) {
      if (o.type == kF32) k_start<float, false><<<dim3(x), kWg, 0, s>>>(part, tr, tc);
      else k_start<bf16, false><<<dim3(x), kWg, 0, s>>>(part, tr, tc);
    } else {
      if (o.type == kF32) k_start<float, true><<<dim3(x), kWg, 0, s>>>(part, tr, tc);
      else k_start<bf16, true><<<dim3(x), kWg, 0, s>>>(part, tr, tc);
    }
  });
}

// All steps by norm.
void launch_by_norm(const Orthogonal &o, const Layout &l, char *w, hipStream_t s) {
  constexpr int kPower = 15;   // numbers of size 1 are held times 2^15
  constexpr double kNothing = 1e-300;   // beside a norm: a matrix of zeros stays one
  const float down = std::ldexp(1.0f, -kPower);
  const Cuts cuts(o);
  float *partial = reinterpret_cast<float *>(w + l.partial);
  Orthogonal x = o, y, a = o;
  x.scales = reinterpret_cast<float *>(w + l.scales);
  a.type = kF32, a.transposed = 0, a.rows = a.cols = o.m, a.n = o.m;
  a.g = w + l.x, a.g_row = o.m, a.g_matrix = o.m * o.m;
  a.squares = reinterpret_cast<double *>(w + l.squares_a), a.parts = norm_parts(o.m, o.m);
  a.xs = w + l.a, a.xt = w + l.b;   // its transpose, the same, is overwritten by B
  a.eps = kNothing, a.scale = 1 << kPower;
  for (int k = 0; k < o.steps; ++k) {
    if (k > 0) x.g = w + l.x, x.type = kF32, x.g_row = o.cols, x.g_matrix = o.rows * o.cols;   // from the step before
    y = x, y.eps = kNothing, y.scale = 1 << kPower;
    launch_start(y, s);
    PairProduct p = shape_of(o, 0);   // A'
    p.a = p.b = o.xs;
    p.factor = down * down;
    p.x = w + l.x, p.x_row = p.x_rows = p.x_cols = o.m, p.x_matrix = o.m * o.m, p.type = kF32;
    launch_pairs(p, cuts.c[0], partial, s);
    launch_start(a, s);
    in_launches(x, (o.matrices + kWg / 64 - 1) / (kWg / 64), kWg,
                [&](const Orthogonal &part, unsigned grid) { k_start_scales<<<dim3(grid), kWg, 0, s>>>(part, a.squares, a.parts, k == 0); });
    p = shape_of(o, 1);               // B'
    p.a = p.b = p.e = w + l.a, p.out = p.out_t = w + l.b;
    p.factor = down * down, p.extra = down, p.scales = x.scales;
    launch_pairs(p, cuts.c[1], partial, s);
    p = shape_of(o, 2);               // n a Y + n^3 B' Y
    p.a = w + l.b, p.b = o.xt, p.e = o.xs;
    p.factor = p.extra = down, p.scales = x.scales + 2;
    const bool last = k + 1 == o.steps;
    p.x = last ? o.x : w + l.x, p.x_matrix = last ? o.x_matrix : o.rows * o.cols, p.x_row = last ? o.x_row : o.cols, p.type = last ? o.type : kF32;
    p.x_rows = o.rows, p.x_cols = o.cols, p.x_transposed = o.transposed;
    launch_pairs(p, cuts.c[2], partial, s);
  }
}

}  // namespace

size_t orthogonal_scratch(const Orthogonal &o) { return layout_of(o).all; }

hipError_t launch_orthogonalize(const Orthogonal &call, void *workspace, hipStream_t s) {
  Orthogonal o = call;
  const Layout l = layout_of(o);
  char *w = static_cast<char *>(workspace);
  o.squares = reinterpret_cast<double *>(w + l.squares);
  o.xs = w + l.xs, o.xt = w + l.xt[0];
  double size = 1.0;
  int ex = exponent_for(size);
  o.scale = std::ldexp(1.0f, ex);
  const auto factors = [&](int k) {   // of step k, and on to the next
    const double next = largest(o.a, o.b, o.c, size);
    const int ea = exponent_for(size * size), eb = exponent_for(largest_inner(o.b, o.c, size * size)), en = k + 1 < o.steps ? exponent_for(next) : 0;
    const StepFactors f = {std::ldexp(1.0f, ea - 2 * ex), (float)std::ldexp(o.c, eb - 2 * ea), (float)std::ldexp(o.b, eb - ea), std::ldexp(1.0f, en - eb - ex),
                           (float)std::ldexp(o.a, en - ex)};
    size = next, ex = en;
    return f;
  };
  if (const int pairs = small_pairs(o)) {
    const int bytes = SmallPlaces((int)o.m, (int)o.n).all;
    SmallOrthogonal small = {o, {}, 0};
    for (int k = 0; k < o.steps; ++k) small.f[k] = factors(k);
    in_launches(small, o.matrices, kSmallWg, [&](const SmallOrthogonal &part, unsigned x) {
      const auto go = [&](auto t) {
        typedef decltype(t) T;
        // three workgroups a CU (by their registers) or two (by shared memory) where they fit
        if (pairs == 1 && bytes <= 40960 - 128) k_small<T, 1, 40960 - 128><<<dim3(x), kSmallWg, 0, s>>>(part);
        else if (pairs == 1 && bytes <= 81920 - 128) k_small<T, 1, 81920 - 128><<<dim3(x), kSmallWg, 0, s>>>(part);
        else if (pairs <= 2) k_small<T, 2, kMostSmall><<<dim3(x), kSmallWg, 0, s>>>(part);
        else k_small<T, 5, kMostSmall><<<dim3(x), kSmallWg, 0, s>>>(part);
      };
      if (o.type == kF32) go(float());
      else go(bf16());
    });
    return hipGetLastError();
  }
  if (o.by_norm) {
    launch_by_norm(o, l, w, s);
    return hipGetLastError();
  }
  launch_start(o, s);
  float *partial = reinterpret_cast<float *>(w + l.partial);
  if (o.steps == 0) return hipGetLastError();
  const Cuts cuts(o);
  const auto square = [&](size_t a, size_t b, size_t out, double factor, size_t e, double extra, size_t e2 = 0, double extra2 = 0.0) {   // symmetric; 0: no such matrix
    PairProduct p = shape_of(o, 1);
    p.a = w + a, p.b = w + b, p.out = p.out_t = w + out;
    p.factor = (float)factor;
    if (e) p.e = w + e, p.extra = (float)extra;
    if (e2) p.e2 = w + e2, p.extra2 = (float)extra2;
    launch_pairs(p, cuts.c[1], partial, s);
  };
  int turn = 0;
  for (int k = 0; k < o.steps;) {
    const bool twice = cuts.two_at_once(o, k);
    const bool last = k + (twice ? 2 : 1) == o.steps;
    const auto two = [](int e) { return std::ldexp(1.0, e); };
    const double inner = largest_inner(o.b, o.c, size * size), next = largest(o.a, o.b, o.c, size);
    const int ea = exponent_for(size * size), eb = exponent_for(inner);
    PairProduct p = shape_of(o, 0);   // A
    p.a = p.b = o.xs, p.out = p.out_t = w + l.a;
    p.factor = (float)two(ea - 2 * ex);
    launch_pairs(p, cuts.c[0], partial, s);
    square(l.a, l.a, l.b, o.c * two(eb - 2 * ea), l.a, o.b * two(eb - ea));   // B
    size_t by = l.b;
    int ey = eb;
    double own = o.a;
    if (twice) {
      const double inner2 = largest_inner(o.b, o.c, next * next);
      const int en = exponent_for(size * size * (inner + 2.0 * std::fabs(o.a))), ea2 = exponent_for(next * next), eb2 = exponent_for(inner2);
      ey = exponent_for(inner2 * inner + std::fabs(o.a) * (inner2 + inner));
      square(l.b, l.a, l.c, two(en - eb - ea), l.a, 2.0 * o.a * two(en - ea));                                       // N
      square(l.c, l.b, l.d, two(ea2 - en - eb), l.a, o.a * o.a * two(ea2 - ea));                                     // the next step's A
      square(l.d, l.d, l.c, o.c * two(eb2 - 2 * ea2), l.d, o.b * two(eb2 - ea2));                                    // B'
      square(l.c, l.b, l.d, two(ey - eb2 - eb), l.c, o.a * two(ey - eb2), l.b, o.a * two(ey - eb));                  // R
      by = l.d, own = o.a * o.a;
    }
    const double then = twice ? largest(o.a, o.b, o.c, next) : next;
    const int to = last ? 0 : exponent_for(then);
    p = shape_of(o, 2);               // a X + B X, or a^2 X + R X
    p.a = w + by, p.b = w + l.xt[turn], p.e = o.xs, p.out = o.xs, p.out_t = w + l.xt[1 - turn];
    p.factor = (float)two(to - ey - ex), p.extra = (float)(own * two(to - ex));
    if (last) p.x = o.x, p.x_matrix = o.x_matrix, p.x_row = o.x_row, p.x_rows = o.rows, p.x_cols = o.cols, p.x_transposed = o.transposed, p.type = o.type;
    launch_pairs(p, cuts.c[2], partial, s);
    size = then, ex = to, turn = 1 - turn;
    k += twice ? 2 : 1;
  }
  return hipGetLastError();
}

}  // namespace qoda
