// Matrix products with what follows them fused into their stores: x w^T, dz w and dz^T x of include/qoda_operators.h.
//
// One kernel for the three forms and both types, on the matrix cores (16 x 16 sums by 32 bf16 products or 4 times 4 fp32 products an
// entry).  A workgroup computes a tile of BM x BN sums, in steps of 128 bytes along l (64 bf16, 32 fp32): the step's two operand tiles
// lie in shared memory twice, and while one pair is multiplied the next is on its way.  A lane's piece of an operand is 16 bytes: 8
// bf16 (one matrix instruction) or 4 fp32 (four).
//
// Operands whose entries are adjacent along l ("rows") lie in shared memory as rows of 128 bytes; the others ("columns") as they are, a
// row for each l, and are transposed as they are read (bf16: by the transposing read, which hands each lane four entries of a column).
// In both the 16-byte chunks of a row are permuted by an exclusive or with bits of the row's number, so that the lanes of a read hit different banks.
//
// The matrix instruction's first operand is b's piece: a lane then holds four sums adjacent in a row of c, and b's entries are dealt
// to the instructions so that those of two instructions are eight adjacent ones: 16 bytes of bf16 to store, and one block of lots.
//
// Measured, bf16: 16384 x 8192 x 2048 441 us (1247 TFLOP/s; the library's product 424), with dropout and residual 471; the input
// gradient of 8192 x 8192 x 2048 through gelu 308, of which 225 the product, 45 the read of pre and 30 the slope; the weight gradient of
// 6144 x 2048 over 8192 rows 198.  fp32: 4096 x 2048 x 2048 242 us (142 TFLOP/s), its input gradient 249.  The matrix cores are busy 93 % of the CUs' time in
// fp32 and 39 to 56 % in bf16, whose tiles' ends wait for memory: a CU holds one such tile, so that nothing else runs meanwhile.  Short sums are bound by
// a tile's start and end: 3300 x 410 x 2100 16 us for 7 steps.

#include "qoda_product_device.h"

namespace qoda {

namespace {

// (Tiles of 128 are held to the registers of two waves a SIMD, which plan_of() counts on; without that the fp32 input gradient's took 272.)
template <class T, int FORM, int BM, int BN, int WM, int WN, bool DIRECT>
__global__ void __launch_bounds__(64 * WM * WN, BN == 128 && BM == 128 ? 2 : 1) k_product(Product p, int tiles_m, int tiles_n, int steps_each, bool loose) {
  constexpr int WG = 64 * WM * WN, FM = BM / WM / 16, FN = BN / WN / 32;
  typedef Operand<T, FORM != kProductColumns, 0, BM, WG, DIRECT> A;
  typedef Operand<T, FORM == kProductRows, 1, BN, WG, DIRECT> B;
  constexpr int kStep = A::kStep;
  __shared__ __align__(16) char a0[BM * kStepBytes], b0[BN * kStepBytes], a1[BM * kStepBytes], b1[BN * kStepBytes];

  int tm, tn;
  tile_of((int)(p.first + blockIdx.x), tiles_m, tiles_n, tm, tn);
  const int i0 = tm * BM, j0 = tn * BN;
  const int k0 = (int)blockIdx.y * steps_each * kStep;
  const int k = (long long)p.k - k0 < (long long)steps_each * kStep ? p.k - k0 : steps_each * kStep;   // of this split
  const int steps = (k + kStep - 1) / kStep;
  A a;
  B b;
  a.start(p.a, p.lda, i0, p.m, k0, k);
  b.start(p.b, p.ldb, j0, p.n, k0, k);
  const int wave = threadIdx.x / 64, wm = wave / WN * (BM / WM), wn = wave % WN * (BN / WN);

  v4f c[FM][2 * FN];
#pragma unroll
  for (int x = 0; x < FM; ++x)
#pragma unroll
    for (int y = 0; y < 2 * FN; ++y) c[x][y] = v4f{0, 0, 0, 0};

  // the sums of a's columns: the waves of the first column of tiles share them, each for some of its rows of c
  constexpr int FS = (FM + WN - 1) / WN;
  const bool with_sums = FORM == kProductColumns && p.sums && tn == 0 && wave % WN * FS < FM;
  float sum[FS] = {};

  typedef v4u PiecesA[FM];
  typedef v4u PiecesB[2 * FN];
  u32 key_a = A::lane_key(wm), key_b = B::lane_key(wn);
  const auto read = [&](PiecesA &fa, PiecesB &fb, lds_ptr ta, lds_ptr tb, int s) {
    // the pieces' places are made anew each time: kept, they would take the registers that pieces need
    asm volatile("" : "+v"(key_a), "+v"(key_b));
#pragma unroll
    for (int y = 0; y < 2 * FN; ++y) fb[y] = B::piece(tb, key_b, wn, y / 2 * 32, y & 1, s);
#pragma unroll
    for (int x = 0; x < FM; ++x) fa[x] = A::piece(ta, key_a, wm, x * 16, 0, s);
  };
  const u32 key_s = A::lane_key(wm + wave % WN * FS * 16);
  const auto add_up = [&](lds_ptr ta) {
    if constexpr (FORM == kProductColumns)
      if (with_sums)
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int x = 0; x < FS; ++x) sum[x] = sum[x] + chunk_sum<T>(A::piece(ta, key_s, wm + wave % WN * FS * 16, x * 16, 0, s));
  };
  const auto multiply_all = [&](const PiecesA &fa, const PiecesB &fb) {
#pragma unroll
    for (int x = 0; x < FM; ++x)
#pragma unroll
      for (int y = 0; y < 2 * FN; ++y) c[x][y] = multiply<T>(fb[y], fa[x], c[x][y]);
  };
  const lds_ptr ta[2] = {(lds_ptr)a0, (lds_ptr)a1}, tb[2] = {(lds_ptr)b0, (lds_ptr)b1};

  // While a step's first half is multiplied its second half is read from shared memory, and while that is multiplied the next step's first
  // half: the matrix cores have work on both sides of the barrier.  It stands between the halves, when everybody has read the step, so
  // that the step after the next may take its place.
  // Direct loads move whole steps only.  A last step that ends inside goes by way of registers and is the first to be taken: its loads
  // and those of the whole step behind it are then on their way together.  So does the last step where rows are not aligned to chunks
  // (loose): the chunk over a row's end, if any, then reads into the next row, which has to be there; an aligned one ends in the same 16 bytes.
  v4u ra[A::kMine], rb[B::kMine];
  const int ragged = DIRECT && (loose || k % kStep != 0) ? 1 : 0;
  const auto request = [&](int t, lds_ptr to_a, lds_ptr to_b) {   // step t in the order in which they are taken
    if constexpr (DIRECT) {
      a.direct((t - ragged) * kStep, to_a);
      b.direct((t - ragged) * kStep, to_b);
    } else {   // by way of registers, which then take the step after it
      A::store(ra, to_a);
      B::store(rb, to_b);
      if (t + 1 < steps) {
        a.fetch((t + 1) * kStep, ra);
        b.fetch((t + 1) * kStep, rb);
      }
    }
  };
  if (steps > 0) {
    if (!DIRECT || ragged) {
      const int first = ragged ? (steps - 1) * kStep : 0;
      a.fetch(first, ra);
      b.fetch(first, rb);
    }
    if (ragged) {
      if (steps > 1) request(1, ta[1], tb[1]);
      A::store(ra, ta[0]);
      B::store(rb, tb[0]);
    } else {
      request(0, ta[0], tb[0]);
      if (steps > 1) request(1, ta[1], tb[1]);
    }
    PiecesA fa0, fa1;
    PiecesB fb0, fb1;
    arrived();
    read(fa0, fb0, ta[0], tb[0], 0);
    for (int t = 0; t < steps; t += 2) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
        if (t + h < steps) {
          read(fa1, fb1, ta[h], tb[h], 1);
          multiply_all(fa0, fb0);
          add_up(ta[h]);
          arrived();   // the next step is there, and nobody reads this one any more
          if (t + h + 2 < steps) request(t + h + 2, ta[h], tb[h]);
          if (t + h + 1 < steps) read(fa0, fb0, ta[1 - h], tb[1 - h], 0);
          multiply_all(fa1, fb1);
          __builtin_amdgcn_sched_barrier(0);
        }
    }
  }

  const int lane = threadIdx.x & 63, g = lane >> 4;
  if constexpr (FORM == kProductColumns)
    if (with_sums)
#pragma unroll
      for (int x = 0; x < FS; ++x) {
        float v = sum[x];   // of a quarter of every step's l
        v = v + __shfl_xor(v, 16);
        v = v + __shfl_xor(v, 32);
        const int i = i0 + wm + (wave % WN * FS + x) * 16 + lane;
        if (lane < 16 && i < p.m) {
          if (p.partial) p.partial[(long long)gridDim.y * p.m * p.n + (long long)blockIdx.y * p.m + i] = v;
          else p.sums[i] = p.accumulate ? p.sums[i] + v : v;
        }
      }
  const auto row = [&](int x) { return i0 + wm + x * 16 + (lane & 15); };
  const auto column = [&](int y) { return j0 + wn + y * 32 + g * 8; };
  const auto sums = [&](int x, int y, float (&v)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = c[x][2 * y + e / 4][e & 3];
  };
  if (p.partial) {
#pragma unroll
    for (int x = 0; x < FM; ++x)
#pragma unroll
      for (int y = 0; y < FN; ++y)
        if (row(x) < p.m && column(y) < p.n) {
          float v[8];
          sums(x, y, v);
          store8(p.partial + ((long long)blockIdx.y * p.m + row(x)) * p.n + column(y), p.n - column(y), v);
        }
    return;
  }
  by_activation<FORM>(p.activation, [&](auto a) {
    // in parts of at most four rows, whose reads are all on their way before the first is needed
    constexpr int kPart = FM % 4 == 0 ? 4 : FM % 3 == 0 ? 3 : FM;
#pragma unroll
    for (int x0 = 0; x0 < FM; x0 += kPart) {
      Beside<T, FORM, decltype(a)::value> beside[kPart][FN];
#pragma unroll
      for (int x = 0; x < kPart; ++x)
#pragma unroll
        for (int y = 0; y < FN; ++y)
          if (row(x0 + x) < p.m && column(y) < p.n) beside[x][y].load(p, row(x0 + x), column(y), p.n - column(y));
#pragma unroll
      for (int x = 0; x < kPart; ++x)
#pragma unroll
        for (int y = 0; y < FN; ++y)
          if (row(x0 + x) < p.m && column(y) < p.n) {
            float v[8];
            sums(x0 + x, y, v);
            finish(p, beside[x][y], row(x0 + x), column(y), p.n - column(y), v);
          }
    }
  });
}

// x w^T for up to 16 rows of x: w is read once and that is the time.  A workgroup takes 16 rows of w, its NW waves the runs of 128 bytes along l in
// turn, straight into the matrix instruction's registers: a lane's 32 bytes of a run are its pieces of two instructions (the
// order along l is the same for both operands, and of no matter).  The waves' sums are joined in shared memory.  2048 x 8192 of bf16, one row:
// 10.5 us a call (3.2 TB/s; empty launches of one stream follow each other in 5); by tiles of 128 with the sum in one part 25.
template <class T, int NW>
__global__ void __launch_bounds__(64 * NW) k_few_rows(Product p) {
  constexpr int E = 16 / (int)sizeof(T), kRun = 8 * E, kAhead = NW > 4 ? (sizeof(T) == 4 ? 2 : 4) : 8;
  __shared__ v4f part[NW][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x / 64, i = lane & 15, g = lane >> 4;
  const int j0 = (int)(p.first + blockIdx.x) * 16;
  const T *b = static_cast<const T *>(p.b) + (long long)(j0 + i < p.n ? j0 + i : p.n - 1) * p.ldb;
  const T *a = static_cast<const T *>(p.a) + (long long)(i < p.m ? i : 0) * p.lda;
  v4f c = {0, 0, 0, 0};
  for (int l0 = wave * kRun; l0 < p.k; l0 += NW * kRun * kAhead) {
    v4u fb[kAhead][2], fa[kAhead][2];
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int l = l0 + u * NW * kRun + (2 * g + h) * E;
        fb[u][h] = load_chunk<T>(b + l, p.k - l);
        fa[u][h] = load_chunk<T>(a + l, i < p.m ? p.k - l : 0);
      }
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h) c = multiply<T>(fb[u][h], fa[u][h], c);
  }
  part[wave][lane] = c;
  __syncthreads();
  // sums of column 4 g + r of the 16 and row i lie in lane 16 g + i, place r
  const int row = (int)threadIdx.x / 2, j = (int)(threadIdx.x & 1) * 8;
  if (row < p.m && j0 + j < p.n) {
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      v[e] = part[0][(j + e) / 4 * 16 + row][e & 3];
#pragma unroll
      for (int w = 1; w < NW; ++w) v[e] = v[e] + part[w][(j + e) / 4 * 16 + row][e & 3];
    }
    by_activation<kProductRows>(p.activation, [&](auto x) {
      Beside<T, kProductRows, decltype(x)::value> beside;
      beside.load(p, row, j0 + j, p.n - j0 - j);
      finish(p, beside, row, j0 + j, p.n - j0 - j, v);
    });
  }
}

// How a product is cut.
enum Tile { kFewRows, kTile32, kTile64, kTile128, kTile192, kTile256 };
struct Plan {
  Tile tile;
  bool direct, loose;
  int tiles_m, tiles_n, splits, steps_each;
};

constexpr int kCus = 256;

// What a cut would take, in us, from what was measured: the matrix cores' rate in a tile of each size, the time of a step that nothing but its
// loads bounds, of a tile's start and end, and of the launch that joins splits.  (3300 x 410 x 832: 16 us with splits by the number of tiles
// alone, 9 without; the fp32 weight gradient of 2100 x 410 over 3300 rows 82 unsplit, 64 in three parts; that of 64 x 64 over 100000 rows 47 in 16
// parts, 36 in as many as this has it take.)
double time_of(const Product &p, int bm, int bn, int a_cu, double rate, long long tiles, int steps, int splits) {
  const int step = kStepBytes / (p.type == kF32 ? 4 : 2), steps_each = (steps + splits - 1) / splits;
  const double flops = 2.0 * bm * bn * step, whole = rate / kCus;
  long long left = tiles * splits;
  double us = 0.0;
  while (left > 0) {   // workgroups that share a CU share its matrix cores; the last ones are fewer
    const long long now = left < (long long)a_cu * kCus ? left : (long long)a_cu * kCus;
    const long long rounds = left / now;
    const int sharing = (int)((now + kCus - 1) / kCus);
    const double alone = bn == 256 || sharing > 2 ? 1.0 : sharing == 2 ? (a_cu > 2 ? 1.1 : 1.0) : 1.5;   // too few waves to fill a SIMD's gaps
    const double one = alone * sharing * flops / whole * 1e6;
    us += (double)rounds * (2.0 + steps_each * (one > 0.5 ? one : 0.5));
    left -= rounds * now;
  }
  if (splits > 1) us += 5.0 + 0.4 * splits + (double)splits * p.m * p.n * 8.0 / 4e6;
  return us;
}

Plan plan_of(const Product &p) {
  Plan q = {};
  const int e = p.type == kF32 ? 4 : 2, step = kStepBytes / e;
  q.splits = 1;
  if (p.m == 0 || (p.n == 0 && !p.sums)) return q;   // nothing to launch
  if (p.form == kProductRows && p.m <= 16) {
    q.tile = kFewRows;
    q.tiles_m = 1, q.tiles_n = (p.n + 15) / 16;
    return q;
  }
  // direct loads: from whole words, by 32-bit offsets inside a tile
  const auto fits = [&](const void *v, long long ld, bool rows, int bytes) {
    return reinterpret_cast<uintptr_t>(v) % bytes == 0 && ld * e % bytes == 0 && (rows ? 256 : step) * ld * e < (1ll << 31);
  };
  const auto both = [&](int bytes) { return fits(p.a, p.lda, p.form != kProductColumns, bytes) && fits(p.b, p.ldb, p.form == kProductRows, bytes); };
  q.loose = !both(16);
  // (loose, across l: the next row, which a chunk over a row's end reads into, is at least a chunk)
  const bool wide_rows = (p.form == kProductRows || p.n >= 8) && (p.form != kProductColumns || p.m >= 8);
  q.direct = p.n > 0 && both(4) && (!q.loose || wide_rows);
  const auto tiles = [&](int bm, int bn) { return (long long)((p.m + bm - 1) / bm) * (p.n > 0 ? (p.n + bn - 1) / bn : 1); };
  const int steps = p.k > 0 ? (p.k + step - 1) / step : 1;
  int bm, bn;
  if (p.m <= 32) {
    // few rows: the other operand is read once, by as many workgroups as fill the device, in parts of at least four steps, and not so many that
    // their join, which adds them one after the other, takes longer than they do
    q.tile = kTile32, bm = 32, bn = 128;
    const long long want = 4 * kCus / tiles(bm, bn), most = steps / 4 < 64 ? steps / 4 : 64;
    q.splits = (int)(want < most ? want : most);
    if (q.splits < 2) q.splits = 1;
  } else {
    // TFLOP/s of whole tiles, 16384 x 8192 x 2048 and 4096 x 2048 x 2048: bf16 1250 (256), 1200 (192 x 256), 1060 (128), 800 (64); fp32, whose matrix
    // instructions take sixteen times as long for a piece, 140 (128), 132 (64)
    const bool wide = p.type == kBf16;
    const struct { Tile tile; int bm, bn, a_cu; double rate; } cuts[] = {{kTile64, 64, 64, 4, wide ? 800e12 : 132e12},
                                                                         {kTile128, 128, 128, 2, wide ? 1060e12 : 140e12},
                                                                         {kTile192, 192, 256, 1, 1200e12},
                                                                         {kTile256, 256, 256, 1, 1250e12}};
    double least = 0.0;
    for (const auto &c : cuts) {
      if (c.tile >= kTile192 && !(q.direct && wide)) continue;
      const long long n = tiles(c.bm, c.bn);
      for (int splits = 1; splits == 1 || (splits <= 64 && splits * 4 <= steps && n * splits <= c.a_cu * kCus && c.tile < kTile192); ++splits) {
        const double us = time_of(p, c.bm, c.bn, c.a_cu, c.rate, n, steps, splits);
        if (least == 0.0 || us < least) least = us, q.tile = c.tile, q.splits = splits, bm = c.bm, bn = c.bn;
      }
    }
  }
  q.tiles_m = (p.m + bm - 1) / bm, q.tiles_n = p.n > 0 ? (p.n + bn - 1) / bn : 1;
  q.steps_each = (steps + q.splits - 1) / q.splits;
  q.splits = (steps + q.steps_each - 1) / q.steps_each;
  return q;
}

template <class T, int FORM, int BM, int BN, int WM, int WN>
void launch(const Product &p, const Plan &q, hipStream_t s) {
  constexpr int WG = 64 * WM * WN;
  in_launches(p, (long long)q.tiles_m * q.tiles_n, WG, [&](const Product &part, unsigned x) {
    const dim3 grid(x, (unsigned)q.splits);
    if (q.direct) k_product<T, FORM, BM, BN, WM, WN, true><<<grid, WG, 0, s>>>(part, q.tiles_m, q.tiles_n, q.steps_each, q.loose);
    else if constexpr (BN < 256) k_product<T, FORM, BM, BN, WM, WN, false><<<grid, WG, 0, s>>>(part, q.tiles_m, q.tiles_n, q.steps_each, false);
  });
}

template <class T, int FORM>
void launch(const Product &p, const Plan &q, hipStream_t s) {
  switch (q.tile) {
    case kFewRows:
      if constexpr (FORM == kProductRows) {
        // with few workgroups more waves each
        if (q.tiles_n >= kCus) in_launches(p, q.tiles_n, 256, [&](const Product &part, unsigned grid) { k_few_rows<T, 4><<<dim3(grid), 256, 0, s>>>(part); });
        else k_few_rows<T, 16><<<dim3((unsigned)q.tiles_n), 1024, 0, s>>>(p);
      }
      return;
    case kTile32: launch<T, FORM, 32, 128, 1, 4>(p, q, s); break;
    case kTile64: launch<T, FORM, 64, 64, 2, 2>(p, q, s); break;
    case kTile128: launch<T, FORM, 128, 128, 2, 2>(p, q, s); break;
    case kTile192:
      if constexpr (sizeof(T) == 2) launch<T, FORM, 192, 256, 2, 4>(p, q, s);
      break;
    case kTile256:
      if constexpr (sizeof(T) == 2) launch<T, FORM, 256, 256, 2, 4>(p, q, s);
      break;
  }
  if (q.splits > 1) {
    const long long blocks = (long long)p.m * ((p.n + 7) / 8), groups = (blocks + 255) / 256;
    k_join<T, FORM><<<dim3((unsigned)(groups < 4 * kCus ? (groups > 0 ? groups : 1) : 4 * kCus)), 256, 0, s>>>(p, q.splits);
  }
}

template <class T>
void launch(const Product &p, const Plan &q, hipStream_t s) {
  switch (p.form) {
    case kProductRows: return launch<T, kProductRows>(p, q, s);
    case kProductMixed: return launch<T, kProductMixed>(p, q, s);
    default: return launch<T, kProductColumns>(p, q, s);
  }
}

}  // namespace

size_t product_scratch(const Product &p) {
  const Plan q = plan_of(p);
  return q.splits < 2 ? 0 : sizeof(float) * (size_t)q.splits * ((size_t)p.m * p.n + (p.sums ? p.m : 0));
}

hipError_t launch_product(const Product &call, hipStream_t s) {
  Product p = call;
  const Plan q = plan_of(p);
  if ((long long)q.tiles_m * q.tiles_n > 0x7fffffffll) return hipErrorInvalidValue;
  if (q.splits < 2) p.partial = nullptr;
  if (p.type == kF32) launch<float>(p, q, s);
  else launch<bf16>(p, q, s);
  return hipGetLastError();
}

}  // namespace qoda
