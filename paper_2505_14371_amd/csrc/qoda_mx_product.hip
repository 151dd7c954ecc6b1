// Products between microscaled matrices, of include/qoda_matrices.h: c[i][j] = sum over l of a(i, l) b(j, l), with the epilogues of qoda_linear.hip.
//
// The matrix instruction sums 128 products an entry, in four blocks of 32 with a scale each: a lane's 16 bytes are one block of one row, and the
// scale is a byte of another register.  One dword of scales holds those of a lane's four pieces (64 rows), which is the order they lie in.  A workgroup computes
// BM x BN sums in steps of 256 entries (128 bytes) along l; a step's codes and scales go straight into shared memory, twice, and while one step is
// multiplied the next is on its way, as in qoda_linear.hip.  Rows are filled up to whole steps, so that there are no ragged ones.
//
// Both operands' pieces take every other four of eight rows: a lane then holds eight sums adjacent in a row of c.
//
// Measured: 16384 x 2048 over 8192 135 to 145 us (3.8 to 4.1 PFLOP/s), with dropout and residual 151 to 163; 8192 x 8192 over 2048 through gelu' 142; 6144 x 2048 over 8192
// in fp32 65.  With nothing loaded behind the first steps the first takes 121 us, and without reads of shared memory too 103, its start and end among them.  The
// instruction by itself reaches 5.9 PFLOP/s on random codes (6.9 on zeros: power is the limit), the one of 32 x 32 x 64 6.7 (9.8).  Tiles of 256 take 1.8 us a step of
// 68 KB; tiles of 128, two a CU, are slower there (176) and faster where ends weigh more than steps, which they overlap (2048 entries through gelu': 141 and 157).

#include <utility>

#include "qoda_mx_device.h"
#include "qoda_product_device.h"

namespace qoda {

namespace {

typedef int v8i __attribute__((ext_vector_type(8)));

template <class F, int... I>
__device__ __forceinline__ void each_of(F &&f, std::integer_sequence<int, I...>) { (f(std::integral_constant<int, I>()), ...); }
template <int N, class F>
__device__ __forceinline__ void each(F &&f) { each_of(f, std::make_integer_sequence<int, N>()); }

// FB, FA: the bytes of the scales' registers.
template <int FB, int FA>
__device__ __forceinline__ v4f multiply_blocks(v4u b, v4u a, v4f c, u32 sb, u32 sa) {
  const v8i x = {(int)b[0], (int)b[1], (int)b[2], (int)b[3], 0, 0, 0, 0}, y = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, c, 4, 4, FB, (int)sb, FA, (int)sa);   // 4: codes of four bits
}

// A side's scales, as they lie: 256 bytes for 64 rows and half a step.
template <int N>
struct Scales {
  static constexpr int kHalf = N * 4;      // bytes of half a step
  const u8 *base;
  long long groups;                        // of 64 rows
  int last;                                // of them, from the tile's first on
  __device__ __forceinline__ void start(const u8 *p, long long rows, int row) {
    groups = (rows + 63) / 64, last = (int)groups - 1 - row / 64;
    base = p + (long long)(row / 64) * 256;
  }
  // Half s of a step, by a wave: 16 bytes a lane.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
  __device__ __forceinline__ void direct(long long step, int s, lds_ptr to) const {
    const int lane = threadIdx.x & 63;
    if (lane >= kHalf / 16) return;
    const int group = lane / 16;   // beyond the last rows: scales of sums that are not stored
    const u8 *p = base + (2 * step + s) * groups * 256;
    const u32 offset = (u32)(group < last ? group : last) * 256u + (lane & 15) * 16;
    const u32 at = __builtin_amdgcn_readfirstlane((u32)(uintptr_t)to + s * kHalf);
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(at), "v"(offset), "s"(p) : "memory", "m0");
  }
#pragma clang diagnostic pop
  // The scales of a wave's pieces 4 q .. 4 q + 3, from its row `row` of the tile on; HALF: of the wave's only two pieces, 32 rows.
  template <bool HALF>
  static __device__ __forceinline__ u32 piece(lds_ptr tile, int row, int q, int s) {
    const u32 w = *LDS(u32, tile + s * kHalf + (row / 64 + q) * 256 + (threadIdx.x & 63) * 4);
    return HALF && row & 32 ? w >> 16 : w;
  }
};

// The sum of a row of a, by a wave, in fp32: workgroups behind the tiles' in the same launch, which fill the device while the last tiles are computed.  (A launch
// of their own after it: the weight gradient of 6144 x 2048 over 8192 rows with its rounding 118 us for 109, small ones 17.4 for 14.4.)
__device__ __forceinline__ void sum_row(const MxProduct &m, long long r) {
  if (r >= m.p.m) return;
  const int lane = threadIdx.x & 63;
  const long long groups = ((long long)m.p.m + 63) / 64;
  float sum = 0.0f;
  for (int block = lane; block < m.steps * 8; block += 64) {
    v4u codes;
    __builtin_memcpy(&codes, m.a + (r * m.steps * 8 + block) * 16, 16);
    const u32 byte = m.a_scales[((block >> 2) * groups + (r >> 6)) * 256 + scale_place((int)(r & 63), block & 3)];
    float part = 0.0f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {   // exact: multiples of half a scale
      float v[8];
      values_of(codes[e], byte, v);
#pragma unroll
      for (int j = 0; j < 8; ++j) part = part + v[j];
    }
    sum = sum + part;
  }
#pragma unroll
  for (int d = 1; d < 64; d *= 2) sum = sum + __shfl_xor(sum, d);
  if (lane == 0) m.row_sums[r] = m.p.accumulate ? m.row_sums[r] + sum : sum;
}

template <class T, int FORM, int BM, int BN, int WM, int WN>
__global__ void __launch_bounds__(64 * WM * WN, 2) k_mx_product(MxProduct m, int tiles_m, int tiles_n, int steps_each) {
  constexpr int WG = 64 * WM * WN, FM = BM / WM / 16, FN = BN / WN / 16, QM = (FM + 3) / 4, QN = (FN + 3) / 4;
  static_assert(FM % 2 == 0 && FN % 2 == 0 && (FM == 2 || FM % 4 == 0) && (FN == 2 || FN % 4 == 0) && WG >= 256, "what the scales' order knows");
  typedef Operand<bf16, true, 1, BM, WG, true> A;   // in words of 16 bits: four codes
  typedef Operand<bf16, true, 1, BN, WG, true> B;
  typedef Scales<BM> SA;
  typedef Scales<BN> SB;
  constexpr u32 kBuffer = (BM + BN) * (kStepBytes + 8);   // both sides' codes and scales of a step
  __shared__ __align__(16) char shared[2 * kBuffer];

  const Product &p = m.p;
  if constexpr (FORM == kProductColumns) {
    const long long behind = m.first + blockIdx.x - (long long)tiles_m * tiles_n;
    if (behind >= 0) return sum_row(m, (behind * gridDim.y + blockIdx.y) * (WG / 64) + threadIdx.x / 64);
  }
  int tm, tn;
  tile_of((int)(m.first + blockIdx.x), tiles_m, tiles_n, tm, tn);
  const int i0 = __builtin_amdgcn_readfirstlane(tm) * BM, j0 = __builtin_amdgcn_readfirstlane(tn) * BN;
  const int step0 = (int)blockIdx.y * steps_each, steps = m.steps - step0 < steps_each ? m.steps - step0 : steps_each;
  A a;
  B b;
  a.start(m.a, (long long)m.steps * 64, i0, p.m, step0 * 64, steps * 64);
  b.start(m.b, (long long)m.steps * 64, j0, p.n, step0 * 64, steps * 64);
  SA sa;
  SB sb;
  sa.start(m.a_scales, p.m, i0);
  sb.start(m.b_scales, p.n, j0);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), wm = wave / WN * (BM / WM), wn = wave % WN * (BN / WN);

  v4f c[FM][FN];
#pragma unroll
  for (int x = 0; x < FM; ++x)
#pragma unroll
    for (int y = 0; y < FN; ++y) c[x][y] = v4f{0, 0, 0, 0};

  struct Pieces {
    v4u a[FM], b[FN];
    u32 sa[QM], sb[QN];
  };
  const lds_ptr base = (lds_ptr)shared;
  u32 now = 0;   // the buffer of the step that is multiplied
  u32 key_a = A::lane_key(wm), key_b = B::lane_key(wn);
  const auto read = [&](Pieces &f, u32 from, int s) {
    asm volatile("" : "+v"(key_a), "+v"(key_b));   // made anew each time, as in k_product
    const lds_ptr ta = base + from, tb = ta + BM * kStepBytes, ts = tb + BN * kStepBytes;
#pragma unroll
    for (int q = 0; q < QN; ++q) f.sb[q] = SB::template piece<FN == 2>(ts + BM * 8, wn, q, s);
#pragma unroll
    for (int q = 0; q < QM; ++q) f.sa[q] = SA::template piece<FM == 2>(ts, wm, q, s);
#pragma unroll
    for (int y = 0; y < FN; ++y) f.b[y] = B::piece(tb, key_b, wn, y / 2 * 32, y & 1, s);
#pragma unroll
    for (int x = 0; x < FM; ++x) f.a[x] = A::piece(ta, key_a, wm, x / 2 * 32, x & 1, s);
  };
  const auto multiply_all = [&](const Pieces &f) {
    each<FM>([&](auto x) {
      each<FN>([&](auto y) { c[x][y] = multiply_blocks<y % 4, x % 4>(f.b[y], f.a[x], c[x][y], f.sb[y / 4], f.sa[x / 4]); });
    });
  };
  const auto here = [&] {   // the sums so far are wanted here: otherwise the compiler takes their instructions behind the barrier and the branch after it
#pragma unroll
    for (int x = 0; x < FM; ++x)
#pragma unroll
      for (int y = 0; y < FN; ++y) asm volatile("" : "+v"(c[x][y]));
  };
  const auto request = [&](int t, u32 to) {
    const lds_ptr ta = base + to, tb = ta + BM * kStepBytes, ts = tb + BN * kStepBytes;
    a.direct(t * 64, ta);
    b.direct(t * 64, tb);
    if (wave < 2) sa.direct(step0 + t, wave, ts);
    else if (wave < 4) sb.direct(step0 + t, wave - 2, ts + BM * 8);
  };
  // One block without branches around what is read and multiplied: behind the last step the next one's pieces are read all the same, from what the buffer
  // holds, and not used.  (With branches the compiler kept copies of the sums.)
  if (steps > 0) {
    request(0, 0);
    if (steps > 1) request(1, kBuffer);
    Pieces f0, f1;
    arrived();
    read(f0, 0, 0);
    for (int t = 0; t < steps; ++t) {
      read(f1, now, 1);
      multiply_all(f0);
      here();
      arrived();   // the next step is there, and nobody reads this one any more
      if (t + 2 < steps) request(t + 2, now);
      now = kBuffer - now;
      read(f0, now, 0);
      multiply_all(f1);
      __builtin_amdgcn_sched_barrier(0);
    }
  }

  const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
  const auto row = [&](int x) { return i0 + wm + x / 2 * 32 + (i >> 2) * 8 + (x & 1) * 4 + (i & 3); };
  const auto column = [&](int y) { return j0 + wn + y * 32 + g * 8; };
  const auto sums = [&](int x, int y, float (&v)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = c[x][2 * y + e / 4][e & 3];
  };
  if (p.partial) {
#pragma unroll
    for (int x = 0; x < FM; ++x)
#pragma unroll
      for (int y = 0; y < FN / 2; ++y)
        if (row(x) < p.m && column(y) < p.n) {
          float v[8];
          sums(x, y, v);
          store8(p.partial + ((long long)blockIdx.y * p.m + row(x)) * p.n + column(y), p.n - column(y), v);
        }
    return;
  }
  by_activation<FORM>(p.activation, [&](auto act) {
    constexpr int kPart = FM < 4 || sizeof(T) == 4 ? 2 : 4;   // rows whose reads are all on their way before the first is needed
#pragma unroll
    for (int x0 = 0; x0 < FM; x0 += kPart) {
      Beside<T, FORM, decltype(act)::value> beside[kPart][FN / 2];
#pragma unroll
      for (int x = 0; x < kPart; ++x)
#pragma unroll
        for (int y = 0; y < FN / 2; ++y)
          if (row(x0 + x) < p.m && column(y) < p.n) beside[x][y].load(p, row(x0 + x), column(y), p.n - column(y));
#pragma unroll
      for (int x = 0; x < kPart; ++x)
#pragma unroll
        for (int y = 0; y < FN / 2; ++y)
          if (row(x0 + x) < p.m && column(y) < p.n) {
            float v[8];
            sums(x0 + x, y, v);
            finish(p, beside[x][y], row(x0 + x), column(y), p.n - column(y), v);
          }
    }
  });
}

// Up to 16 rows of x, plain ones rounded here: b is read once, and that is the time.  A workgroup takes 32 rows of b, its NW waves the half steps in turn; a
// lane's block of x is 32 adjacent entries, so that its scale needs no other lane.
template <class T, int FORM, int NW, bool PLAIN>
__global__ void __launch_bounds__(64 * NW) k_mx_few_rows(MxProduct m) {
  constexpr int kAhead = 2;
  __shared__ v4f part[NW][2][64];
  const Product &p = m.p;
  const int lane = threadIdx.x & 63, wave = threadIdx.x / 64, i = lane & 15, g = lane >> 4;
  const int j0 = (int)(m.first + blockIdx.x) * 32;
  const long long groups = ((long long)p.n + 63) / 64, row_bytes = (long long)m.steps * 128;
  const u8 *b[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int j = j0 + (i >> 2) * 8 + h * 4 + (i & 3);
    b[h] = m.b + (long long)(j < p.n ? j : p.n - 1) * row_bytes + g * 16;
  }
  const u8 *sb = m.b_scales + (long long)(j0 / 64) * 256 + lane * 4 + (j0 & 32 ? 2 : 0);
  const u8 *a = PLAIN ? nullptr : m.a + (long long)(i < p.m ? i : 0) * row_bytes + g * 16;
  const u8 *sa = PLAIN ? nullptr : m.a_scales + scale_place(i, g);   // up to 16 rows: one group
  const T *x = static_cast<const T *>(m.x) + (long long)(i < p.m ? i : 0) * m.ldx;
  v4f c[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
  const int halves = 2 * m.steps;
  for (int t0 = wave; t0 < halves; t0 += NW * kAhead) {
    v4u fb[kAhead][2], fa[kAhead];
    u32 qb[kAhead], qa[kAhead];
    Eight<T> e[PLAIN ? kAhead : 1][4];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int t = t0 + u * NW;
      if (t < halves) {
#pragma unroll
        for (int h = 0; h < 2; ++h) __builtin_memcpy(&fb[u][h], b[h] + (long long)t * 64, 16);
        unsigned short w;
        __builtin_memcpy(&w, sb + (long long)t * groups * 256, 2);
        qb[u] = w;
        if constexpr (PLAIN) {
          const long long l = (long long)t * 128 + g * 32;
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const long long left = p.k - l - 8 * k;
            e[u][k].load(x + l + 8 * k, i < p.m ? (left < 8 ? (int)left : 8) : 0);
          }
        } else {
          __builtin_memcpy(&fa[u], a + (long long)t * 64, 16);
          qa[u] = sa[(long long)t * 256];
        }
      }
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      if (t0 + u * NW >= halves) break;
      if constexpr (PLAIN) {
        u32 most = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const u32 one = most_of(e[u][k]);
          most = most > one ? most : one;
        }
        qa[u] = scale_byte(most, false);
#pragma unroll
        for (int k = 0; k < 4; ++k) fa[u][k] = qa[u] == 255u ? 0u : codes_nearest(e[u][k], scale_of(qa[u]));
      } else if (i >= p.m) {
        fa[u] = v4u{0, 0, 0, 0};
      }
      c[0] = multiply_blocks<0, 0>(fb[u][0], fa[u], c[0], qb[u], qa[u]);
      c[1] = multiply_blocks<1, 0>(fb[u][1], fa[u], c[1], qb[u], qa[u]);
    }
  }
  part[wave][0][lane] = c[0];
  part[wave][1][lane] = c[1];
  __syncthreads();
  // the sum of row i and column 8 g + 4 h + r of the 32 lies in lane 16 g + i of half h, place r
  const int row = (int)threadIdx.x / 4, q = threadIdx.x & 3, j = j0 + q * 8;
  if (row < p.m && row < 16 && j < p.n) {
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      v[e] = part[0][e / 4][q * 16 + row][e & 3];
#pragma unroll
      for (int w = 1; w < NW; ++w) v[e] = v[e] + part[w][e / 4][q * 16 + row][e & 3];
    }
    by_activation<FORM>(p.activation, [&](auto act) {
      Beside<T, FORM, decltype(act)::value> beside;
      beside.load(p, row, j, p.n - j);
      finish(p, beside, row, j, p.n - j, v);
    });
  }
}

enum Tile { kFewRows, kTile64, kTile128, kTile256 };
struct Plan {
  Tile tile;
  int tiles_m, tiles_n, splits, steps_each;
};

constexpr int kCus = 256;

// What a cut would take, in us, from what was measured: the matrix cores' rate in whole tiles of a size, the time of a step in a workgroup that is alone on its CU, what a
// tile's end reads and writes at the rate of memory (half of it is hidden where a CU holds several workgroups), and the join of splits.  Measured and
// estimated: 16384 x 2048 over 8192 with dropout and residual by 256 168 and 175, by 128 185 and 199; 8192 x 8192 over 2048 through gelu' by 256 157 and 142, by
// 128 142 and 132; 64 x 64 over 16384 in 8 parts 9.5 and 15.
struct Kind {
  Tile tile;
  int side, a_cu;
  double rate, least;
};
constexpr Kind kKinds[] = {{kTile64, 64, 4, 2000e12, 0.45}, {kTile128, 128, 2, 3100e12, 0.6}, {kTile256, 256, 1, 3800e12, 1.3}};

double time_of(const Product &p, const Kind &kind, long long tiles, int steps, int splits) {
  const int steps_each = (steps + splits - 1) / splits;
  const double one = 2.0 * kind.side * kind.side * kMxStep / (kind.rate / kCus) * 1e6;
  long long left = tiles * splits;
  double us = 0.0;
  while (left > 0) {
    const long long now = left < (long long)kind.a_cu * kCus ? left : (long long)kind.a_cu * kCus, rounds = left / now;
    const double step = (double)((now + kCus - 1) / kCus) * one;
    us += (double)rounds * (2.0 + steps_each * (step > kind.least ? step : kind.least));
    left -= rounds * now;
  }
  const double entry = p.form == kProductColumns || p.type == kF32 ? 4.0 : 2.0, moved = 1.0 + (p.pre ? 1.0 : 0.0) + (p.extra || p.accumulate ? 1.0 : 0.0);
  const double end = (double)p.m * p.n * entry * moved / 5e6;
  if (splits > 1) return us + 5.0 + 0.4 * splits + (double)splits * p.m * p.n * 8.0 / 4e6 + end;
  return us + (kind.a_cu == 1 ? end : 0.5 * end);
}

bool few_rows(const Product &p) { return p.form != kProductColumns && p.m <= 16; }

Plan plan_of(const MxProduct &m) {
  const Product &p = m.p;
  Plan q = {};
  q.splits = 1;
  if (p.m == 0 || p.n == 0) {   // sums of rows at most
    q.tile = kTile64;
    return q;
  }
  if (few_rows(p)) {
    q.tile = kFewRows, q.tiles_m = 1, q.tiles_n = (p.n + 31) / 32;
    return q;
  }
  const int steps = m.steps > 0 ? m.steps : 1;
  double least = 0.0;
  int side = 0;
  for (const Kind &c : kKinds) {
    const long long n = ((p.m + c.side - 1ll) / c.side) * ((p.n + c.side - 1ll) / c.side);
    for (int splits = 1; splits == 1 || (splits <= 64 && splits * 2 <= steps && n * splits <= c.a_cu * kCus); ++splits) {
      const double us = time_of(p, c, n, steps, splits);
      if (least == 0.0 || us < least) least = us, q.tile = c.tile, q.splits = splits, side = c.side;
    }
  }
  q.tiles_m = (int)((p.m + side - 1ll) / side), q.tiles_n = (int)((p.n + side - 1ll) / side);
  q.steps_each = (steps + q.splits - 1) / q.splits;
  q.splits = (steps + q.steps_each - 1) / q.steps_each;
  return q;
}

template <class T, int FORM, int BM, int BN, int WM, int WN>
void launch_tiles(const MxProduct &m, const Plan &q, hipStream_t s) {
  constexpr int WG = 64 * WM * WN;
  const long long sums = m.row_sums ? (m.p.m + WG / 64 - 1) / (WG / 64) : 0;   // workgroups that sum rows, spread over the splits
  in_launches(m, (long long)q.tiles_m * q.tiles_n + (sums + q.splits - 1) / q.splits, WG, [&](const MxProduct &part, unsigned x) {
    k_mx_product<T, FORM, BM, BN, WM, WN><<<dim3(x, (unsigned)q.splits), WG, 0, s>>>(part, q.tiles_m, q.tiles_n, q.steps_each);
  });
}

template <class T, int FORM>
void launch(const MxProduct &m, const Plan &q, hipStream_t s) {
  switch (q.tile) {
    case kFewRows:
      if constexpr (FORM != kProductColumns) {
        // with few workgroups more waves each
        const bool many = q.tiles_n >= 4 * kCus;
        const auto go = [&](auto plain) {
          constexpr bool kPlain = decltype(plain)::value;
          if (many) in_launches(m, q.tiles_n, 256, [&](const MxProduct &part, unsigned grid) { k_mx_few_rows<T, FORM, 4, kPlain><<<dim3(grid), 256, 0, s>>>(part); });
          else k_mx_few_rows<T, FORM, 16, kPlain><<<dim3((unsigned)q.tiles_n), 1024, 0, s>>>(m);
        };
        if (m.a) go(std::false_type());
        else go(std::true_type());
      }
      return;
    case kTile64: launch_tiles<T, FORM, 64, 64, 2, 2>(m, q, s); break;
    case kTile128: launch_tiles<T, FORM, 128, 128, 2, 2>(m, q, s); break;
    case kTile256: launch_tiles<T, FORM, 256, 256, 2, 4>(m, q, s); break;
  }
  if (q.splits > 1) {
    const long long blocks = (long long)m.p.m * ((m.p.n + 7) / 8), groups = (blocks + 255) / 256;
    k_join<T, FORM><<<dim3((unsigned)(groups < 4 * kCus ? groups : 4 * kCus)), 256, 0, s>>>(m.p, q.splits);
  }
}

template <class T>
void launch(const MxProduct &m, const Plan &q, hipStream_t s) {
  if (m.p.form == kProductRows) launch<T, kProductRows>(m, q, s);
  else launch<T, kProductMixed>(m, q, s);
}

}  // namespace

// Every workgroup of k_mx_few_rows rounds all of x: 0.3 ns for each 32 rows of b and half step.  Where that is more than a launch's 3.5 us, x is rounded before: one
// row, 8192 -> 50304, 71 us inside and 45 before; 2048 -> 8192 5.3 and 8.8.
bool mx_takes_plain_rows(const Product &p) { return few_rows(p) && ((p.n + 31ll) / 32) * ((p.k + 127ll) / 128) <= 12000; }

size_t mx_product_scratch(const MxProduct &m) {
  const Plan q = plan_of(m);
  return q.splits < 2 ? 0 : sizeof(float) * (size_t)q.splits * (size_t)m.p.m * m.p.n;
}

hipError_t launch_mx_product(const MxProduct &call, hipStream_t s) {
  MxProduct m = call;
  const Plan q = plan_of(m);
  if ((long long)q.tiles_m * q.tiles_n > 0x7fffffffll) return hipErrorInvalidValue;
  if (q.splits < 2) m.p.partial = nullptr;
  if (m.p.form == kProductColumns) launch<float, kProductColumns>(m, q, s);
  else if (m.p.type == kF32) launch<float>(m, q, s);
  else launch<bf16>(m, q, s);
  return hipGetLastError();
}

}  // namespace qoda
