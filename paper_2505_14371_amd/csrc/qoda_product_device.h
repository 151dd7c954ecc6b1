// What the matrix products' kernels share: operand tiles in shared memory, the matrix instruction, what becomes of a tile's sums, and the join of sums that
// were split along l.
#pragma once

#include <type_traits>

#include "qoda_operators_device.h"

namespace qoda {

namespace {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef short v4s __attribute__((ext_vector_type(4)));

constexpr int kStepBytes = 128;

#define LDS(type, p) (reinterpret_cast<__attribute__((address_space(3))) type *>(p))
typedef __attribute__((address_space(3))) char *lds_ptr;

// The chunk's place in its row of a "rows" tile.  SIDE 1 (b): the 16 rows that a read touches are 8 q + 4 t + r; SIDE 0: 16 adjacent ones.
template <int SIDE>
__device__ __forceinline__ int row_swizzle(int row) {
  return SIDE == 0 ? (row >> 1) & 7 : ((row >> 1) & 1) | ((row >> 2) & 6);
}
// ... and in row l of a "columns" tile of N entries.  bf16: a read touches rows 8 g + r and 32 (SIDE 0) or every other 8 of 64 bytes of each;
// fp32: rows 4 g and 64 bytes, or every other 16 of 128.
template <class T, int SIDE, int N>
__device__ __forceinline__ int column_swizzle(int l) {
  constexpr int kChunks = N * (int)sizeof(T) / 16, kMask = (kChunks & -kChunks) - 1;   // inside the row, whose chunks may be 24
  if constexpr (sizeof(T) == 2) return (SIDE == 0 ? ((l & 3) << 1) | (l & 8) : (l & 3) << 2) & kMask;
  else return (SIDE == 0 ? l & 12 : ((l & 4) << 1) | ((l >> 3) & 1)) & kMask;
}

// A chunk of 16 bytes of which the first `valid` entries (any number) exist; the others come as 0.
template <class T>
__device__ __forceinline__ v4u load_chunk(const T *p, int valid) {
  constexpr int E = 16 / (int)sizeof(T);
  v4u v = {0, 0, 0, 0};
  if (valid >= E) {
    __builtin_memcpy(&v, p, 16);
  } else if (valid > 0) {   // all at once, those beyond the end from the last one's place: a branch for each would wait for each
    u32 e[E];
#pragma unroll
    for (int j = 0; j < E; ++j) {
      const T *q = p + (j < valid ? j : valid - 1);
      if constexpr (sizeof(T) == 4) e[j] = __float_as_uint(*q);
      else e[j] = q->bits;
    }
#pragma unroll
    for (int j = 0; j < E; ++j) e[j] = j < valid ? e[j] : 0u;
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = sizeof(T) == 4 ? e[j] : e[2 * j % E] | e[(2 * j + 1) % E] << 16;
  }
  return v;
}

// One operand's tile: N entries across (rows of c for SIDE 0, columns for SIDE 1) by a step of l, moved by the WG threads.  DIRECT: by
// loads straight into shared memory, 16 bytes a lane, which need addresses of whole words; otherwise by way of registers.
template <class T, bool ROWS, int SIDE, int N, int WG, bool DIRECT>
struct Operand {
  static constexpr int E = 16 / (int)sizeof(T);                 // entries of a chunk
  static constexpr int kStep = kStepBytes / (int)sizeof(T);     // l of a step
  static constexpr int kRowChunks = ROWS ? 8 : N / E;           // chunks of a row in shared memory
  static constexpr int kMine = N * 8 / WG;                      // chunks that a thread moves
  static_assert(N * 8 % WG == 0, "whole chunks a thread");
  static constexpr bool kPower = (N & (N - 1)) == 0;
  static_assert(ROWS || kPower || (N % 64 == 0 && SIDE == 0 && sizeof(T) == 2), "what piece() knows");

  const T *base;     // entry (first, 0)
  long long ld;
  int across, k;     // entries that exist across from the tile's first on, and along l
  u32 offset[DIRECT ? kMine : 1];   // of the chunks that the thread's direct loads move, from the step's first entry, in bytes

  // place `at` in shared memory, in chunks: its row, and which chunk of it lies there
  static __device__ __forceinline__ void place(int at, int &row, int &chunk) {
    row = at / kRowChunks;
    chunk = (at % kRowChunks) ^ (ROWS ? row_swizzle<SIDE>(row) : column_swizzle<T, SIDE, N>(row));
  }
  __device__ __forceinline__ void start(const void *p, long long ld_, int first, int end, int k0, int k_) {
    ld = ld_;
    across = end - first;
    k = k_;
    base = static_cast<const T *>(p) + (ROWS ? (long long)first * ld + k0 : (long long)k0 * ld + first);
    if constexpr (DIRECT)
#pragma unroll
      for (int q = 0; q < kMine; ++q) {
        int row, chunk;
        place(q * WG + (int)threadIdx.x, row, chunk);
        // beyond the edge: what is loaded there is multiplied into sums that are not stored
        if (ROWS) offset[q] = (u32)((row < across ? row : across - 1) * ld * (int)sizeof(T)) + chunk * 16;
        else offset[q] = (u32)(row * ld * (int)sizeof(T)) + (chunk * E < across ? chunk * 16 : 0);
      }
  }
  // A whole step straight into shared memory.  The instruction is written out because the compiler, which cannot tell
  // a step's place from the others', would wait for these loads before every read of shared memory; arrived() waits for them.  (It says that
  // it does not keep m0 across: nothing else here uses it.)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
  __device__ __forceinline__ void direct(int l, lds_ptr to) const {
    const char *p = reinterpret_cast<const char *>(base + (ROWS ? (long long)l : (long long)l * ld));
    const u32 at = __builtin_amdgcn_readfirstlane((u32)(uintptr_t)to + (threadIdx.x & ~63u) * 16);
#pragma unroll
    for (int q = 0; q < kMine; ++q)
      asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(at + q * WG * 16), "v"(offset[q]), "s"(p) : "memory", "m0");
  }
#pragma clang diagnostic pop
  // Any step by way of registers, entries beyond an edge 0.
  __device__ __forceinline__ void fetch(int l, v4u (&v)[kMine]) const {
#pragma unroll
    for (int q = 0; q < kMine; ++q) {
      int row, chunk;
      place(q * WG + (int)threadIdx.x, row, chunk);
      const int a = ROWS ? row : chunk * E, b = l + (ROWS ? chunk * E : row);
      const int valid = ROWS ? (a < across ? k - b : 0) : (b < k ? across - a : 0);
      v[q] = load_chunk<T>(base + (ROWS ? a * ld + b : b * ld + a), valid);
    }
  }
  static __device__ __forceinline__ void store(const v4u (&v)[kMine], lds_ptr to) {
#pragma unroll
    for (int q = 0; q < kMine; ++q) *LDS(v4u, to + (q * WG + threadIdx.x) * 16) = v[q];
  }
  // The lane's piece of 16 entries across (from `first` on; SIDE 1: every other four from first + 4 t on), half s of the step, `first` counting from
  // the wave's own first entry.  Where it lies is the lane's key, which lane_key() makes once, with `first`, t and s in bits that the key has
  // no carry into: an exclusive or with a constant, or a constant offset.
  static __device__ __forceinline__ u32 lane_key(int wave_first) {
    const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
    if constexpr (ROWS) {
      const int a = wave_first + (SIDE == 0 ? i : (i >> 2) * 8 + (i & 3));
      return (u32)(a * 128 + ((g ^ row_swizzle<SIDE>(a)) * 16));
    } else if constexpr (sizeof(T) == 2) {
      // the lane names four adjacent entries of row 8 g + i / 4 (and of the row four further on), and receives one column's four
      const int l = g * 8 + (i >> 2);
      if constexpr (!kPower) return (u32)(l * N * 2 + ((i & 3) >> 1) * 16 + (i & 1) * 8);
      const int chunk = (SIDE == 0 ? (i & 3) >> 1 : i & 3) ^ column_swizzle<T, SIDE, N>(l);
      return (u32)((l * N * 2 + chunk * 16 + (SIDE == 0 ? (i & 1) * 8 : 0)) ^ (wave_first * 2));
    } else {
      const int l = g * 4;
      const int chunk = (SIDE == 0 ? i >> 2 : (i >> 2) * 2) ^ column_swizzle<T, SIDE, N>(l);
      return (u32)((l * N * 4 + chunk * 16 + (i & 3) * 4) ^ (wave_first * 4));
    }
  }
  static __device__ __forceinline__ v4u piece(lds_ptr tile, u32 key, int wave_first, int first, int t, int s) {
    if constexpr (ROWS) {
      return *LDS(v4u, tile + (key ^ (s * 64)) + (first * 128 + t * 512));
    } else if constexpr (sizeof(T) == 2) {
      lds_ptr p = tile + (key ^ (first * 2));
      if constexpr (!kPower) {   // rows are no power of two long: the chunks' permutation, of their lower three bits, apart from the rest
        const u32 chunks = (u32)(wave_first + first) / 8, swizzle = (threadIdx.x & 12) << 3;
        p = tile + (key + (chunks & ~7u) * 16 + (((chunks & 7u) * 16) ^ swizzle));
      }
      v4u v;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const v4s r = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS(v4s, p + ((s * 32 + h * 4) * N * 2 + t * 8)));
        const uint2 w = __builtin_bit_cast(uint2, r);
        v[2 * h] = w.x, v[2 * h + 1] = w.y;
      }
      return v;
    } else {
      const lds_ptr p = tile + (key ^ (first * 4 + t * 16));
      v4u v;
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = *LDS(u32, p + (s * 16 + j) * N * 4);
      return v;
    }
  }
};

// A barrier of the workgroup behind which every wave's reads and writes of shared memory, direct loads among them, are done.
__device__ __forceinline__ void arrived() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0);   // every counter
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// ... behind which all but the last step's direct loads are done where `left` is more than 0 (then there are LOADS of them a wave), and with AHEAD = 0 always all.  Loads arrive in
// their order.  (The branch is written out because the instruction takes a constant.)
template <int LOADS, int AHEAD>
__device__ __forceinline__ void arrived_but(int left) {
  static_assert(AHEAD <= 1, "what is written out");
  if constexpr (AHEAD == 0) return arrived();
  __builtin_amdgcn_sched_barrier(0);
  left = __builtin_amdgcn_readfirstlane(left);
  asm volatile("s_cmp_gt_i32 %0, 0\n\ts_cbranch_scc1 1f\n\ts_waitcnt vmcnt(0)\n1:\n\ts_waitcnt vmcnt(%1) lgkmcnt(0)" ::"s"(left), "n"(LOADS) : "memory", "scc");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

template <class T>
__device__ __forceinline__ v4f multiply(v4u b, v4u a, v4f c) {
  if constexpr (sizeof(T) == 2) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, b), __builtin_bit_cast(v8bf, a), c, 0, 0, 0);
  } else {
    const v4f x = __builtin_bit_cast(v4f, b), y = __builtin_bit_cast(v4f, a);
#pragma unroll
    for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(x[j], y[j], c, 0, 0, 0);
    return c;
  }
}

// The sum of a chunk's entries.
template <class T>
__device__ __forceinline__ float chunk_sum(v4u v) {
  if constexpr (sizeof(T) == 2) {
    float s[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) s[j] = __uint_as_float(v[j] << 16) + __uint_as_float(v[j] & 0xFFFF0000u);
    return (s[0] + s[1]) + (s[2] + s[3]);
  } else {
    const v4f f = __builtin_bit_cast(v4f, v);
    return (f[0] + f[1]) + (f[2] + f[3]);
  }
}

// What the end of a product reads beside the sums, requested ahead of its use.
template <class T, int FORM, int ACT>
struct Beside {
  Eight<T> pre, extra;
  Eight<float> was;
  __device__ __forceinline__ void load(const Product &p, int i, int j, int n) {
    if constexpr (FORM == kProductColumns) {
      if (p.accumulate) was.load(static_cast<const float *>(p.out) + (long long)i * p.ldo + j, n);
    } else {
      if constexpr (FORM == kProductMixed && ACT != kActNone) pre.load(static_cast<const T *>(p.pre) + (long long)i * p.ldp + j, n);
      if (p.extra) extra.load(static_cast<const T *>(p.extra) + (long long)i * p.lde + j, n);
    }
  }
};

// c[i][j .. j + 7] (n of them exist; j a multiple of 8), after the sum over l, to where the call wants them.
template <class T, int FORM, int ACT>
__device__ __forceinline__ void finish(const Product &p, const Beside<T, FORM, ACT> &o, int i, int j, int n, float (&c)[8]) {
  float other[8];
  if constexpr (FORM == kProductColumns) {
    if (p.accumulate) {
      o.was.get(other);
#pragma unroll
      for (int e = 0; e < 8; ++e) c[e] = other[e] + c[e];
    }
    store8(static_cast<float *>(p.out) + (long long)i * p.ldo + j, n, c);
  } else {
    if constexpr (FORM == kProductRows) {
      if (p.bias) {
        load8(p.bias + j, n, other);
#pragma unroll
        for (int e = 0; e < 8; ++e) c[e] = c[e] + other[e];
      }
      if (p.pre) store8(static_cast<T *>(p.pre) + (long long)i * p.ldp + j, n, c);
#pragma unroll
      for (int e = 0; e < 8; ++e) c[e] = act<T, ACT>(c[e]);
    } else if constexpr (ACT != kActNone) {
      o.pre.get(other);
#pragma unroll
      for (int e = 0; e < 8; ++e) c[e] = c[e] * act_slope<T, ACT>(other[e]);
    }
    if (p.drop.threshold) drop8(p.drop, (u32)i, (u32)j >> 3, c);
    if (p.extra) {
      o.extra.get(other);
#pragma unroll
      for (int e = 0; e < 8; ++e) c[e] = other[e] + c[e];
    }
    store8(static_cast<T *>(p.out) + (long long)i * p.ldo + j, n, c);
  }
}

// Calls f with the activation as a constant: the choice is made once for all of a thread's sums.
template <int FORM, class F>
__device__ __forceinline__ void by_activation(int a, F &&f) {
  if constexpr (FORM == kProductColumns) return f(std::integral_constant<int, kActNone>());
  switch (a) {
    case kActRelu: return f(std::integral_constant<int, kActRelu>());
    case kActLeakyRelu: return f(std::integral_constant<int, kActLeakyRelu>());
    case kActGelu: return f(std::integral_constant<int, kActGelu>());
    case kActSilu: return f(std::integral_constant<int, kActSilu>());
    default: return f(std::integral_constant<int, kActNone>());
  }
}

// Workgroups go to the eight XCDs in turn, and each XCD has a cache of its own: an XCD gets a run of tiles that are adjacent in c, column by
// column in bands of kBand rows of tiles, so that what its workgroups load at one time are few rows of a and few of b.
constexpr int kXcds = 8, kBand = 8;
template <class I>
__device__ __forceinline__ I xcd_run(I id, I total) {   // the place in that order of workgroup `id`
  const I x = id % kXcds, q = id / kXcds, each = total / kXcds, more = total % kXcds;
  return x * each + (x < more ? x : more) + q;
}
__device__ __forceinline__ void band_tile(int at, int tiles_m, int tiles_n, int &tm, int &tn) {
  const int band = at / (kBand * tiles_n), in = at - band * kBand * tiles_n;
  const int rows = tiles_m - band * kBand < kBand ? tiles_m - band * kBand : kBand;
  tm = band * kBand + in % rows;
  tn = in / rows;
}
__device__ __forceinline__ void tile_of(int id, int tiles_m, int tiles_n, int &tm, int &tn) { band_tile(xcd_run(id, tiles_m * tiles_n), tiles_m, tiles_n, tm, tn); }

// The splits' sums added up in their order, and finished.
template <class T, int FORM>
__global__ void __launch_bounds__(256) k_join(Product p, int splits) {
  const long long blocks = (p.n + 7) / 8, total = (long long)p.m * blocks, first = (long long)blockIdx.x * 256 + threadIdx.x, stride = (long long)gridDim.x * 256;
  by_activation<FORM>(p.activation, [&](auto a) {
    for (long long q = first; q < total; q += stride) {
      const int i = (int)(q / blocks), j = (int)(q - i * blocks) * 8, n = p.n - j;
      float c[8] = {}, v[8];
      const float *from = p.partial + (long long)i * p.n + j;
      const long long each = (long long)p.m * p.n;
      for (int s = 0; s < splits; s += 4) {   // four on their way
        Eight<float> part[4];
#pragma unroll
        for (int u = 0; u < 4; ++u)
          if (s + u < splits) part[u].load(from + (s + u) * each, n);
#pragma unroll
        for (int u = 0; u < 4; ++u)
          if (s + u < splits) {
            part[u].get(v);
#pragma unroll
            for (int e = 0; e < 8; ++e) c[e] = c[e] + v[e];
          }
      }
      Beside<T, FORM, decltype(a)::value> beside;
      beside.load(p, i, j, n);
      finish(p, beside, i, j, n, c);
    }
  });
  if constexpr (FORM == kProductColumns)
    if (p.sums)
      for (long long i = first; i < p.m; i += stride) {
        float v = 0.0f;
        for (int s = 0; s < splits; ++s) v = v + p.partial[(long long)splits * p.m * p.n + (long long)s * p.m + i];
        p.sums[i] = p.accumulate ? p.sums[i] + v : v;
      }
}

}  // namespace

}  // namespace qoda
