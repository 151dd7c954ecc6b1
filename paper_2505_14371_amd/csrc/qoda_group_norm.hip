// Group normalisation with an activation, channels last, and its gradient (include/qoda_operators.h).
//
// Every value is read once where a group's values fit the registers of a workgroup: the mean, the squares about it and the result all
// come from there, so that the variance is no difference of large sums.  Two shapes of work:
//   rows   one position: a group is one run of adjacent channels.  A team of lanes takes a row, eight entries a lane at a time.
//   maps   several positions: a workgroup takes a block of channels that holds whole groups (or a part of one large group) at some or
//          all positions; a thread owns eight channels at every so many positions.  Sums run per channel first, because that is what the
//          gradients of weight and bias are, and a group's are sums of its channels'.  Where a block has more values than a workgroup holds, its
//          positions are split: one launch for the pieces' sums and one for the result, where there are many pieces with one between them that joins
//          their sums.
//
// Measured: rows of 2048, 16384 of them, bf16: forward 24 us (5.6 TB/s), gradient with residual 61 + 7 for the join (4.4 TB/s); a map of 64 x 256 x
// 256 in fp32 12.5 us, the gradient of 128 x 1024 x 128 in bf16 with silu 52 (without an activation 41).  In pieces: 8 x 65536 x 128 of bf16 in 32 groups 79 us,
// its gradient 147.  Small ones are bound by the launch and by the sums over the workgroup.

#include <type_traits>

#include "qoda_operators_device.h"

namespace qoda {

namespace {

constexpr int kThreads = 256;

// Sums over teams of 16 or 64 adjacent lanes, the same in every lane.
template <int TEAM>
__device__ __forceinline__ float lanes_sum(float v) {
  const auto move = [](float x, auto ctrl) {
    return __uint_as_float((u32)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), decltype(ctrl)::value, 0xF, 0xF, true));
  };
  v = v + move(v, std::integral_constant<int, 0xB1>());    // lane ^ 1
  v = v + move(v, std::integral_constant<int, 0x4E>());    // lane ^ 2
  v = v + move(v, std::integral_constant<int, 0x141>());   // the other four of eight
  v = v + move(v, std::integral_constant<int, 0x140>());   // the other eight of sixteen
  if constexpr (TEAM == 64) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(b[0]) + __uint_as_float(b[1]);
  }
  return v;
}
// ... of a team that may be the whole workgroup.  red: a float for each wave, free again after the next barrier.
template <int TEAM>
__device__ __forceinline__ float team_sum(float v, float *red) {
  if constexpr (TEAM <= 64) {
    return lanes_sum<TEAM>(v);
  } else {
    v = lanes_sum<64>(v);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x / 64] = v;
    __syncthreads();
    float s = 0.0f;
#pragma unroll
    for (int w = 0; w < TEAM / 64; ++w) s = s + red[w];
    return s;
  }
}

// Two at once, with one barrier.  red: two floats for each wave.
template <int TEAM>
__device__ __forceinline__ void team_sums(float &a, float &b, float2 *red) {
  if constexpr (TEAM <= 64) {
    a = lanes_sum<TEAM>(a), b = lanes_sum<TEAM>(b);
  } else {
    a = lanes_sum<64>(a), b = lanes_sum<64>(b);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x / 64] = {a, b};
    __syncthreads();
    a = b = 0.0f;
#pragma unroll
    for (int w = 0; w < TEAM / 64; ++w) a = a + red[w].x, b = b + red[w].y;
  }
}

template <bool EVEN = false>
__device__ __forceinline__ void vector8(const float *p, float otherwise, int n, float (&v)[8]) {
  if (p) {
    load8<EVEN>(p, n, v);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = otherwise;
  }
}

template <class T>
__device__ __forceinline__ void act8(int a, float (&v)[8]) {
  const auto all = [&](auto c) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = act<T, decltype(c)::value>(v[j]);
  };
  switch (a) {
    case kActRelu: return all(std::integral_constant<int, kActRelu>());
    case kActLeakyRelu: return all(std::integral_constant<int, kActLeakyRelu>());
    case kActGelu: return all(std::integral_constant<int, kActGelu>());
    case kActSilu: return all(std::integral_constant<int, kActSilu>());
    default: return;
  }
}
// v times the slope at z
template <class T>
__device__ __forceinline__ void slope8(int a, const float (&z)[8], float (&v)[8]) {
  const auto all = [&](auto c) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = v[j] * act_slope<T, decltype(c)::value>(z[j]);
  };
  switch (a) {
    case kActRelu: return all(std::integral_constant<int, kActRelu>());
    case kActLeakyRelu: return all(std::integral_constant<int, kActLeakyRelu>());
    case kActGelu: return all(std::integral_constant<int, kActGelu>());
    case kActSilu: return all(std::integral_constant<int, kActSilu>());
    default: return;
  }
}

// Eight normalised values times weight plus bias, through the activation.
template <class T, bool EVEN = false>
__device__ __forceinline__ void normalised8(const GroupNorm &g, long long c, int n, float mean, float rstd, float (&v)[8]) {
  float w[8], b[8];
  vector8<EVEN>(g.weight ? g.weight + c : nullptr, 1.0f, n, w);
  vector8<EVEN>(g.bias ? g.bias + c : nullptr, 0.0f, n, b);
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = __builtin_fmaf((v[j] - mean) * rstd, w[j], b[j]);
  act8<T>(g.activation, v);
}

// h: the normalised values of x; d: dy through the activation; w: the weights.
template <class T, bool EVEN = false>
__device__ __forceinline__ void back8(const GroupNorm &g, long long c, int n, float mean, float rstd, float (&h)[8], float (&d)[8], float (&w)[8]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) h[j] = (h[j] - mean) * rstd;
  vector8<EVEN>(g.weight ? g.weight + c : nullptr, 1.0f, n, w);
  if (g.activation != kActNone) {
    float z[8];
    vector8<EVEN>(g.bias ? g.bias + c : nullptr, 0.0f, n, z);
#pragma unroll
    for (int j = 0; j < 8; ++j) z[j] = __builtin_fmaf(h[j], w[j], z[j]);
    slope8<T>(g.activation, z, d);
  }
}

// ------------------------------------------------------------------------------------------------ rows
// Row r is group r % groups of sample r / groups: `len` channels.
struct Row {
  long long n, c0;   // sample, first channel
  __device__ __forceinline__ Row(const GroupNorm &g, long long r, long long len) {
    if (g.groups == 1) n = r, c0 = 0;
    else n = r / g.groups, c0 = (r - n * g.groups) * len;
  }
};

// A team a row, V times eight entries a lane.
template <class T, int TEAM, int V, bool EVEN>
__global__ void __launch_bounds__(kThreads) k_norm_rows(GroupNorm g) {
  __shared__ float red[2][kThreads / 64];
  const int lane = threadIdx.x % TEAM;
  const int len = (int)(g.channels / g.groups);
  const long long rows = g.samples * g.groups;
  long long r = (g.first + blockIdx.x) * (kThreads / TEAM) + threadIdx.x / TEAM;
  const bool real = r < rows;
  if (!real) r = rows - 1;   // a team without a row goes along with the last one's, and stores nothing
  const Row row(g, r, len);
  const T *x = static_cast<const T *>(g.x) + row.n * g.x_sample + row.c0;
  Eight<T> raw[V];
#pragma unroll
  for (int v = 0; v < V; ++v) raw[v].template load<EVEN>(x + (lane + v * TEAM) * 8, len - (lane + v * TEAM) * 8);
  float s = 0.0f;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    float e[8];
    raw[v].get(e);   // 0 beyond the row
    s = s + (((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7])));
  }
  const float mean = team_sum<TEAM>(s, red[0]) / (float)len;
  s = 0.0f;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    float e[8];
    raw[v].get(e);
    const int n = len - (lane + v * TEAM) * 8;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float d = (EVEN ? n > 0 : j < n) ? e[j] - mean : 0.0f;
      s = __builtin_fmaf(d, d, s);
    }
  }
  const float rstd = 1.0f / sqrtf(team_sum<TEAM>(s, red[1]) / (float)len + g.eps);
  if (!real) return;
  if (lane == 0) g.mean[r] = mean, g.rstd[r] = rstd;
  T *y = static_cast<T *>(g.out) + row.n * g.out_sample + row.c0;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int at = (lane + v * TEAM) * 8, n = len - at;
    if (n > 0) {
      float e[8];
      raw[v].get(e);
      normalised8<T, EVEN>(g, row.c0 + at, n, mean, rstd, e);
      store8<EVEN>(y + at, n, e);
    }
  }
}

// Rows longer than the registers hold: a workgroup a row, read three times.
template <class T>
__global__ void __launch_bounds__(1024) k_norm_long_rows(GroupNorm g) {
  __shared__ float red[2][16];
  const long long r = g.first + blockIdx.x, len = g.channels / g.groups;
  const Row row(g, r, len);
  const T *x = static_cast<const T *>(g.x) + row.n * g.x_sample + row.c0;
  T *y = static_cast<T *>(g.out) + row.n * g.out_sample + row.c0;
  const auto clip = [](long long n) { return n < 8 ? (int)n : 8; };
  float s = 0.0f, e[8];
  for (long long at = threadIdx.x * 8; at < len; at += 8192) {
    load8(x + at, clip(len - at), e);
    s = s + (((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7])));
  }
  const float mean = team_sum<1024>(s, red[0]) / (float)len;
  s = 0.0f;
  for (long long at = threadIdx.x * 8; at < len; at += 8192) {
    const int n = clip(len - at);
    load8(x + at, n, e);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float d = j < n ? e[j] - mean : 0.0f;
      s = __builtin_fmaf(d, d, s);
    }
  }
  const float rstd = 1.0f / sqrtf(team_sum<1024>(s, red[1]) / (float)len + g.eps);
  if (threadIdx.x == 0) g.mean[r] = mean, g.rstd[r] = rstd;
  for (long long at = threadIdx.x * 8; at < len; at += 8192) {
    const int n = clip(len - at);
    load8(x + at, n, e);
    normalised8<T>(g, row.c0 + at, n, mean, rstd, e);
    store8(y + at, n, e);
  }
}

// The gradient of rows.  A team takes rows of one group, `step` samples apart, and keeps its channels' sums for dweight and dbias in
// registers; the workgroup's teams join theirs in shared memory and store one row of partial sums.  grid: (groups, workgroups a group).
template <class T, int TEAM, int V, bool EVEN>
__global__ void __launch_bounds__(kThreads) k_norm_rows_grad(GroupNorm g) {
  constexpr int kTeams = kThreads / TEAM;
  __shared__ float2 red[2][kThreads / 64];
  __shared__ float join[kTeams > 1 ? TEAM * V * 8 : 1];
  const int lane = threadIdx.x % TEAM, team = threadIdx.x / TEAM;
  const int len = (int)(g.channels / g.groups);
  const long long gr = g.first + blockIdx.x, c0 = gr * len;
  float sw[V][8] = {}, sb[V][8] = {};
  const float inv = 1.0f / (float)len;
  int turn = 0;
  for (long long first = (long long)blockIdx.y * kTeams; first < g.samples; first += (long long)gridDim.y * kTeams, turn ^= 1) {
    const long long n = first + team < g.samples ? first + team : g.samples - 1;
    const bool real = first + team < g.samples;
    const T *x = static_cast<const T *>(g.x) + n * g.x_sample + c0, *dy = static_cast<const T *>(g.dy) + n * g.dy_sample + c0;
    Eight<T> rx[V], rd[V], re[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int at = (lane + v * TEAM) * 8;
      rx[v].template load<EVEN>(x + at, len - at);
      rd[v].template load<EVEN>(dy + at, len - at);
      if (g.extra) re[v].template load<EVEN>(static_cast<const T *>(g.extra) + n * g.extra_sample + c0 + at, len - at);
    }
    const float mean = g.mean[n * g.groups + gr], rstd = g.rstd[n * g.groups + gr];
    float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int at = (lane + v * TEAM) * 8;
      if (at < len) {
        float h[8], d[8], w[8];
        rx[v].get(h);
        rd[v].get(d);   // 0 beyond the row
        back8<T, EVEN>(g, c0 + at, len - at, mean, rstd, h, d, w);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          if (!EVEN && len - at <= j) d[j] = 0.0f, h[j] = 0.0f;
          if (real) sw[v][j] = __builtin_fmaf(d[j], h[j], sw[v][j]), sb[v][j] = sb[v][j] + d[j];
          const float u = d[j] * w[j];
          s1 = s1 + u;
          s2 = __builtin_fmaf(u, h[j], s2);
        }
      }
    }
    team_sums<TEAM>(s1, s2, red[turn]);   // by turns: the readers of one place are done before the next barrier but one
    const float m1 = s1 * inv, m2 = s2 * inv;
    if (real) {
      T *dx = static_cast<T *>(g.out) + n * g.out_sample + c0;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const int at = (lane + v * TEAM) * 8;
        if (at < len) {
          float h[8], d[8], w[8], o[8];
          rx[v].get(h);
          rd[v].get(d);
          back8<T, EVEN>(g, c0 + at, len - at, mean, rstd, h, d, w);
          if (g.extra) re[v].get(o);
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float q = __builtin_fmaf(-h[j], m2, __builtin_fmaf(d[j], w[j], -m1)) * rstd;
            d[j] = g.extra ? o[j] + q : q;
          }
          store8<EVEN>(dx + at, len - at, d);
        }
      }
    }
  }
  if (!g.scratch) return;
  // partial sums of this workgroup: [2][channels]
  float *part = g.scratch + (long long)blockIdx.y * 2 * g.channels + c0;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    if constexpr (kTeams > 1) {
      for (int t = 0; t < kTeams; ++t) {   // the teams in their order
        __syncthreads();
        if (team == t)
#pragma unroll
          for (int v = 0; v < V; ++v)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              float *o = &join[(v * 8 + j) * TEAM + lane];
              const float mine = k == 0 ? sw[v][j] : sb[v][j];
              *o = t == 0 ? mine : *o + mine;
            }
      }
      if (team == kTeams - 1)   // this team's own writes
#pragma unroll
        for (int v = 0; v < V; ++v) {
          const int at = (lane + v * TEAM) * 8;
          float e[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) e[j] = join[(v * 8 + j) * TEAM + lane];
          if (at < len) store8<EVEN>(part + k * g.channels + at, len - at, e);
        }
    } else {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const int at = (lane + v * TEAM) * 8;
        if (at < len) store8<EVEN>(part + k * g.channels + at, len - at, k == 0 ? sw[v] : sb[v]);
      }
    }
  }
}

// Rows longer than the registers hold: a workgroup a row.  dweight and dbias come from k_norm_long_channels.
template <class T>
__global__ void __launch_bounds__(1024) k_norm_long_rows_grad(GroupNorm g) {
  __shared__ float red[2][16];
  const long long r = g.first + blockIdx.x, len = g.channels / g.groups;
  const Row row(g, r, len);
  const float mean = g.mean[r], rstd = g.rstd[r];
  const T *x = static_cast<const T *>(g.x) + row.n * g.x_sample + row.c0, *dy = static_cast<const T *>(g.dy) + row.n * g.dy_sample + row.c0;
  const auto clip = [](long long n) { return n < 8 ? (int)n : 8; };
  float s1 = 0.0f, s2 = 0.0f, h[8], d[8], w[8];
  for (long long at = threadIdx.x * 8; at < len; at += 8192) {
    const int n = clip(len - at);
    load8(x + at, n, h);
    load8(dy + at, n, d);
    back8<T>(g, row.c0 + at, n, mean, rstd, h, d, w);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float u = j < n ? d[j] * w[j] : 0.0f;
      s1 = s1 + u;
      s2 = j < n ? __builtin_fmaf(u, h[j], s2) : s2;
    }
  }
  const float m1 = team_sum<1024>(s1, red[0]) / (float)len, m2 = team_sum<1024>(s2, red[1]) / (float)len;
  for (long long at = threadIdx.x * 8; at < len; at += 8192) {
    const int n = clip(len - at);
    load8(x + at, n, h);
    load8(dy + at, n, d);
    back8<T>(g, row.c0 + at, n, mean, rstd, h, d, w);
    float o[8] = {};
    if (g.extra) load8(static_cast<const T *>(g.extra) + row.n * g.extra_sample + row.c0 + at, n, o);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float q = __builtin_fmaf(-h[j], m2, __builtin_fmaf(d[j], w[j], -m1)) * rstd;
      d[j] = g.extra ? o[j] + q : q;
    }
    store8(static_cast<T *>(g.out) + row.n * g.out_sample + row.c0 + at, n, d);
  }
}
// ... the partial sums over samples blockIdx.y, blockIdx.y + gridDim.y, ... of a thread's eight channels.
template <class T>
__global__ void __launch_bounds__(kThreads) k_norm_long_channels(GroupNorm g) {
  const long long len = g.channels / g.groups;
  const long long per_group = (len + 7) / 8, q = (long long)blockIdx.x * kThreads + threadIdx.x;
  if (q >= per_group * g.groups) return;
  const long long gr = q / per_group, at = (q - gr * per_group) * 8, c = gr * len + at;
  const int n = len - at < 8 ? (int)(len - at) : 8;
  float sw[8] = {}, sb[8] = {};
  for (long long s = blockIdx.y; s < g.samples; s += gridDim.y) {
    float h[8], d[8], w[8];
    load8(static_cast<const T *>(g.x) + s * g.x_sample + c, n, h);
    load8(static_cast<const T *>(g.dy) + s * g.dy_sample + c, n, d);
    back8<T>(g, c, n, g.mean[s * g.groups + gr], g.rstd[s * g.groups + gr], h, d, w);
#pragma unroll
    for (int j = 0; j < 8; ++j) sw[j] = __builtin_fmaf(d[j], h[j], sw[j]), sb[j] = sb[j] + d[j];
  }
  float *part = g.scratch + (long long)blockIdx.y * 2 * g.channels + c;
  store8(part, n, sw);
  store8(part + g.channels, n, sb);
}

// dweight and dbias from `count` rows of partial sums [2][channels]: 16 columns a workgroup, its 64 teams of 16 lanes take rows in turn.  With `to`: the
// sums of parts of `each` rows, a row a part.  A part's workgroups are adjacent.
__global__ void __launch_bounds__(1024) k_norm_join(GroupNorm g, const float *part, long long count, long long each, float *to) {
  __shared__ float red[64][16 + 1];
  const int lane = threadIdx.x & 15, team = threadIdx.x / 16;
  const long long total = 2 * g.channels;
  const long long columns = (total + 15) / 16, id = g.first + blockIdx.x, y = to ? id / columns : 0, x = id - y * columns, c = x * 16 + lane;
  const long long first = y * each, end = first + each < count ? first + each : count;
  float s = 0.0f;
  if (c < total) {
    long long r = first + team;
    for (; r + 3 * 64 < end; r += 4 * 64) {   // four on their way
      float v[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) v[q] = part[(r + q * 64) * total + c];
#pragma unroll
      for (int q = 0; q < 4; ++q) s = s + v[q];
    }
    for (; r < end; r += 64) s = s + part[r * total + c];
  }
  red[team][lane] = s;
  __syncthreads();
  const int column = threadIdx.x / 64;   // a wave adds up a column's
  s = lanes_sum<64>(red[threadIdx.x & 63][column]);
  const long long o = x * 16 + column;
  if ((threadIdx.x & 63) == 0 && o < total) {
    if (to) {
      to[y * total + o] = s;
      return;
    }
    float *out = o < g.channels ? g.dweight : g.dbias;
    const long long at = o < g.channels ? o : o - g.channels;
    if (out) out[at] = g.accumulate ? out[at] + s : s;
  }
}

// ------------------------------------------------------------------------------------------------ maps
// How a launch cuts [samples][positions][channels].  A block is `width` channels (the last may be shorter): whole groups, or, with
// blocks_a_group > 1, a part of one.  A piece is `chunk` positions of a block.
struct Maps {
  int per;               // channels of a group
  int width, blocks;     // channels of a block, blocks
  int blocks_a_group;
  int vectors;           // ceil(width / 8): threads across
  int rows;              // positions at a time
  int chunk, chunks;     // positions of a piece, pieces
  int pieces_a_group;    // chunks, times blocks_a_group
  bool apart;            // the pieces' sums are joined by a launch of their own, not by each workgroup that needs them
};

// What a workgroup works on, and its thread's channels.
template <int NT>
struct Place {
  long long n;
  int block, chunk;
  long long c0;       // the block's first channel
  int width;          // its channels
  u32 p0, p1;         // its positions
  int vec, row;       // the thread's
  int own;            // channels that it owns (<= 0: none), from c0 + 8 vec on
  __device__ __forceinline__ Place(const GroupNorm &g, const Maps &m) {
    const u32 id = (u32)g.first + blockIdx.x, each = (u32)(m.blocks * m.chunks);
    n = id / each;
    const int piece = (int)(id - (u32)n * each);
    chunk = piece / m.blocks;
    block = piece - chunk * m.blocks;
    if (m.blocks_a_group > 1) {
      const int gr = block / m.blocks_a_group, in = block - gr * m.blocks_a_group;
      c0 = (long long)gr * m.per + in * m.width;
      width = m.per - in * m.width < m.width ? m.per - in * m.width : m.width;
    } else {
      c0 = (long long)block * m.width;
      width = g.channels - c0 < m.width ? (int)(g.channels - c0) : m.width;
    }
    p0 = (u32)chunk * m.chunk;
    p1 = g.positions - p0 < m.chunk ? (u32)g.positions : p0 + m.chunk;
    row = threadIdx.x / m.vectors;
    vec = threadIdx.x - row * m.vectors;
    own = row < m.rows ? width - vec * 8 : 0;
  }
};

// v[j] of every thread summed per channel over the rows of the workgroup: into sums[0 .. width).  lanes: NT * 8 floats.
template <int NT>
__device__ __forceinline__ void channel_sums(const Maps &m, const Place<NT> &at, const float (&v)[8], float *lanes, float *sums) {
  __syncthreads();
  if (at.own > 0)
#pragma unroll
    for (int j = 0; j < 8; ++j) lanes[(at.row * 8 + j) * m.vectors + at.vec] = v[j];
  __syncthreads();
  const int across = m.vectors * 8;
  // several threads a channel, a power of two, adjacent in the rows that they take
  int share = 1;
  while (share * 2 * across <= NT && share * 2 <= m.rows) share *= 2;
  float s = 0.0f;
  const int t = threadIdx.x, q = t % across, r0 = t / across;
  for (int c = q; c < across && r0 < share; c += NT)   // one turn, but for blocks wider than the workgroup
  {
    s = 0.0f;
    for (int r = r0; r < m.rows; r += share) s = s + lanes[r * across + c];
    const int j = c / m.vectors, vec = c - j * m.vectors;
    if (share == 1 && vec * 8 + j < at.width) sums[vec * 8 + j] = s;
  }
  if (share > 1) {
    __syncthreads();
    if (r0 < share) lanes[r0 * across + q] = s;
    __syncthreads();
    if (t < across) {
      s = 0.0f;
      for (int r = 0; r < share; ++r) s = s + lanes[r * across + t];
      const int j = t / m.vectors, vec = t - j * m.vectors;
      if (vec * 8 + j < at.width) sums[vec * 8 + j] = s;
    }
  }
  __syncthreads();
}

// Sums of each group's channels: out[g] for the groups of the block (one, where the block is a part of a group).
template <int NT>
__device__ __forceinline__ void group_sums(const Maps &m, const Place<NT> &at, const float *channels, float *out) {
  const int per = m.blocks_a_group > 1 ? at.width : m.per, groups = at.width / per;
  if (per <= 16) {
    for (int q = threadIdx.x; q < groups; q += NT) {
      float s = 0.0f;
      for (int c = 0; c < per; ++c) s = s + channels[q * per + c];
      out[q] = s;
    }
  } else {
    for (int q = threadIdx.x / 64; q < groups; q += NT / 64) {
      float s = 0.0f;
      for (int c = threadIdx.x & 63; c < per; c += 64) s = s + channels[q * per + c];
      s = lanes_sum<64>(s);
      if ((threadIdx.x & 63) == 0) out[q] = s;
    }
  }
  __syncthreads();
}

// channels of a block, by the workgroup's threads: what its sums take of shared memory bounds how many workgroups a CU holds
constexpr int widest(int threads) { return threads == 64 ? 512 : 2048; }

// The group of each of a thread's channels, within the block.
__device__ __forceinline__ void groups8(const Maps &m, int c, int (&q)[8]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) q[j] = m.blocks_a_group > 1 ? 0 : (c + j) / m.per;
}

enum MapsPass { kWhole = 0, kPieces = 1, kJoined = 2 };

// Up to so many pieces of a sample (gradient) or of a group (forward) are joined by each workgroup that needs them, which saves a launch; more are joined
// once, so that a map's time grows with its size and not with its square.  Gradient of bf16, joined by each and once: 32 pieces (2 x 4096 x 64) 16.3 and
// 18.4 us, 64 (57 x 4096 x 128 in one group) 86 and 69, 512 (8 x 65536 x 128) 416 and 152.  Forward, 256 pieces (8 x 65536 x 128): 104 and 79 us.
constexpr int kTogether = 32, kTogetherForward = 128;

// The values of a piece: `per` channels, or a block's share of them, at `chunk` positions, or what is left.
__device__ __forceinline__ float piece_values(const GroupNorm &g, const Maps &m, int piece) {
  const int in = m.blocks_a_group > 1 ? piece % m.blocks_a_group : 0, ch = m.blocks_a_group > 1 ? piece / m.blocks_a_group : piece;
  const int w = m.blocks_a_group > 1 ? (m.per - in * m.width < m.width ? m.per - in * m.width : m.width) : m.per;
  const int p = g.positions - (long long)ch * m.chunk < m.chunk ? (int)(g.positions - (long long)ch * m.chunk) : m.chunk;
  return (float)w * (float)p;
}
// Mean and 1 / sqrt(variance + eps) of a group from its pieces' means and squares (Chan et al.: squares about the common mean), by a team of lanes, the
// same in each.
template <int TEAM>
__device__ __forceinline__ void join_pieces(const GroupNorm &g, const Maps &m, const float *s, float &mean, float &rstd) {
  __shared__ float red[2][TEAM > 64 ? TEAM / 64 : 1];
  const float total = (float)m.per * (float)g.positions;
  const int lane = threadIdx.x % TEAM;
  mean = 0.0f;
  for (int i = lane; i < m.pieces_a_group; i += TEAM) mean = __builtin_fmaf(s[2ll * i], piece_values(g, m, i) / total, mean);
  mean = team_sum<TEAM>(mean, red[0]);
  float sq = 0.0f;
  for (int i = lane; i < m.pieces_a_group; i += TEAM) {
    const float d = s[2ll * i] - mean;
    sq = sq + __builtin_fmaf(d * d, piece_values(g, m, i), s[2ll * i + 1]);
  }
  rstd = 1.0f / sqrtf(team_sum<TEAM>(sq, red[1]) / total + g.eps);
}
// A workgroup a group: its pieces are read once, where each workgroup that makes a piece's result would read all of them.
__global__ void __launch_bounds__(1024) k_norm_maps_join(GroupNorm g, Maps m) {
  float mean, rstd;
  const long long r = g.first + blockIdx.x;
  join_pieces<1024>(g, m, g.scratch + r * m.pieces_a_group * 2, mean, rstd);
  if (threadIdx.x == 0) g.mean[r] = mean, g.rstd[r] = rstd;
}

// kWhole: a block's values are in registers from the mean to the result.  kPieces: mean and squares of a piece, per group, to
// scratch[n][group][piece][2].  kJoined: those of the group's pieces joined, where k_norm_maps_join has not done that, and the result.
template <class T, int NT, int U, int PASS, bool EVEN>
__global__ void __launch_bounds__(NT) k_norm_maps(GroupNorm g, Maps m) {
  __shared__ float lanes[PASS == kJoined ? 1 : NT * 8];
  __shared__ float channels[PASS == kJoined ? 1 : widest(NT)];
  __shared__ float means[widest(NT)], rstds[widest(NT)];   // per group of the block
  const Place<NT> at(g, m);
  const T *x = static_cast<const T *>(g.x) + at.n * g.x_sample + at.c0 + at.vec * 8;
  Eight<T> raw[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const u32 p = at.p0 + at.row + u * m.rows;
    raw[u].template load<EVEN>(x + (long long)p * g.x_pos, p < at.p1 ? at.own : 0);
  }
  int q[8];
  groups8(m, at.vec * 8, q);
  const int per = m.blocks_a_group > 1 ? at.width : m.per, groups = at.width / per;
  const long long first = m.blocks_a_group > 1 ? at.block / m.blocks_a_group : at.c0 / m.per;   // the block's first group
  if constexpr (PASS != kJoined) {
    const float count = (float)per * (float)(at.p1 - at.p0);
    float v[8] = {};
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float e[8];
      raw[u].get(e);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = v[j] + e[j];
    }
    channel_sums<NT>(m, at, v, lanes, channels);
    group_sums<NT>(m, at, channels, means);
    for (int k = threadIdx.x; k < groups; k += NT) means[k] = means[k] / count;
    __syncthreads();
    float mean[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      mean[j] = (EVEN ? at.own > 0 : j < at.own) ? means[q[j]] : 0.0f;
      v[j] = 0.0f;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float e[8];
      raw[u].get(e);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float d = at.p0 + at.row + u * m.rows < at.p1 && (EVEN ? at.own > 0 : j < at.own) ? e[j] - mean[j] : 0.0f;
        v[j] = __builtin_fmaf(d, d, v[j]);
      }
    }
    channel_sums<NT>(m, at, v, lanes, channels);
    group_sums<NT>(m, at, channels, rstds);
    if constexpr (PASS == kPieces) {
      const int piece = m.blocks_a_group > 1 ? at.chunk * m.blocks_a_group + at.block % m.blocks_a_group : at.chunk;
      for (int k = threadIdx.x; k < groups; k += NT) {
        float *o = g.scratch + ((at.n * g.groups + first + k) * m.pieces_a_group + piece) * 2;
        o[0] = means[k], o[1] = rstds[k];
      }
      return;
    }
    for (int k = threadIdx.x; k < groups; k += NT) rstds[k] = 1.0f / sqrtf(rstds[k] / count + g.eps);
  } else {
    for (int k = threadIdx.x / 64; k < groups; k += NT / 64) {   // a wave a group
      const long long r = at.n * g.groups + first + k;
      float mean, rstd;
      if (m.apart) mean = g.mean[r], rstd = g.rstd[r];
      else join_pieces<64>(g, m, g.scratch + r * m.pieces_a_group * 2, mean, rstd);
      if ((threadIdx.x & 63) == 0) means[k] = mean, rstds[k] = rstd;
    }
  }
  __syncthreads();
  if (!(PASS == kJoined && m.apart) && at.chunk == 0 && (m.blocks_a_group == 1 || at.block % m.blocks_a_group == 0))
    for (int k = threadIdx.x; k < groups; k += NT) {
      g.mean[at.n * g.groups + first + k] = means[k];
      g.rstd[at.n * g.groups + first + k] = rstds[k];
    }
  if (at.own <= 0) return;
  float w[8], b[8];
  vector8<EVEN>(g.weight ? g.weight + at.c0 + at.vec * 8 : nullptr, 1.0f, at.own, w);
  vector8<EVEN>(g.bias ? g.bias + at.c0 + at.vec * 8 : nullptr, 0.0f, at.own, b);
  float mean[8], rstd[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) mean[j] = (EVEN ? at.own > 0 : j < at.own) ? means[q[j]] : 0.0f, rstd[j] = (EVEN ? at.own > 0 : j < at.own) ? rstds[q[j]] : 0.0f;
  T *y = static_cast<T *>(g.out) + at.n * g.out_sample + at.c0 + at.vec * 8;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const u32 p = at.p0 + at.row + u * m.rows;
    if (p < at.p1) {
      float e[8];
      raw[u].get(e);
#pragma unroll
      for (int j = 0; j < 8; ++j) e[j] = __builtin_fmaf((e[j] - mean[j]) * rstd[j], w[j], b[j]);
      act8<T>(g.activation, e);
      store8<EVEN>(y + (long long)p * g.out_pos, at.own, e);
    }
  }
}

// What dx needs of groups wider than a block: the sums of a sample's channels, [n][2][channels], weighted and summed over each of its groups, to
// out[n][group][2].  A workgroup a group.
__global__ void __launch_bounds__(1024) k_norm_group_sums(GroupNorm g, const float *sums, float2 *out) {
  __shared__ float2 red[16];
  const u32 r = (u32)g.first + blockIdx.x, gr = r % (u32)g.groups;
  const long long n = r / (u32)g.groups, c0 = gr * (g.channels / g.groups), end = c0 + g.channels / g.groups;
  const float *s = sums + n * 2 * g.channels;
  float s1 = 0.0f, s2 = 0.0f;
  for (long long c = c0 + threadIdx.x; c < end; c += 1024) {
    const float w = g.weight ? g.weight[c] : 1.0f;
    s2 = __builtin_fmaf(s[c], w, s2);
    s1 = __builtin_fmaf(s[g.channels + c], w, s1);
  }
  team_sums<1024>(s1, s2, red);
  if (threadIdx.x == 0) out[r] = {s1, s2};
}

// The gradient.  Per channel of a piece: the sums of d (dy through the activation) and of d h, to scratch[n][chunk][2][channels];
// from them come dweight and dbias, and, weighted and summed over a group, what dx needs.  kJoined: they come from `sums`, [n][2][channels] where
// the chunks have been joined (m.apart) and as kPieces left them otherwise, or, for groups wider than a block, from `of_groups`.
template <class T, int NT, int U, int PASS, bool EVEN>
__global__ void __launch_bounds__(NT) k_norm_maps_grad(GroupNorm g, Maps m, const float *sums, const float2 *of_groups) {
  __shared__ float lanes[PASS == kJoined ? 1 : NT * 8];
  __shared__ float cw[widest(NT)], cb[widest(NT)];   // per channel: the sums of d h and of d
  const Place<NT> at(g, m);
  const long long c = at.c0 + at.vec * 8;
  const T *x = static_cast<const T *>(g.x) + at.n * g.x_sample + c, *dy = static_cast<const T *>(g.dy) + at.n * g.dy_sample + c;
  Eight<T> rx[U], rd[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const u32 p = at.p0 + at.row + u * m.rows;
    const int n = p < at.p1 ? at.own : 0;
    rx[u].template load<EVEN>(x + (long long)p * g.x_pos, n);
    rd[u].template load<EVEN>(dy + (long long)p * g.dy_pos, n);
  }
  int q[8];
  groups8(m, at.vec * 8, q);
  const int per = m.blocks_a_group > 1 ? at.width : m.per, groups = at.width / per;
  const long long first = m.blocks_a_group > 1 ? at.block / m.blocks_a_group : at.c0 / m.per;
  // What goes through the activation is computed as in the forward pass, operation by operation: an entry is on the same side of a kink in both, and
  // a mean far from 0 costs nothing (as x (rstd w) + (b - mean rstd w) it would be a difference of large numbers).
  float mean[8], rstd[8], w[8], b[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const bool mine = EVEN ? at.own > 0 : j < at.own;
    mean[j] = mine ? g.mean[at.n * g.groups + first + q[j]] : 0.0f;
    rstd[j] = mine ? g.rstd[at.n * g.groups + first + q[j]] : 0.0f;
    w[j] = b[j] = 0.0f;
  }
  if (at.own > 0) {
    vector8<EVEN>(g.weight ? g.weight + c : nullptr, 1.0f, at.own, w);
    vector8<EVEN>(g.bias ? g.bias + c : nullptr, 0.0f, at.own, b);
  }
  // h: the normalised values; d: dy through the activation
  const auto back = [&](int u, float (&h)[8], float (&d)[8]) {
    rx[u].get(h);
    rd[u].get(d);
#pragma unroll
    for (int j = 0; j < 8; ++j) h[j] = (h[j] - mean[j]) * rstd[j];
    if (g.activation != kActNone) {
      float z[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) z[j] = __builtin_fmaf(h[j], w[j], b[j]);
      slope8<T>(g.activation, z, d);
    }
  };
  if constexpr (PASS != kJoined) {
    float vw[8] = {}, vb[8] = {};
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (at.p0 + at.row + u * m.rows < at.p1) {
        float h[8], d[8];
        back(u, h, d);
#pragma unroll
        for (int j = 0; j < 8; ++j) vw[j] = __builtin_fmaf(d[j], h[j], vw[j]), vb[j] = vb[j] + d[j];
      }
    channel_sums<NT>(m, at, vw, lanes, cw);
    channel_sums<NT>(m, at, vb, lanes, cb);
    float *o = g.scratch + ((at.n * m.chunks + at.chunk) * 2) * g.channels + at.c0;
    for (int k = threadIdx.x; k < at.width; k += NT) o[k] = cw[k], o[g.channels + k] = cb[k];
    if constexpr (PASS == kPieces) return;
  } else {
    if (m.blocks_a_group > 1) {
      if (threadIdx.x == 0) {
        const float2 of = of_groups[at.n * g.groups + first];
        cb[0] = of.x, cw[0] = of.y;
      }
    } else {
      const int parts = m.apart ? 1 : m.chunks;
      for (int k = threadIdx.x; k < at.width; k += NT) {
        const float *s = sums + at.n * parts * 2 * g.channels + at.c0 + k;
        float s1 = 0.0f, s2 = 0.0f;
        for (int ch = 0; ch < parts; ch += 8) {   // eight on their way
          float v1[8], v2[8];
#pragma unroll
          for (int u = 0; u < 8; ++u) {
            const float *p = s + (long long)(ch + u < parts ? ch + u : parts - 1) * 2 * g.channels;
            v2[u] = p[0], v1[u] = p[g.channels];
          }
#pragma unroll
          for (int u = 0; u < 8; ++u)
            if (ch + u < parts) s2 = s2 + v2[u], s1 = s1 + v1[u];
        }
        cw[k] = s2, cb[k] = s1;
      }
    }
  }
  __syncthreads();
  __shared__ float m1[widest(NT)], m2[widest(NT)];
  const float total = (float)m.per * (float)g.positions;
  if (m.blocks_a_group > 1) {
    if (threadIdx.x == 0) m1[0] = cb[0] / total, m2[0] = cw[0] / total;
    __syncthreads();
  } else {
    for (int k = threadIdx.x; k < at.width; k += NT) {
      const float wk = g.weight ? g.weight[at.c0 + k] : 1.0f;
      cw[k] = cw[k] * wk, cb[k] = cb[k] * wk;
    }
    __syncthreads();
    group_sums<NT>(m, at, cb, m1);
    group_sums<NT>(m, at, cw, m2);
    for (int k = threadIdx.x; k < groups; k += NT) m1[k] = m1[k] / total, m2[k] = m2[k] / total;
    __syncthreads();
  }
  if (at.own <= 0) return;
  float e1[8], e2[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const bool mine = EVEN ? at.own > 0 : j < at.own;
    e1[j] = mine ? m1[q[j]] : 0.0f;
    e2[j] = mine ? m2[q[j]] : 0.0f;
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const u32 p = at.p0 + at.row + u * m.rows;
    if (p < at.p1) {
      float h[8], d[8], o[8];
      if (g.extra) load8<EVEN>(static_cast<const T *>(g.extra) + at.n * g.extra_sample + p * g.extra_pos + c, at.own, o);
      back(u, h, d);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float v = __builtin_fmaf(-h[j], e2[j], __builtin_fmaf(d[j], w[j], -e1[j])) * rstd[j];
        d[j] = g.extra ? o[j] + v : v;
      }
      store8<EVEN>(static_cast<T *>(g.out) + at.n * g.out_sample + p * g.out_pos + c, at.own, d);
    }
  }
}

// ------------------------------------------------------------------------------------------------ launches
long long gcd(long long a, long long b) { return b == 0 ? a : gcd(b, a % b); }

// A block: whole groups and whole vectors of eight, so that no thread's channels cross a block's edge more often than at the end; at least 128
// bytes of a row, more where few positions would leave threads idle; at most as many channels as widest() says.
Maps maps_of(const GroupNorm &g, int threads, int each, int bytes = 128) {
  Maps m = {};
  m.per = (int)(g.channels / g.groups);
  m.blocks_a_group = 1;
  const int most = widest(threads);
  if (m.per > most) {
    m.blocks_a_group = (m.per + most - 1) / most;
    m.width = most;
    m.blocks = m.blocks_a_group * (int)g.groups;
  } else {
    long long unit = m.per / gcd(m.per, 8) * 8;
    if (unit > 512 || unit > g.channels) unit = m.per;
    const long long least = bytes / (g.type == kF32 ? 4 : 2);
    long long w = unit;
    while (w < g.channels && w + unit <= most && (w < least || (w + 7) / 8 * g.positions < (threads < kThreads ? threads : kThreads))) w += unit;
    if (w > g.channels) w = g.channels;
    m.width = (int)w;
    m.blocks = (int)((g.channels + w - 1) / w);
  }
  m.vectors = (m.width + 7) / 8;
  m.rows = threads / m.vectors;
  m.chunk = m.rows * each;
  m.chunks = (int)((g.positions + m.chunk - 1) / m.chunk);
  m.pieces_a_group = m.chunks * m.blocks_a_group;
  return m;
}
constexpr long long kMostWorkgroups = 0x7fffffff;   // 32-bit numbers in the kernels
long long workgroups(const GroupNorm &g, const Maps &m) { return (long long)m.blocks * m.chunks * g.samples; }
bool whole(const GroupNorm &g, const Maps &m) { return m.chunks == 1 && m.blocks_a_group == 1 && workgroups(g, m) <= kMostWorkgroups; }

// Small samples, many of them: a wave each, whose barriers are nothing (65536 samples of 4 positions and 16 channels: 93 us, in
// workgroups of 256 410; 1000 of 16 and 64 6.7, 8.9; 500 of 32 and 64 7.5 either way).
bool wave_whole(const GroupNorm &g, const Maps &m) { return whole(g, m) && workgroups(g, m) >= 512; }

// The rows' cut: lanes of a team and eights a lane, or neither: longer.  The gradient keeps two sums for each of its entries: fewer a lane.
struct Rows {
  int team, each;
};
Rows rows_of(const GroupNorm &g, bool gradient) {
  const long long v = (g.channels / g.groups + 7) / 8;
  if (v <= 16) return {16, 1};
  if (v <= 64) return {64, 1};
  if (gradient && v <= 128) return {64, 2};
  if (gradient && v <= 256) return {256, 1};
  if (v <= 256) return {64, 4};
  if (v <= 1024) return {256, 4};
  return {0, 0};
}
// Workgroups that share a group's rows: enough to fill the device a few times, but with four turns each before that, so that their partial
// sums (8 bytes a channel) are little beside the rows.
long long rows_workgroups(const GroupNorm &g, const Rows &r) {
  const long long teams = kThreads / r.team, turns = (g.samples + teams - 1) / teams;
  const auto at_least_one = [](long long v) { return v < 1 ? 1 : v; };
  const long long least = at_least_one(256 / g.groups), most = at_least_one(1024 / g.groups);
  long long want = turns / 4;
  want = want < least ? least : want > most ? most : want;
  return turns < want ? turns : want;
}
constexpr long long kLongSplits = 64;

// Parts in which rows of partial sums are joined first: with many samples of few channels one workgroup would take them all (65536 samples of 4 positions
// and 16 channels: 137 us in one part).
long long join_parts(long long count) {
  const long long parts = (count + 1023) / 1024;
  return count <= 4096 ? 1 : parts < 256 ? parts : 256;
}

template <int N>
using number = std::integral_constant<int, N>;

// Calls f with whether every eight entries exist together or not at all.
template <class F>
void by_even(const GroupNorm &g, F &&f) {
  bool even = g.channels / g.groups % 8 == 0;
  if (!even && g.positions > 1) {   // small groups side by side in blocks of whole eights
    even = g.channels % 8 == 0;
    for (const Maps &m : {maps_of(g, kThreads, 1), maps_of(g, kThreads, 1, 64), maps_of(g, 64, 1)})
      even = even && (m.blocks_a_group == 1 ? m.width : m.per) % 8 == 0;
  }
  if (even) f(std::true_type());
  else f(std::false_type());
}

template <class T>
hipError_t norm(const GroupNorm &g, hipStream_t s) {
  hipError_t rc = hipSuccess;
  by_even(g, [&](auto even) {
    constexpr bool kEven = decltype(even)::value;
    if (g.positions == 1) {
      const long long rows = g.samples * g.groups;
      const Rows r = rows_of(g, false);
      if (r.team == 0) {
        in_launches(g, rows, 1024, [&](const GroupNorm &some, unsigned grid) { k_norm_long_rows<T><<<dim3(grid), 1024, 0, s>>>(some); });
        return;
      }
      in_launches(g, (rows + kThreads / r.team - 1) / (kThreads / r.team), kThreads, [&](const GroupNorm &some, unsigned grid) {
        if (r.team == 16) k_norm_rows<T, 16, 1, kEven><<<dim3(grid), kThreads, 0, s>>>(some);
        else if (r.team == 64 && r.each == 1) k_norm_rows<T, 64, 1, kEven><<<dim3(grid), kThreads, 0, s>>>(some);
        else if (r.team == 64) k_norm_rows<T, 64, 4, kEven><<<dim3(grid), kThreads, 0, s>>>(some);
        else k_norm_rows<T, 256, 4, kEven><<<dim3(grid), kThreads, 0, s>>>(some);
      });
      return;
    }
    Maps m;
    const auto run = [&](auto threads, auto each, auto pass) {
      constexpr int kNt = decltype(threads)::value;
      in_launches(g, workgroups(g, m), kNt, [&](const GroupNorm &some, unsigned grid) {
        k_norm_maps<T, kNt, decltype(each)::value, decltype(pass)::value, kEven><<<dim3(grid), kNt, 0, s>>>(some, m);
      });
    };
    if (m = maps_of(g, 64, 2), wave_whole(g, m)) run(number<64>(), number<2>(), number<kWhole>());
    else if (m = maps_of(g, 64, 8), wave_whole(g, m)) run(number<64>(), number<8>(), number<kWhole>());
    else if (m = maps_of(g, 256, 2), whole(g, m)) run(number<256>(), number<2>(), number<kWhole>());
    else if (m = maps_of(g, 256, 4), whole(g, m)) run(number<256>(), number<4>(), number<kWhole>());
    else if (m = maps_of(g, 256, 8), whole(g, m)) run(number<256>(), number<8>(), number<kWhole>());
    else if (m = maps_of(g, 1024, 8), whole(g, m)) run(number<1024>(), number<8>(), number<kWhole>());
    else {
      m = maps_of(g, 256, 8);
      if (workgroups(g, m) > kMostWorkgroups) {
        rc = hipErrorInvalidValue;
        return;
      }
      m.apart = m.pieces_a_group > kTogetherForward;
      run(number<256>(), number<8>(), number<kPieces>());
      if (m.apart)
        in_launches(g, g.samples * g.groups, 1024, [&](const GroupNorm &some, unsigned grid) { k_norm_maps_join<<<dim3(grid), 1024, 0, s>>>(some, m); });
      run(number<256>(), number<8>(), number<kJoined>());
    }
  });
  return rc != hipSuccess ? rc : hipGetLastError();
}

// The gradient's cut of maps, and whether one launch does it.
struct GradMaps {
  Maps m;
  int threads, each;
  bool whole;
};
GradMaps grad_maps(const GroupNorm &g) {
  GradMaps q = {maps_of(g, 64, 2), 64, 2, true};
  if (wave_whole(g, q.m)) return q;
  q = {maps_of(g, 64, 4), 64, 4, true};
  if (wave_whole(g, q.m)) return q;
  q = {maps_of(g, 256, 2), 256, 2, true};
  if (whole(g, q.m)) return q;
  q = {maps_of(g, 256, 4), 256, 4, true};
  if (whole(g, q.m)) return q;
  if (g.type == kBf16) {   // two tensors of fp32 would not stay in the registers
    q = {maps_of(g, 512, 8, 64), 512, 8, true};
    if (whole(g, q.m)) return q;
  }
  q = {maps_of(g, 256, 4), 256, 4, false};
  q.m.apart = q.m.chunks > kTogether || q.m.blocks_a_group > 1;
  return q;
}
// Rows of partial sums that dweight and dbias are made of.
long long rows_of_sums(const GroupNorm &g, const Maps &m) { return g.samples * (m.apart ? 1 : m.chunks); }
// ... and floats in front of them: those of the pieces that they are joined from, and the groups' sums.
long long before_sums(const GroupNorm &g, const Maps &m) {
  return !m.apart ? 0 : g.samples * 2 * (m.chunks * g.channels + (m.blocks_a_group > 1 ? g.groups : 0));
}

template <class T>
hipError_t norm_grad(const GroupNorm &call, hipStream_t s) {
  GroupNorm g = call;
  const bool sums = g.dweight || g.dbias;
  long long count = 0;   // rows of partial sums, from part on
  float *part = g.scratch;
  // `rows` rows of partial sums, in parts of `each`
  const auto join = [&](const float *from, long long rows, long long each, float *to) {
    const long long columns = (2 * g.channels + 15) / 16, parts = to ? (rows + each - 1) / each : 1;
    in_launches(g, columns * parts, 1024, [&](const GroupNorm &some, unsigned grid) { k_norm_join<<<dim3(grid), 1024, 0, s>>>(some, from, rows, each, to); });
  };
  hipError_t rc = hipSuccess;
  by_even(g, [&](auto even) {
    constexpr bool kEven = decltype(even)::value;
    if (g.samples > 0 && g.positions == 1) {
      const Rows r = rows_of(g, true);
      if (!sums) g.scratch = nullptr;
      if (r.team == 0) {
        if (sums) {
          count = g.samples < kLongSplits ? g.samples : kLongSplits;
          const long long eights = ((g.channels / g.groups + 7) / 8) * g.groups;
          k_norm_long_channels<T><<<dim3((unsigned)((eights + kThreads - 1) / kThreads), (unsigned)count), kThreads, 0, s>>>(g);
        }
        in_launches(g, g.samples * g.groups, 1024, [&](const GroupNorm &some, unsigned grid) { k_norm_long_rows_grad<T><<<dim3(grid), 1024, 0, s>>>(some); });
        return;
      }
      count = rows_workgroups(g, r);
      in_launches(g, g.groups, kThreads, [&](const GroupNorm &some, unsigned x) {
        const dim3 grid(x, (unsigned)count);
        if (r.team == 16) k_norm_rows_grad<T, 16, 1, kEven><<<grid, kThreads, 0, s>>>(some);
        else if (r.team == 64 && r.each == 1) k_norm_rows_grad<T, 64, 1, kEven><<<grid, kThreads, 0, s>>>(some);
        else if (r.team == 64) k_norm_rows_grad<T, 64, 2, kEven><<<grid, kThreads, 0, s>>>(some);
        else if (r.each == 1) k_norm_rows_grad<T, 256, 1, kEven><<<grid, kThreads, 0, s>>>(some);
        else k_norm_rows_grad<T, 256, 4, kEven><<<grid, kThreads, 0, s>>>(some);
      });
    } else if (g.samples > 0 && g.positions > 0) {
      const GradMaps q = grad_maps(g);
      if (workgroups(g, q.m) > kMostWorkgroups) {
        rc = hipErrorInvalidValue;
        return;
      }
      count = rows_of_sums(g, q.m);
      part = g.scratch + before_sums(g, q.m);
      float2 *of_groups = nullptr;
      const auto run = [&](auto threads, auto each, auto pass) {
        constexpr int kNt = decltype(threads)::value;
        in_launches(g, workgroups(g, q.m), kNt, [&](const GroupNorm &some, unsigned grid) {
          k_norm_maps_grad<T, kNt, decltype(each)::value, decltype(pass)::value, kEven><<<dim3(grid), kNt, 0, s>>>(some, q.m, part, of_groups);
        });
      };
      if (!q.whole) {
        run(number<256>(), number<4>(), number<kPieces>());
        if (q.m.apart) {
          join(g.scratch, g.samples * q.m.chunks, q.m.chunks, part);
          if (q.m.blocks_a_group > 1) {
            of_groups = reinterpret_cast<float2 *>(g.scratch + g.samples * 2 * q.m.chunks * g.channels);
            in_launches(g, g.samples * g.groups, 1024, [&](const GroupNorm &some, unsigned grid) { k_norm_group_sums<<<dim3(grid), 1024, 0, s>>>(some, part, of_groups); });
          }
        }
        run(number<256>(), number<4>(), number<kJoined>());
      } else if (q.threads == 64) {
        if (q.each == 2) run(number<64>(), number<2>(), number<kWhole>());
        else run(number<64>(), number<4>(), number<kWhole>());
      } else if (q.threads == 512) {
        if constexpr (sizeof(T) == 2) run(number<512>(), number<8>(), number<kWhole>());
      } else if (q.each == 2) {
        run(number<256>(), number<2>(), number<kWhole>());
      } else {
        run(number<256>(), number<4>(), number<kWhole>());
      }
    }
  });
  if (rc != hipSuccess) return rc;
  if (sums) {
    if (const long long parts = join_parts(count); parts > 1) {
      float *to = part + count * 2 * g.channels;
      const long long each = (count + parts - 1) / parts;
      join(part, count, each, to);
      join(to, (count + each - 1) / each, parts, nullptr);
    } else {
      join(part, count, count, nullptr);
    }
  }
  return hipGetLastError();
}

}  // namespace

size_t group_norm_scratch(const GroupNorm &g, bool gradient) {
  if (g.samples == 0 || g.positions == 0 || g.channels == 0) return 0;
  if (!gradient) {
    if (g.positions == 1 || wave_whole(g, maps_of(g, 64, 8)) || whole(g, maps_of(g, 256, 8)) || whole(g, maps_of(g, 1024, 8))) return 0;
    return (size_t)(g.samples * g.groups * maps_of(g, 256, 8).pieces_a_group) * 2 * sizeof(float);
  }
  long long count, before = 0;
  if (g.positions == 1) {
    if (!g.dweight && !g.dbias) return 0;
    const Rows r = rows_of(g, true);
    count = r.team == 0 ? (g.samples < kLongSplits ? g.samples : kLongSplits) : rows_workgroups(g, r);
  } else {
    const Maps m = grad_maps(g).m;
    count = rows_of_sums(g, m), before = before_sums(g, m);
  }
  const long long parts = join_parts(count);
  return (size_t)(before + (count + (parts > 1 ? parts : 0)) * 2 * g.channels) * sizeof(float);
}

hipError_t launch_group_norm(const GroupNorm &g, hipStream_t s) { return g.type == kF32 ? norm<float>(g, s) : norm<bf16>(g, s); }
hipError_t launch_group_norm_grad(const GroupNorm &g, hipStream_t s) { return g.type == kF32 ? norm_grad<float>(g, s) : norm_grad<bf16>(g, s); }

}  // namespace qoda
