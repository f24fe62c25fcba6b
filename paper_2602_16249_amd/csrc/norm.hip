// Group norm with an activation over token tensors [B,N,C], channels last: an image's group of Cg = C / G channels has mean and
// variance over its N x Cg values, z = gamma (x - mean) rstd + beta, out = act(z).  B tokens of N = 1 and one group are the layer
// norm of every token.
//
// All of it is bound by memory: a few operations a value.  Two families:
//   rows     N = 1, one group, rows that fit a wave's registers: 4 to 64 lanes hold a row, statistics and values from one reading.
//   groups   everything else: a workgroup takes a run of an image's tokens times a block of at most 256 pieces of channels (whole
//            groups, or a share of one), every thread one column of pieces; a first launch leaves per group and workgroup a mean and a
//            sum of squares about it, a second one puts these together and makes the values.  Groups that one workgroup holds need one
//            launch, and it takes as many images as fit: 131072 x 1 x 64 in 4 groups, bf16, with an image each took 491 us, backward 910.
// A variance is always the mean square about a mean: of a workgroup's own values in registers, and between workgroups by
// M2 = sum of (M2_i + n_i (mean_i - mean)^2).  No difference of squares, so offsets and outliers cost no digits.
#include "launch.h"
#include "timing.h"

#include "cluster_common.h"
#include "dense_common.h"

#include <algorithm>

namespace affmae {
namespace {

constexpr int kThreads = 256;
constexpr int kHeldParts = 4;
constexpr int kWaves = kThreads / kWave;

int cdiv(long long a, long long b) { return (int)((a + b - 1) / b); }
size_t up256(size_t n) { return (n + 255) / 256 * 256; }

// z = xhat gamma + beta, out = act(z); BRIEF: see normal_cdf
template <bool BRIEF, int E>
__device__ __forceinline__ void normalise(float (&v)[E], float mean, float rstd, bool affine, const float (&gm)[E], const float (&bt)[E], int act) {
#pragma unroll
  for (int e = 0; e < E; ++e) {
    v[e] = (v[e] - mean) * rstd;
    if (affine) v[e] = __builtin_fmaf(v[e], gm[e], bt[e]);
  }
  act_values<BRIEF, E>(v, act);
}
// x becomes xhat, g (dout) becomes dz = dout act'(z)
template <bool BRIEF, int E>
__device__ __forceinline__ void slopes(float (&x)[E], float (&g)[E], float mean, float rstd, bool affine, const float (&gm)[E], const float (&bt)[E], int act) {
#pragma unroll
  for (int e = 0; e < E; ++e) x[e] = (x[e] - mean) * rstd;
  if (act != kActNone) {
    float z[E];
#pragma unroll
    for (int e = 0; e < E; ++e) z[e] = affine ? __builtin_fmaf(x[e], gm[e], bt[e]) : x[e];
    act_slopes<BRIEF, E>(g, z, act);
  }
}

// ------------------------------------------------------------------------------------------------------------------ rows

// the sum over the LANES lanes that hold a row, received by all of them: part of a wave, or the workgroup
template <int LANES>
__device__ __forceinline__ float row_sum(float v, int lane, float (&acc)[kWaves]) {
  if constexpr (LANES <= kWave) {
    return lanes_sum<1, LANES / 2>(v, lane);
  } else {
    static_assert(LANES == kThreads);
    v = wave_sum(v);
    __syncthreads();
    if (lane == 0) acc[threadIdx.x / kWave] = v;
    __syncthreads();
    return (acc[0] + acc[1]) + (acc[2] + acc[3]);
  }
}

// LANES lanes a row, PIECES pieces a lane; TAIL: rows end inside a piece.  One row of a lane group on its way at a time: more
// workgroups hide each other's ways better than more rows a workgroup (131072 x 64 bf16: 8.3 us, with four rows 9.8).
template <typename T, int LANES, int PIECES, bool TAIL>
__global__ __launch_bounds__(kThreads) void norm_rows_fwd_kernel(const T* __restrict__ x, const T* __restrict__ gamma, const T* __restrict__ beta, int rows,
                                                                 int C, float eps, int act, T* __restrict__ out, float* __restrict__ mean,
                                                                 float* __restrict__ rstd) {
  constexpr int E = kPiece<T>, kRows = kThreads / LANES;  // of a turn
  __shared__ float acc[kWaves];
  const int lane = threadIdx.x & (kWave - 1), l = threadIdx.x % LANES, at = threadIdx.x / LANES;
  const float inv = 1.f / (float)C;
  const auto there = [&](int c) { return TAIL ? C - c : E; };  // values from c on, if fewer than a piece
  float gm[PIECES][E], bt[PIECES][E];
#pragma unroll
  for (int p = 0; p < PIECES; ++p) {
    const int c = (p * LANES + l) * E;
    if (gamma && c < C) {
      load_some<E>(gamma + c, there(c), gm[p]);
      load_some<E>(beta + c, there(c), bt[p]);
    }
  }
  for (long long first = (long long)blockIdx.x * kRows; first < rows; first += (long long)gridDim.x * kRows) {
    const long long row = std::min<long long>(first + at, rows - 1);  // (further ones repeat the last: all lanes stay active)
    float v[PIECES][E];
    float s = 0.f;
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
      const int c = (p * LANES + l) * E;
      if (c < C) {
        load_some<E>(x + row * C + c, there(c), v[p]);
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e) v[p][e] = 0.f;
      }
    }
#pragma unroll
    for (int p = 0; p < PIECES; ++p)
#pragma unroll
      for (int e = 0; e < E; ++e) s += v[p][e];
    const float m = row_sum<LANES>(s, lane, acc) * inv;
    s = 0.f;
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
      const int c = (p * LANES + l) * E;
      if (c < C) {
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (!TAIL || c + e < C) s = __builtin_fmaf(v[p][e] - m, v[p][e] - m, s);
      }
    }
    const float r = 1.f / sqrtf(row_sum<LANES>(s, lane, acc) * inv + eps);
    if (first + at >= rows) continue;
    if (l == 0) {
      mean[row] = m;
      rstd[row] = r;
    }
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
      const int c = (p * LANES + l) * E;
      if (c >= C) continue;
      normalise<sizeof(T) == 2, E>(v[p], m, r, gamma != nullptr, gm[p], bt[p], act);
      store_some<E>(out + row * C + c, there(c), v[p]);
    }
  }
}

// dx, and per workgroup the sums of dz xhat and dz of every channel: part [workgroups][2][C].  TURNS rows of a lane group on their way
// at a time: two of short rows (65536 x 256 bf16: 22.0 us, with one 23.5, with four 24.7), one of long ones.
template <typename T, int LANES, int PIECES, int TURNS, bool TAIL>
__global__ __launch_bounds__(kThreads) void norm_rows_bwd_kernel(const T* __restrict__ x, const T* __restrict__ gamma, const T* __restrict__ beta,
                                                                 const float* __restrict__ mean, const float* __restrict__ rstd, const T* __restrict__ dout,
                                                                 int rows, int C, int act, T* __restrict__ dx, float* __restrict__ part) {
  constexpr int E = kPiece<T>, kRows = kThreads / LANES;
  __shared__ float sums[kRows][LANES * E];
  __shared__ float acc[kWaves];
  const int lane = threadIdx.x & (kWave - 1), l = threadIdx.x % LANES, at = threadIdx.x / LANES;
  const float inv = 1.f / (float)C;
  const auto there = [&](int c) { return TAIL ? C - c : E; };  // values from c on, if fewer than a piece
  float gm[PIECES][E], bt[PIECES][E], dg[PIECES][E], db[PIECES][E];
#pragma unroll
  for (int p = 0; p < PIECES; ++p) {
    const int c = (p * LANES + l) * E;
    if (gamma && c < C) {
      load_some<E>(gamma + c, there(c), gm[p]);
      load_some<E>(beta + c, there(c), bt[p]);
    }
#pragma unroll
    for (int e = 0; e < E; ++e) dg[p][e] = db[p][e] = 0.f;
  }
  for (long long first = (long long)blockIdx.x * kRows * TURNS; first < rows; first += (long long)gridDim.x * kRows * TURNS) {
    float v[TURNS][PIECES][E], g[TURNS][PIECES][E], m[TURNS], r[TURNS];
#pragma unroll
    for (int t = 0; t < TURNS; ++t) {
      const long long row = std::min<long long>(first + t * kRows + at, rows - 1);
      m[t] = mean[row];
      r[t] = rstd[row];
#pragma unroll
      for (int p = 0; p < PIECES; ++p) {
        const int c = (p * LANES + l) * E;
        if (c < C) {
          load_some<E>(x + row * C + c, there(c), v[t][p]);
          load_some<E>(dout + row * C + c, there(c), g[t][p]);
        }
      }
    }
#pragma unroll
    for (int t = 0; t < TURNS; ++t) {
      const long long row = first + t * kRows + at;
      float s1 = 0.f, s2 = 0.f;
#pragma unroll
      for (int p = 0; p < PIECES; ++p) {
        if ((p * LANES + l) * E >= C) continue;
        slopes<sizeof(T) == 2, E>(v[t][p], g[t][p], m[t], r[t], gamma != nullptr, gm[p], bt[p], act);
#pragma unroll
        for (int e = 0; e < E; ++e) {
          if (row < rows) {
            dg[p][e] = __builtin_fmaf(g[t][p][e], v[t][p][e], dg[p][e]);
            db[p][e] += g[t][p][e];
          }
          if (gamma) g[t][p][e] *= gm[p][e];
          s1 += g[t][p][e];
          s2 = __builtin_fmaf(g[t][p][e], v[t][p][e], s2);
        }
      }
      s1 = row_sum<LANES>(s1, lane, acc) * inv;
      s2 = row_sum<LANES>(s2, lane, acc) * inv;
      if (row >= rows) continue;
#pragma unroll
      for (int p = 0; p < PIECES; ++p) {
        const int c = (p * LANES + l) * E;
        if (c >= C) continue;
#pragma unroll
        for (int e = 0; e < E; ++e) g[t][p][e] = r[t] * (g[t][p][e] - s1 - v[t][p][e] * s2);
        store_some<E>(dx + row * C + c, there(c), g[t][p]);
      }
    }
  }
  if (!part) return;
  // the lane groups' sums, one piece of columns after another
#pragma unroll
  for (int which = 0; which < 2; ++which)
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
      __syncthreads();
#pragma unroll
      for (int e = 0; e < E; ++e) sums[at][l * E + e] = which ? db[p][e] : dg[p][e];
      __syncthreads();
      for (int i = threadIdx.x; i < LANES * E; i += kThreads) {
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < kRows; ++k) s += sums[k][i];
        const int c = p * LANES * E + i;
        if (c < C) part[((size_t)blockIdx.x * 2 + which) * C + c] = s;
      }
    }
}

// The sums over i < n of part[i][which][c], which = 0 into dgamma, 1 into dbeta: RUNS runs of parts beside each other, as many channels
// a workgroup as that leaves threads; the i-th workgroup of channel_blocks(C).
template <int THREADS, int RUNS>
struct ChannelSums {
  static constexpr int kChannels = THREADS / RUNS;
  static int blocks(int C) { return 2 * cdiv(C, kChannels); }
  static __device__ __forceinline__ void run(const float* __restrict__ part, int n, int C, int block, float* sums, float* __restrict__ dgamma, float* __restrict__ dbeta) {
    const int which = block & 1, c = (block >> 1) * kChannels + (int)threadIdx.x % kChannels, run = threadIdx.x / kChannels;
    const float* from = part + (size_t)which * C + std::min(c, C - 1);
    float s = 0.f;
#pragma unroll 8
    for (int i = run; i < n; i += RUNS) s += from[(size_t)i * 2 * C];
    sums[threadIdx.x] = s;
    __syncthreads();
    if (run != 0 || c >= C) return;
    s = 0.f;
#pragma unroll
    for (int k = 0; k < RUNS; ++k) s += sums[k * kChannels + threadIdx.x];
    (which ? dbeta : dgamma)[c] = s;
  }
};
using RowSums = ChannelSums<1024, 32>;    // a launch of its own
using GroupSums = ChannelSums<kThreads, 16>;  // beside the workgroups that write dx

__global__ __launch_bounds__(1024) void norm_channel_sums_kernel(const float* __restrict__ part, int n, int C, float* __restrict__ dgamma, float* __restrict__ dbeta) {
  __shared__ float sums[1024];
  RowSums::run(part, n, C, blockIdx.x, sums, dgamma, dbeta);
}

// ---------------------------------------------------------------------------------------------------------------- groups

// How an image is cut: columns are pieces of E channels.
struct Cut {
  int E;
  int group_cols;  // of a group
  int shares;      // blocks of columns that share a group, 1 where blocks hold whole groups
  int block_cols;  // columns of a block
  int block_groups;
  int blocks;      // of an image's columns
  int images;      // of a workgroup
  int lanes;       // threads over each other in a column of an image
  int rows;        // tokens of a workgroup
  int slabs;       // workgroups over an image's tokens
  int team;       // lanes that add up a group's values of a workgroup
  int join_team;  // lanes that put a group's parts together, kHeldParts each
  uint32_t cols_magic, lanes_magic, group_magic;
  __host__ __device__ int parts() const { return slabs * shares; }  // of a group
};

struct Groups {  // what the kernels take
  const void *x, *gamma, *beta, *dout;
  int B, N, C, G;
  Cut k;
  unsigned first;  // workgroup of the launch
  unsigned work;   // workgroups of the launch, the grid filled up to a multiple of 8
  float eps;
  int act;
  void* out;            // out, or dx
  float *mean, *rstd;   // [B,G]
  float2* group_part;   // [B][G][parts]: mean and M2, or the sums of dh and dh xhat
  float2* totals;       // [B][G]: these sums of the whole group, where a launch of its own adds them up
  float* channel_part;  // [runs][slabs][2][C]
  int run;              // images of a workgroup of the sums, one after another
  float *dgamma, *dbeta;
  int sums;  // workgroups in front of the others that add up channel_part
};

// a thread's place: column of the block, its group among all of the workgroup's, first channel; the workgroup's images and tokens
struct Place {
  int b, block, slab;  // b: the thread's image
  int b0, images;      // the workgroup's
  int col, q, im, lane_row;
  int c, group, groups, cols, group_cols;
  bool active;
  int row0, row1;
  size_t base;
  __device__ __forceinline__ Place(const Groups& a, unsigned work) {
    const Cut& k = a.k;
    const unsigned per_image = (unsigned)k.blocks * k.slabs;
    const unsigned batch = work / per_image, rest = work - batch * per_image;
    slab = rest / k.blocks;
    block = rest - slab * k.blocks;
    const int row = exact_div(threadIdx.x, k.block_cols, k.cols_magic);
    col = threadIdx.x - row * k.block_cols;
    im = exact_div(row, k.lanes, k.lanes_magic);
    lane_row = row - im * k.lanes;
    int first_col;
    if (k.shares > 1) {  // a share of one group
      group = block / k.shares;
      const int share = block - group * k.shares;
      first_col = group * k.group_cols + share * k.block_cols;
      cols = std::min(k.block_cols, k.group_cols - share * k.block_cols);
      groups = 1;
      group_cols = cols;
    } else {
      group = block * k.block_groups;
      first_col = group * k.group_cols;
      groups = std::min(k.block_groups, a.G - group);
      cols = groups * k.group_cols;
      group_cols = k.group_cols;
    }
    c = (first_col + (col < cols ? col : 0)) * k.E;
    row0 = slab * k.rows;
    row1 = row0 + std::min(k.rows, a.N - row0);  // (row0 + k.rows may be beyond 31 bits)
    take(a, batch);
  }
  // the images of the batch-th workgroup of a block and slab
  __device__ __forceinline__ void take(const Groups& a, unsigned batch) {
    const Cut& k = a.k;
    b0 = batch * k.images;
    images = std::min(k.images, a.B - b0);
    active = im < images && col < cols;
    b = b0 + (active ? im : 0);
    q = active ? im * groups + (k.shares > 1 ? 0 : exact_div(col, k.group_cols, k.group_magic)) : 0;
    base = (size_t)b * a.N * a.C + c;
  }
  __device__ __forceinline__ int sets() const { return images * groups; }
  // the q-th of the workgroup's groups among all
  __device__ __forceinline__ size_t set(const Groups& a, int q) const {
    const int im = a.k.images > 1 ? q / groups : 0;
    return (size_t)(b0 + im) * a.G + group + q - im * groups;
  }
  __device__ __forceinline__ int part(const Groups& a) const { return a.k.shares > 1 ? slab * a.k.shares + block % a.k.shares : slab; }
};

__device__ __forceinline__ void add(float& s, float v) { s += v; }
__device__ __forceinline__ void add(float2& s, float2 v) {
  s.x += v.x;
  s.y += v.y;
}
// the sum over `width` lanes (a power of two) next to each other, received by all of them
__device__ __forceinline__ float sum_over(float v, int width) {
  for (int o = width >> 1; o > 0; o >>= 1) v += __shfl_xor(v, o);
  return v;
}
__device__ __forceinline__ float2 sum_over(float2 v, int width) { return make_float2(sum_over(v.x, width), sum_over(v.y, width)); }

// f(group of the workgroup's, lane in its team) for all groups, by teams of `width` lanes; teams without one repeat the last (`there` false).
// (By whole waves one group after another waited for LDS or memory once per group: 8 us of the 14 that 32 groups took.)
template <typename F>
__device__ __forceinline__ void for_groups(int groups, int width, F f) {
  const int teams = kThreads / width, team = threadIdx.x / width, l = threadIdx.x & (width - 1);
  for (int first = 0; first < groups; first += teams) f(std::min(first + team, groups - 1), l, first + team < groups);
}

// per group of the workgroup's, the sums over its threads of v (a value or two): result[q], read by all threads afterwards
template <typename V>
__device__ __forceinline__ void group_sums(const Groups& a, const Place& w, V v, V (&values)[kThreads], V (&result)[kThreads]) {
  const Cut& k = a.k;
  __syncthreads();
  values[threadIdx.x] = v;
  __syncthreads();
  const int n = k.lanes * w.group_cols;
  const uint32_t magic = k.shares > 1 ? 0u : k.group_magic;
  for_groups(w.sets(), k.team, [&](int q, int l, bool there) {
    const int im = k.images > 1 ? q / w.groups : 0;
    const V* from = values + im * k.lanes * k.block_cols + (q - im * w.groups) * w.group_cols;
    V s = {};
    for (int i = l; i < n; i += k.team) {
      const int row = k.shares > 1 ? i / w.group_cols : exact_div(i, w.group_cols, magic);
      add(s, from[row * k.block_cols + i - row * w.group_cols]);
    }
    s = sum_over(s, k.team);
    if (l == 0 && there) result[q] = s;
  });
  __syncthreads();
}

// values of a group's part i
__device__ __forceinline__ float part_count(const Groups& a, int i) {
  const Cut& k = a.k;
  const int slab = i / k.shares, share = i - slab * k.shares;
  const int cols = k.shares > 1 ? std::min(k.block_cols, k.group_cols - share * k.block_cols) : k.group_cols;
  return (float)(std::min(k.rows, a.N - slab * k.rows)) * (float)(cols * k.E);
}
// mean and rstd of a whole group from its parts, by a team whose l-th lane this is; parts that a lane holds are read once
__device__ __forceinline__ void join_statistics(const Groups& a, size_t bg, int l, int team, float& mean, float& rstd) {
  const int parts = a.k.parts();
  const float2* from = a.group_part + bg * parts;
  const float n = (float)a.N * (float)(a.k.group_cols * a.k.E);
  float2 held[kHeldParts];
#pragma unroll
  for (int i = 0; i < kHeldParts; ++i) held[i] = l + i * team < parts ? from[l + i * team] : make_float2(0.f, 0.f);
  float s = 0.f;
  const auto each = [&](auto f) {
#pragma unroll
    for (int i = 0; i < kHeldParts; ++i) {
      const int at = l + i * team;
      if (at < parts) f(held[i], part_count(a, at));
    }
    for (int at = l + kHeldParts * team; at < parts; at += team) f(from[at], part_count(a, at));
  };
  each([&](float2 v, float count) { s += v.x * (count / n); });
  mean = sum_over(s, team);
  s = 0.f;
  each([&](float2 v, float count) { s += v.y + count * (v.x - mean) * (v.x - mean); });
  rstd = 1.f / sqrtf(sum_over(s, team) / n + a.eps);
}
__device__ __forceinline__ float2 join_sums(const Groups& a, size_t bg, int l, int team) {
  const int parts = a.k.parts();
  const float2* from = a.group_part + bg * parts;
  float2 s = make_float2(0.f, 0.f);
#pragma unroll 4
  for (int i = l; i < parts; i += team) add(s, from[i]);
  return sum_over(s, team);
}

// WHOLE: the workgroup holds all of its groups' values: statistics and output in one launch
template <typename T, int E, int V, bool WHOLE>
__global__ __launch_bounds__(kThreads) void norm_stats_kernel(Groups a) {
  __shared__ float values[kThreads], result[kThreads];
  const unsigned work = WHOLE ? xcd_contiguous_block(blockIdx.x, gridDim.x) : blockIdx.x;
  if (WHOLE && work >= a.work) return;
  const Place w(a, a.first + work);
  const Cut& k = a.k;
  float v[V][E];
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int row = w.row0 + i * k.lanes + w.lane_row;
    if (w.active && row < w.row1) {
      load_piece<E>((const T*)a.x + w.base + (size_t)row * a.C, v[i]);
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) v[i][e] = 0.f;
    }
  }
#pragma unroll
  for (int i = 0; i < V; ++i)
#pragma unroll
    for (int e = 0; e < E; ++e) s += v[i][e];
  group_sums(a, w, s, values, result);
  const float n = (float)(w.row1 - w.row0) * (float)(w.group_cols * E);
  const float mean = result[w.q] / n;
  s = 0.f;
#pragma unroll
  for (int i = 0; i < V; ++i)
    if (w.active && w.row0 + i * k.lanes + w.lane_row < w.row1) {
#pragma unroll
      for (int e = 0; e < E; ++e) s = __builtin_fmaf(v[i][e] - mean, v[i][e] - mean, s);
    }
  const float m_first = (int)threadIdx.x < w.sets() ? result[threadIdx.x] / n : 0.f;
  group_sums(a, w, s, values, result);
  const size_t set = (int)threadIdx.x < w.sets() ? w.set(a, threadIdx.x) : 0;
  if constexpr (WHOLE) {
    if ((int)threadIdx.x < w.sets()) {
      a.mean[set] = m_first;
      a.rstd[set] = 1.f / sqrtf(result[threadIdx.x] / n + a.eps);
    }
    if (!w.active) return;
    const float rstd = 1.f / sqrtf(result[w.q] / n + a.eps);
    float gm[E], bt[E];
    if (a.gamma) {
      load_piece<E>((const T*)a.gamma + w.c, gm);
      load_piece<E>((const T*)a.beta + w.c, bt);
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int row = w.row0 + i * k.lanes + w.lane_row;
      if (row >= w.row1) continue;
      normalise<sizeof(T) == 2, E>(v[i], mean, rstd, a.gamma != nullptr, gm, bt, a.act);
      store_piece<E>((T*)a.out + w.base + (size_t)row * a.C, v[i]);
    }
  } else {
    if ((int)threadIdx.x < w.sets()) a.group_part[set * k.parts() + w.part(a)] = make_float2(m_first, result[threadIdx.x]);
  }
}

// the parts of a group put together by a launch of its own, a wave a group: statistics, or with BWD the sums
template <bool BWD>
__global__ __launch_bounds__(kThreads) void norm_join_kernel(Groups a, int groups) {
  const int bg = blockIdx.x * kWaves + threadIdx.x / kWave, lane = threadIdx.x & (kWave - 1);
  if (bg >= groups) return;
  if constexpr (BWD) {
    const float2 s = join_sums(a, bg, lane, kWave);
    if (lane == 0) a.totals[bg] = s;
  } else {
    float m, r;
    join_statistics(a, bg, lane, kWave, m, r);
    if (lane == 0) {
      a.mean[bg] = m;
      a.rstd[bg] = r;
    }
  }
}

// JOIN: the workgroup puts its groups' parts together itself
template <typename T, int E, int V, bool JOIN>
__global__ __launch_bounds__(kThreads) void norm_apply_kernel(Groups a) {
  __shared__ float means[kThreads], rstds[kThreads];
  const Place w(a, a.first + blockIdx.x);
  const Cut& k = a.k;
  float v[V][E];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int row = w.row0 + i * k.lanes + w.lane_row;
    if (w.active && row < w.row1) load_piece<E>((const T*)a.x + w.base + (size_t)row * a.C, v[i]);
  }
  float gm[E], bt[E];
  if (a.gamma) {
    load_piece<E>((const T*)a.gamma + w.c, gm);
    load_piece<E>((const T*)a.beta + w.c, bt);
  }
  const size_t bg = (size_t)w.b * a.G + w.group;
  float mean, rstd;
  if constexpr (JOIN) {
    for_groups(w.groups, k.join_team, [&](int q, int l, bool there) {
      float m, r;
      join_statistics(a, bg + q, l, k.join_team, m, r);
      if (l == 0 && there) {
        means[q] = m;
        rstds[q] = r;
        if (w.slab == 0 && (k.shares == 1 || w.block % k.shares == 0)) {
          a.mean[bg + q] = m;
          a.rstd[bg + q] = r;
        }
      }
    });
    __syncthreads();
    mean = means[w.q];
    rstd = rstds[w.q];
  } else {
    mean = a.mean[bg + w.q];
    rstd = a.rstd[bg + w.q];
  }
  if (!w.active) return;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int row = w.row0 + i * k.lanes + w.lane_row;
    if (row >= w.row1) continue;
    normalise<sizeof(T) == 2, E>(v[i], mean, rstd, a.gamma != nullptr, gm, bt, a.act);
    store_piece<E>((T*)a.out + w.base + (size_t)row * a.C, v[i]);
  }
}

// the workgroup's sums of dg and db of its channels, into part `to` of channel_part
template <int E>
__device__ __forceinline__ void channel_sums(const Groups& a, const Place& w, const float (&dg)[E], const float (&db)[E], float2 (&sums)[kThreads * E], size_t to) {
  const Cut& k = a.k;
  const int c0 = w.c - (w.col < w.cols ? w.col : 0) * E;  // the block's first channel
#pragma unroll
  for (int e = 0; e < E; ++e) sums[threadIdx.x * E + e] = make_float2(dg[e], db[e]);
  __syncthreads();
  float* part = a.channel_part + to * 2 * a.C + c0;
  for (int i = threadIdx.x; i < w.cols * E; i += kThreads) {
    float2 t = make_float2(0.f, 0.f);
    for (int j = 0; j < k.images * k.lanes; ++j) add(t, sums[j * k.block_cols * E + i]);
    part[i] = t.x;
    part[a.C + i] = t.y;
  }
}

// Groups that one workgroup holds: their sums and dx in one launch, from one reading, further images in further turns; channel_part
// [workgroups of a block][2][C].
template <typename T, int E, int V>
__global__ __launch_bounds__(kThreads) void norm_bwd_whole_kernel(Groups a, int batches) {
  __shared__ float2 values[kThreads], result[kThreads];
  __shared__ float2 sums[kThreads * E];
  const unsigned work = xcd_contiguous_block(blockIdx.x, gridDim.x);
  if (work >= a.work) return;
  Place w(a, work);
  const Cut& k = a.k;
  const unsigned first = work / k.blocks, all = a.work / k.blocks;
  float gm[E], bt[E], dg[E], db[E];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    gm[e] = 1.f;
    bt[e] = dg[e] = db[e] = 0.f;
  }
  if (a.gamma) {
    load_piece<E>((const T*)a.gamma + w.c, gm);
    load_piece<E>((const T*)a.beta + w.c, bt);
  }
  const float inv = 1.f / ((float)a.N * (float)(k.group_cols * E));
  for (unsigned batch = first; batch < (unsigned)batches; batch += all) {
    w.take(a, batch);
    float x[V][E], g[V][E];
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int row = i * k.lanes + w.lane_row;
      if (w.active && row < a.N) {
        load_piece<E>((const T*)a.x + w.base + (size_t)row * a.C, x[i]);
        load_piece<E>((const T*)a.dout + w.base + (size_t)row * a.C, g[i]);
      }
    }
    const size_t set = w.set(a, w.q);
    const float mean = a.mean[set], rstd = a.rstd[set];
    float2 s = make_float2(0.f, 0.f);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      if (!w.active || i * k.lanes + w.lane_row >= a.N) continue;
      slopes<sizeof(T) == 2, E>(x[i], g[i], mean, rstd, a.gamma != nullptr, gm, bt, a.act);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        dg[e] = __builtin_fmaf(g[i][e], x[i][e], dg[e]);
        db[e] += g[i][e];
        g[i][e] *= gm[e];
        s.x += g[i][e];
        s.y = __builtin_fmaf(g[i][e], x[i][e], s.y);
      }
    }
    group_sums(a, w, s, values, result);
    const float s1 = result[w.q].x * inv, s2 = result[w.q].y * inv;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int row = i * k.lanes + w.lane_row;
      if (!w.active || row >= a.N) continue;
#pragma unroll
      for (int e = 0; e < E; ++e) g[i][e] = rstd * (g[i][e] - s1 - x[i][e] * s2);
      store_piece<E>((T*)a.out + w.base + (size_t)row * a.C, g[i]);
    }
  }
  if (a.channel_part) channel_sums<E>(a, w, dg, db, sums, first);
}

// per workgroup: the sums of dz xhat and dz of its channels over a run of images, and per image those of dh xhat and dh of its groups.
// RUN: the run may be longer than an image.  (One kernel for both would hold twice the sums: 16 x 4096 x 384, one group, bf16: 58.6 us backward
// instead of 53.3.)
template <typename T, int E, bool RUN>
__global__ __launch_bounds__(kThreads) void norm_bwd_sums_kernel(Groups a) {
  __shared__ float2 values[kThreads], result[kThreads];
  __shared__ float2 sums[kThreads * E];
  constexpr int kAhead = RUN ? 1 : 4;  // tokens on their way (runs are of short images: 16384 x 8200 in bf16 601 us, with four 818)
  Place w(a, a.first + blockIdx.x);
  const Cut& k = a.k;
  const int run = w.b0, first = RUN ? run * a.run : run, last = RUN ? std::min(a.B, first + a.run) : run + 1;  // (the launch counts runs in the place of images)
  float gm[E], bt[E], dg[E], db[E];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    gm[e] = 1.f;
    bt[e] = dg[e] = db[e] = 0.f;
  }
  if (a.gamma) {
    load_piece<E>((const T*)a.gamma + w.c, gm);
    load_piece<E>((const T*)a.beta + w.c, bt);
  }
  for (int image = first; image < last; ++image) {
    if constexpr (RUN) w.take(a, image);
    const size_t bg = (size_t)image * a.G + w.group;
    const float mean = a.mean[bg + w.q], rstd = a.rstd[bg + w.q];
    float own[2][E] = {};  // of the image
    float(&ig)[E] = RUN ? own[0] : dg, (&ib)[E] = RUN ? own[1] : db;
    if (w.active) {
#pragma unroll kAhead
      for (int row = w.row0 + w.lane_row; row < w.row1; row += k.lanes) {
        float x[E], g[E];
        load_piece<E>((const T*)a.x + w.base + (size_t)row * a.C, x);
        load_piece<E>((const T*)a.dout + w.base + (size_t)row * a.C, g);
        slopes<sizeof(T) == 2, E>(x, g, mean, rstd, a.gamma != nullptr, gm, bt, a.act);
#pragma unroll
        for (int e = 0; e < E; ++e) {
          ig[e] = __builtin_fmaf(g[e], x[e], ig[e]);
          ib[e] += g[e];
        }
      }
    }
    float2 s = make_float2(0.f, 0.f);
#pragma unroll
    for (int e = 0; e < E; ++e) {
      s.x = __builtin_fmaf(gm[e], ib[e], s.x);
      s.y = __builtin_fmaf(gm[e], ig[e], s.y);
      if constexpr (RUN) {
        dg[e] += ig[e];
        db[e] += ib[e];
      }
    }
    group_sums(a, w, s, values, result);
    if ((int)threadIdx.x < w.groups) a.group_part[(bg + threadIdx.x) * k.parts() + w.part(a)] = result[threadIdx.x];
  }
  if (a.channel_part) channel_sums<E>(a, w, dg, db, sums, (size_t)run * k.slabs + w.slab);
}

template <typename T, int E, int V, bool JOIN>
__global__ __launch_bounds__(kThreads) void norm_bwd_apply_kernel(Groups a, Cut parts_cut, int channel_parts) {
  __shared__ float2 totals[kThreads];
  if ((int)blockIdx.x < a.sums) return GroupSums::run(a.channel_part, channel_parts, a.C, blockIdx.x, &totals[0].x, a.dgamma, a.dbeta);
  const Place w(a, a.first + blockIdx.x - a.sums);
  const Cut& k = a.k;
  const size_t bg = (size_t)w.b * a.G + w.group;
  float x[V][E], g[V][E];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int row = w.row0 + i * k.lanes + w.lane_row;
    if (w.active && row < w.row1) {
      load_piece<E>((const T*)a.x + w.base + (size_t)row * a.C, x[i]);
      load_piece<E>((const T*)a.dout + w.base + (size_t)row * a.C, g[i]);
    }
  }
  const float mean = a.mean[bg + w.q], rstd = a.rstd[bg + w.q];
  float gm[E], bt[E];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    gm[e] = 1.f;
    bt[e] = 0.f;
  }
  if (a.gamma) {
    load_piece<E>((const T*)a.gamma + w.c, gm);
    load_piece<E>((const T*)a.beta + w.c, bt);
  }
  const float inv = 1.f / ((float)a.N * (float)(k.group_cols * E));
  float2 s;
  if constexpr (JOIN) {
    Groups p = a;
    p.k = parts_cut;
    for_groups(w.groups, parts_cut.join_team, [&](int q, int l, bool there) {
      const float2 t = join_sums(p, bg + q, l, parts_cut.join_team);
      if (l == 0 && there) totals[q] = t;
    });
    __syncthreads();
    s = totals[w.q];
  } else {
    s = a.totals[bg + w.q];
  }
  if (!w.active) return;
  const float s1 = s.x * inv, s2 = s.y * inv;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const int row = w.row0 + i * k.lanes + w.lane_row;
    if (row >= w.row1) continue;
    slopes<sizeof(T) == 2, E>(x[i], g[i], mean, rstd, a.gamma != nullptr, gm, bt, a.act);
#pragma unroll
    for (int e = 0; e < E; ++e) g[i][e] = rstd * (g[i][e] * gm[e] - s1 - x[i][e] * s2);
    store_piece<E>((T*)a.out + w.base + (size_t)row * a.C, g[i]);
  }
}

// ------------------------------------------------------------------------------------------------------------------ host

constexpr int kHeld = 64;      // values of a thread that holds its run of tokens in registers
constexpr int kHeldFew = 16;   // ... where that leaves fewer than kFullGrid workgroups
constexpr long long kFullGrid = 512;
constexpr int kJoinParts = 256;  // more parts of a group than this are put together by a launch of its own

int power_of_two(int n) {  // at least n, at most a wave
  int p = 1;
  while (p < n && p < kWave) p *= 2;
  return p;
}
void cut_images(Cut& k, int images, int lanes) {
  k.images = images;
  k.lanes = lanes;
  k.lanes_magic = div_magic(lanes);
  k.team = power_of_two(lanes * (k.block_cols / k.block_groups));
}
// blocks of at most `most` groups, or shares of one
Cut cut_columns(int C, int G, int E, int most = kThreads) {
  Cut k = {};
  k.E = E;
  k.group_cols = C / G / E;
  if (k.group_cols > kThreads) {
    k.shares = cdiv(k.group_cols, kThreads);
    k.block_cols = cdiv(k.group_cols, k.shares);
    k.shares = cdiv(k.group_cols, k.block_cols);
    k.block_groups = 1;
    k.blocks = G * k.shares;
  } else {
    k.shares = 1;
    k.blocks = cdiv(G, std::min(most, kThreads / k.group_cols));
    k.block_groups = cdiv(G, k.blocks);
    k.blocks = cdiv(G, k.block_groups);
    k.block_cols = k.block_groups * k.group_cols;
  }
  k.cols_magic = div_magic(k.block_cols);
  k.group_magic = div_magic(k.group_cols);
  cut_images(k, 1, kThreads / k.block_cols);
  return k;
}
void cut_rows(Cut& k, int N, long long rows) {
  k.rows = (int)std::min<long long>(rows, N);
  k.slabs = cdiv(N, k.rows);
  k.join_team = power_of_two(cdiv(k.parts(), kHeldParts));
}
// Groups that fit a workgroup whose threads hold V pieces each: one launch instead of two (64 x 49 x 768 in 32 groups, bf16: 7.9 us instead
// of 20.8).  As many of them as fit, fewer where that leaves CUs without a workgroup, but no less than 128 bytes of a token's row:
// 64 x 1024 x 256 in 32 groups, bf16, 32 bytes a workgroup, takes 31.6 us.  Then as many images as fit, with the same proviso; with
// `several`, narrower blocks until there are four of them (32768 x 1 x 768 in 12 groups, fp32: 70 us instead of 148).
bool cut_whole(int B, int N, int C, int G, int E, int el, int V, Cut* k, bool several = false) {
  const long long cols = C / G / E, lanes = cdiv(N, V);  // of a group, of an image
  if (cols > kThreads || lanes * cols > kThreads) return false;
  const int least = (int)std::min<long long>(G, cdiv(128 / (E * el), cols));
  int most = (int)std::min<long long>(G, kThreads / (lanes * cols));
  if (most < least) return false;
  const auto images_of = [&](int groups) { return std::min<long long>(kThreads / (groups * cols) / lanes, (long long)B * cdiv(G, groups) / kFullGrid); };
  const auto fewer = [&] { return most = std::max(least, (most + 1) / 2); };
  while (most > least && (long long)B * cdiv(G, most) < kFullGrid) fewer();
  while (several && most > least && images_of(most) < 4 && (long long)B * cdiv(G, most) >= 2 * kFullGrid) fewer();
  *k = cut_columns(C, G, E, most);
  const long long images = images_of(k->block_groups);
  if (images > 1) cut_images(*k, (int)images, k->lanes / (int)images);
  cut_rows(*k, N, N);
  return true;
}
// Threads hold `held` values each: few where images have fewer tokens than a thread would hold pieces (4096 x 16 x 256 in 32 groups, bf16:
// 19.3 us with few, 15.4 so; 131072 x 1 x 64 in 4 groups, fp32: 24.5 with few).
Cut cut_held(int B, int N, int C, int G, int E, int el, int* held) {
  Cut k;
  *held = kHeldFew;
  if (N < kHeld / E && cut_whole(B, N, C, G, E, el, kHeldFew / E, &k, true) && k.images > 1) return k;
  *held = kHeld;
  if (cut_whole(B, N, C, G, E, el, kHeld / E, &k)) return k;
  k = cut_columns(C, G, E);
  for (int h : {kHeld, kHeldFew}) {
    *held = h;
    cut_rows(k, N, (long long)h / E * k.lanes);
    if ((long long)B * k.blocks * k.slabs >= kFullGrid) break;
  }
  return k;
}
// Backward of groups that fit a workgroup: few values a thread where that takes several images (131072 x 1 x 64 in 4 groups, bf16: 19 us, with
// kHeldBwd 26).  Single values are read twice instead, unless several images fit: 2048 x 49 x 765 in 15 groups, bf16, 459 us against 691.
constexpr int kHeldBwd = 32;  // values of x, and of dout
bool cut_bwd_whole(int B, int N, int C, int G, int E, int el, Cut* k, int* held, int* batches, int* workgroups) {
  *held = kHeldFew;
  if (!(cut_whole(B, N, C, G, E, el, kHeldFew / E, k, true) && k->images > 1)) {
    *held = kHeldBwd;
    if (!cut_whole(B, N, C, G, E, el, kHeldBwd / E, k)) return false;
    if (E == 1 && k->images == 1) return false;
  }
  *batches = cdiv(B, k->images);
  // (of a block: as many as are on the chip at a time, by the registers that the kernel takes; 2048 x 49 x 768 in 32 groups, bf16: 156 us,
  // with 1024 workgroups 209)
  *workgroups = std::min(*batches, std::max(1, (*held == kHeldFew ? 1024 : 768) / k->blocks));
  return true;
}
// for sums: about 1024 workgroups, of at least four turns
Cut cut_sums(int B, int N, int C, int G, int E) {
  Cut k = cut_columns(C, G, E);
  const long long slabs = std::max(1ll, 1024 / ((long long)B * k.blocks));
  cut_rows(k, N, std::max<long long>(4 * k.lanes, cdiv(N, slabs)));
  return k;
}
// Images of a workgroup of the sums.  A workgroup leaves sums of its channels, 8 bytes a channel, written and read once: at most 2048 of them, however many
// images there are, and where images are short as many together as make that a quarter of what is read of x and dout, if it leaves 1024
// workgroups.  (Layer norm of 65536 x 4100 in fp32, one row a workgroup: 2714 us and 2.15 GB of workspace; so 1490 us and 70 MB.)  Beside images of 64
// bytes a channel and more they are little: at most 8192 of them (2500 x 400 x 256, one group, bf16: 528 us with one image a workgroup, 556 with two).
int run_of(int B, int N, const Cut& k, int el) {
  const long long image = (long long)el * N, together = std::min<long long>(cdiv(16, image), (long long)B * k.blocks / 1024);
  return (int)std::max<long long>(cdiv(B, image < 64 ? 2048 : 8192), k.slabs > 1 ? 1 : together);
}

// Rows that the row kernels hold: at most 4 pieces a lane, by a wave as long as that is enough, else by the workgroup.
constexpr int kMostPieces = 4;
bool rows_fit(int N, int C, int G, int E) { return N == 1 && G == 1 && cdiv(C, E) <= kThreads * kMostPieces; }
int row_lanes(int pieces) {
  if (pieces > kWave * kMostPieces) return kThreads;
  int lanes = 4;
  while (lanes < kWave && lanes < pieces) lanes *= 2;
  return lanes;
}
int rows_bwd_blocks(int rows) { return std::min(cdiv(rows, 16), 1024); }

// f(lanes, pieces, whether rows end inside a piece)
template <typename F>
hipError_t for_row_shape(int C, int E, F f) {
  const int all = cdiv(C, E), lanes = row_lanes(all), pieces = cdiv(all, lanes);
  const auto shape = [&](auto lanes_, auto pieces_) { return C % E ? f(lanes_, pieces_, std::true_type()) : f(lanes_, pieces_, std::false_type()); };
  using std::integral_constant;
  if (lanes == 4) return shape(integral_constant<int, 4>(), integral_constant<int, 1>());
  if (lanes == 8) return shape(integral_constant<int, 8>(), integral_constant<int, 1>());
  if (lanes == 16) return shape(integral_constant<int, 16>(), integral_constant<int, 1>());
  if (lanes == 32) return shape(integral_constant<int, 32>(), integral_constant<int, 1>());
  if (lanes == kThreads) return pieces <= 2 ? shape(integral_constant<int, kThreads>(), integral_constant<int, 2>()) : shape(integral_constant<int, kThreads>(), integral_constant<int, 4>());
  if (pieces == 1) return shape(integral_constant<int, 64>(), integral_constant<int, 1>());
  if (pieces == 2) return shape(integral_constant<int, 64>(), integral_constant<int, 2>());
  return shape(integral_constant<int, 64>(), integral_constant<int, 4>());
}

template <typename T>
hipError_t rows_fwd(const NormArgs& a, hipStream_t stream) {
  return for_row_shape(a.C, kPiece<T>, [&](auto lanes, auto pieces, auto tail) {
    constexpr int L = lanes, P = pieces;
    const unsigned grid = (unsigned)std::min(cdiv(a.B, kThreads / L), 8192);
    AFFMAE_LAUNCH("norm_rows_fwd_kernel", stream, (norm_rows_fwd_kernel<T, L, P, tail>), dim3(grid), dim3(kThreads), 0, stream, (const T*)a.x, (const T*)a.gamma,
                  (const T*)a.beta, a.B, a.C, a.eps, a.act, (T*)a.out, a.mean, a.rstd);
    return hipGetLastError();
  });
}
template <typename T>
hipError_t rows_bwd(const NormArgs& a, hipStream_t stream) {
  const int blocks = rows_bwd_blocks(a.B);
  float* part = a.dgamma ? static_cast<float*>(a.workspace) : nullptr;
  const hipError_t rc = for_row_shape(a.C, kPiece<T>, [&](auto lanes, auto pieces, auto tail) {
    constexpr int L = lanes, P = pieces, U = P == 1 ? 2 : 1;
    AFFMAE_LAUNCH("norm_rows_bwd_kernel", stream, (norm_rows_bwd_kernel<T, L, P, U, tail>), dim3(blocks), dim3(kThreads), 0, stream, (const T*)a.x, (const T*)a.gamma,
                  (const T*)a.beta, a.mean, a.rstd, (const T*)a.dout, a.B, a.C, a.act, (T*)a.dx, part);
    return hipGetLastError();
  });
  if (rc != hipSuccess || !part) return rc;
  AFFMAE_LAUNCH("norm_channel_sums_kernel", stream, norm_channel_sums_kernel, dim3(RowSums::blocks(a.C)), dim3(1024), 0, stream, part, blocks, a.C, a.dgamma, a.dbeta);
  return hipGetLastError();
}

Groups groups_of(const NormArgs& a, const Cut& k) {
  Groups g = {};
  g.x = a.x; g.gamma = a.gamma; g.beta = a.beta; g.dout = a.dout;
  g.B = a.B; g.N = a.N; g.C = a.C; g.G = a.G; g.k = k; g.eps = a.eps; g.act = a.act;
  g.mean = a.mean; g.rstd = a.rstd;
  return g;
}

dim3 eights(unsigned n) { return dim3((n + 7) / 8 * 8); }
// f(workgroups) for all of a cut's, in launches of as many as the runtime takes, g.sums more beside them
template <typename F>
void for_workgroups(Groups& g, int B, F f) {
  const long long all = (long long)cdiv(B, g.k.images) * g.k.blocks * g.k.slabs;
  for (long long first = 0; first < all;) {
    const long long n = std::min(all - first, kMaxBlocks - g.sums);
    g.first = (unsigned)first;
    g.work = (unsigned)n;
    f(dim3((unsigned)n));
    first += n;
  }
}

template <typename T, int E>
hipError_t groups_fwd(const NormArgs& a, hipStream_t stream) {
  int held;
  const Cut k = cut_held(a.B, a.N, a.C, a.G, E, sizeof(T), &held);
  Groups g = groups_of(a, k);
  g.out = a.out;
  g.group_part = static_cast<float2*>(a.workspace);
  const dim3 threads(kThreads);
  const auto run = [&](auto values) {
    constexpr int V = decltype(values)::value / E;
    const auto all = [&](const char* name, auto kernel) {
      (void)name;
      for_workgroups(g, a.B, [&](dim3 grid) { AFFMAE_LAUNCH(name, stream, kernel, grid, threads, 0, stream, g); });
    };
    if (k.parts() == 1)
      return for_workgroups(g, a.B, [&](dim3 grid) {
        AFFMAE_LAUNCH("norm_stats_kernel", stream, (norm_stats_kernel<T, E, V, true>), eights(grid.x), threads, 0, stream, g);
      });
    all("norm_stats_kernel", norm_stats_kernel<T, E, V, false>);
    if (k.parts() <= kJoinParts) return all("norm_apply_kernel", norm_apply_kernel<T, E, V, true>);
    AFFMAE_LAUNCH("norm_join_kernel", stream, norm_join_kernel<false>, dim3(cdiv((long long)a.B * a.G, kWaves)), threads, 0, stream, g, a.B * a.G);
    all("norm_apply_kernel", norm_apply_kernel<T, E, V, false>);
  };
  if (held == kHeld)
    run(std::integral_constant<int, kHeld>());
  else
    run(std::integral_constant<int, kHeldFew>());
  return hipGetLastError();
}

struct BwdSpace {
  size_t totals, channels, all;
};
BwdSpace bwd_space(int B, int C, int G, const Cut& k, int run) {
  BwdSpace s;
  s.totals = up256((size_t)B * G * k.parts() * sizeof(float2));
  s.channels = s.totals + up256((size_t)B * G * sizeof(float2));
  s.all = s.channels + (size_t)cdiv(B, run) * k.slabs * 2 * C * sizeof(float);
  return s;
}

template <typename T, int E>
hipError_t groups_bwd(const NormArgs& a, hipStream_t stream) {
  Cut whole;
  int held, batches, workgroups;
  if (cut_bwd_whole(a.B, a.N, a.C, a.G, E, sizeof(T), &whole, &held, &batches, &workgroups)) {
    Groups g = groups_of(a, whole);
    g.out = a.dx;
    g.channel_part = a.dgamma ? static_cast<float*>(a.workspace) : nullptr;
    g.work = (unsigned)workgroups * whole.blocks;
    const auto kernel = held == kHeldFew ? norm_bwd_whole_kernel<T, E, kHeldFew / E> : norm_bwd_whole_kernel<T, E, kHeldBwd / E>;
    AFFMAE_LAUNCH("norm_bwd_whole_kernel", stream, kernel, eights(g.work), dim3(kThreads), 0, stream, g, batches);
    if (a.dgamma)
      AFFMAE_LAUNCH("norm_channel_sums_kernel", stream, norm_channel_sums_kernel, dim3(RowSums::blocks(a.C)), dim3(1024), 0, stream, g.channel_part, workgroups, a.C, a.dgamma,
                    a.dbeta);
    return hipGetLastError();
  }
  const Cut sums = cut_sums(a.B, a.N, a.C, a.G, E);
  const int run = run_of(a.B, a.N, sums, sizeof(T)), runs = cdiv(a.B, run);
  const BwdSpace at = bwd_space(a.B, a.C, a.G, sums, run);
  char* ws = static_cast<char*>(a.workspace);
  Groups g = groups_of(a, sums);
  g.out = a.dx;
  g.group_part = reinterpret_cast<float2*>(ws);
  g.totals = reinterpret_cast<float2*>(ws + at.totals);
  g.channel_part = a.dgamma ? reinterpret_cast<float*>(ws + at.channels) : nullptr;
  g.run = run;
  const dim3 threads(kThreads);
  const auto sums_kernel = run > 1 ? norm_bwd_sums_kernel<T, E, true> : norm_bwd_sums_kernel<T, E, false>;
  for_workgroups(g, runs, [&](dim3 grid) { AFFMAE_LAUNCH("norm_bwd_sums_kernel", stream, sums_kernel, grid, threads, 0, stream, g); });
  const bool join = sums.parts() <= kJoinParts;
  if (!join) AFFMAE_LAUNCH("norm_join_kernel", stream, norm_join_kernel<true>, dim3(cdiv((long long)a.B * a.G, kWaves)), threads, 0, stream, g, a.B * a.G);
  constexpr int V = kHeldBwd / E;
  Cut k = cut_columns(a.C, a.G, E);
  cut_rows(k, a.N, (long long)V * k.lanes);
  g.k = k;
  const auto kernel = join ? norm_bwd_apply_kernel<T, E, V, true> : norm_bwd_apply_kernel<T, E, V, false>;
  g.dgamma = a.dgamma;
  g.dbeta = a.dbeta;
  g.sums = a.dgamma ? GroupSums::blocks(a.C) : 0;
  for_workgroups(g, a.B, [&](dim3 grid) {
    AFFMAE_LAUNCH("norm_bwd_apply_kernel", stream, kernel, dim3(grid.x + g.sums), threads, 0, stream, g, sums, runs * sums.slabs);
    g.sums = 0;
  });
  return hipGetLastError();
}

// What the group kernels move at a time: 16 bytes, or less where a group ends inside that, down to single values (2048 x 49 x 768
// in 32, 64 and 128 groups, bf16, pieces of 16, 8 and 4 bytes: 88, 117 and 213 us, 159, 183 and 280 backward; x 765 in 15, single values:
// 399 and 458).
int group_piece(int C, int G, int dtype) {
  int E = dtype == 1 ? 8 : 4;
  while (C / G % E) E /= 2;
  return E;
}
// f(values of a piece)
template <typename T, typename F>
hipError_t for_group_piece(const NormArgs& a, F f) {
  using std::integral_constant;
  const int E = group_piece(a.C, a.G, a.dtype);
  if constexpr (sizeof(T) == 2) {
    if (E == 8) return f(integral_constant<int, 8>());
  }
  return E == 4 ? f(integral_constant<int, 4>()) : E == 2 ? f(integral_constant<int, 2>()) : f(integral_constant<int, 1>());
}
template <typename T>
hipError_t fwd(const NormArgs& a, hipStream_t stream) {
  if (rows_fit(a.N, a.C, a.G, kPiece<T>)) return rows_fwd<T>(a, stream);
  return for_group_piece<T>(a, [&](auto piece) { return groups_fwd<T, decltype(piece)::value>(a, stream); });
}
template <typename T>
hipError_t bwd(const NormArgs& a, hipStream_t stream) {
  if (rows_fit(a.N, a.C, a.G, kPiece<T>)) return rows_bwd<T>(a, stream);
  return for_group_piece<T>(a, [&](auto piece) { return groups_bwd<T, decltype(piece)::value>(a, stream); });
}

}  // namespace

size_t norm_fwd_workspace_bytes(int B, int N, int C, int G, int dtype) {
  if (rows_fit(N, C, G, dtype == 1 ? 8 : 4)) return 0;
  int held;
  const Cut k = cut_held(B, N, C, G, group_piece(C, G, dtype), dtype == 1 ? 2 : 4, &held);
  return k.parts() > 1 ? (size_t)B * G * k.parts() * sizeof(float2) : 0;
}
size_t norm_bwd_workspace_bytes(int B, int N, int C, int G, int dtype) {
  if (rows_fit(N, C, G, dtype == 1 ? 8 : 4)) return (size_t)rows_bwd_blocks(B) * 2 * C * sizeof(float);
  const int E = group_piece(C, G, dtype);
  Cut whole;
  int held, batches, workgroups;
  if (cut_bwd_whole(B, N, C, G, E, dtype == 1 ? 2 : 4, &whole, &held, &batches, &workgroups)) return (size_t)workgroups * 2 * C * sizeof(float);
  const Cut sums = cut_sums(B, N, C, G, E);
  return bwd_space(B, C, G, sums, run_of(B, N, sums, dtype == 1 ? 2 : 4)).all;
}
hipError_t launch_norm_fwd(const NormArgs& a, hipStream_t stream) { return a.dtype == 1 ? fwd<bf16_t>(a, stream) : fwd<float>(a, stream); }
hipError_t launch_norm_bwd(const NormArgs& a, hipStream_t stream) { return a.dtype == 1 ? bwd<bf16_t>(a, stream) : bwd<float>(a, stream); }

}  // namespace affmae
