// Attention between all tokens, backward.  With p = exp(z - lse) worked out again and g = dout, per image and head (attn_fwd.hip has z):
//     dP_ij = <g_i, v_j>,  D_i = <g_i, out_i>,  dZ_ij = p_ij (dP_ij - D_i),  dS_ij = dZ_ij (1 - tanh^2),
//     dq_i = scale sum_j dS_ij k_j,  dk_j = scale sum_i dS_ij q_i,  dv_j = sum_i p_ij g_i,  dslope_h = -sum_ij dZ_ij |x_i - y_j|.
// Two kernels, one that keeps queries and lets keys come by (dq, D, dslope) and one the other way round (dk, dv): seven products of
// two of a pair's vectors instead of five, and nothing is added up by atomics: the results are the same in every run, and grouped
// heads' gradients add up in registers.
#include "attn_common.h"
#include "timing.h"

#include <algorithm>

namespace affmae {
namespace {

template <typename T, int D, bool TERMS>
__global__ __launch_bounds__(kAttnThreads, 2) void attn_bwd_query_kernel(AttnParams p) {
  using R = TileRows<T, D>;
  constexpr int BN = R::BN;
  extern __shared__ __align__(16) char lds[];
  __shared__ KeyNotes<BN> notes[2];
  const int work = xcd_contiguous_block(blockIdx.x, gridDim.x);
  if (work >= p.work) return;
  const int group = exact_div(work, p.blocks, p.blocks_magic), block = work - group * p.blocks;
  const int split = group / (p.B * p.Hk), bh = group - split * p.B * p.Hk, b = bh / p.Hk, hk = bh - b * p.Hk;
  const int lane = threadIdx.x & 63, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int block0 = block * kAttnRows, r0 = block0 + wave * 32;
  const bool busy = r0 < p.rows;
  const Row own = own_row(p, b, hk, r0);
  const Source<T, D, true> keys(p, p.k, b, hk), values(p, p.v, b, hk);
  Fixed<T, D> q, g;
  q.load((const char*)p.q + own.at * p.d * R::E, half, p.d * R::E, own.there);
  g.load((const char*)p.dout + own.at * p.d * R::E, half, p.d * R::E, own.there);
  float sum = 0.f;  // D
#pragma unroll
  for (int s = 0; s < R::kSteps; ++s) {
    const int at = (2 * s + half) * 16;
    Piece<T> o;
    o.zero();
    if (own.there && at < p.d * R::E) __builtin_memcpy(&o, (const char*)p.out + own.at * p.d * R::E + at, 16);
    sum += Piece<T>::dot(g.x[s], o);
    if (p.negate) q.x[s].negate();
  }
  sum = other_half_sum(sum);
  if (own.there && half == 0 && split == 0) p.rowsum[own.at] = sum;
  const float seen = own.there ? p.lse[own.at] : 0.f;
  const float lse = seen == -__builtin_inff() ? __builtin_inff() : seen * kLog2e;  // (no key: every p is 0)
  const bool capped = TERMS && p.cap > 0.f;
  const float factor = capped ? p.scale / p.cap : p.scale * kLog2e;

  const int tiles = (p.Nk + BN - 1) / BN;
  Walk walk;
  walk.spans = nullptr;
  walk.mixed = false;
  walk.end = min(tiles, (split + 1) * p.split_tiles);
  walk.tile_rows = BN; walk.G = 1; walk.g_magic = 0u;
  if (p.q_doc) {
    walk.spans = p.k_span + (size_t)b * ((p.Nk + kSpan - 1) / kSpan);
    walk.own(p.q_span + (size_t)b * ((p.Nq + kSpan - 1) / kSpan), exact_div(block0, p.G, p.g_magic), exact_div(min(block0 + kAttnRows, p.rows) - 1, p.G, p.g_magic));
  }
  walk.start(split * p.split_tiles);

  const auto fetch = [&](int t, int buffer, KeyNote<BN>& note, bool& masked) __attribute__((always_inline)) {
    char* dst = lds + buffer * 2 * R::kBytes;
    bool pads = false;
    masked = t * BN + BN > p.Nk;
    if (walk.spans) {
      const Span x = walk.of(t, p.Nk);
      pads = __builtin_amdgcn_readfirstlane(x.pad);
      masked = masked || walk.mixed || pads || __builtin_amdgcn_readfirstlane(x.lo) != walk.lo || __builtin_amdgcn_readfirstlane(x.hi) != walk.lo;
    }
    keys.load(dst, t * BN, pads);
    values.load(dst + R::kBytes, t * BN, pads);
    if (masked || (TERMS && p.slope)) note.fetch(p, b, t * BN);
  };

  f32x16 dq[D / 32] = {};
  float by_distance = 0.f, rest = 0.f, distances = 0.f;  // sums of dZ |x - y|, of dZ, of p |x - y|
  KeyNote<BN> note = {};
  bool masked = false;
  int t = walk.next(p.Nk);
  if (t < walk.end) {
    fetch(t, 0, note, masked);
    note.keep(notes[0]);
  }
  for (int buffer = 0; t < walk.end; buffer ^= 1) {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    const int following = walk.next(p.Nk);
    bool next_masked = false;
    if (following < walk.end) fetch(following, buffer ^ 1, note, next_masked);
    const char* kt = lds + buffer * 2 * R::kBytes;
    const char* vt = kt + R::kBytes;
    if (busy) {
      const KeyNotes<BN>& n = notes[buffer];
#pragma unroll
      for (int kb = 0; kb < R::kBlocks; ++kb) {
        f32x16 s = row_products<T, D>(kt, kb, q, lane);
        const f32x16 dp = row_products<T, D>(vt, kb, g, lane);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int j = 32 * kb + 16 * (i >> 3) + 8 * half + (i & 7);
          if constexpr (TERMS) {
            float bend = 0.f, distance = 0.f;
            const float z = score<sizeof(T) == 4>(s[i], p, factor, own.x - n.x[j], own.y - n.y[j], own.slope, bend, distance);
            float pr = __builtin_amdgcn_exp2f(z - lse), dz = pr * (dp[i] - sum);
            if (masked && n.doc[j] != own.doc) pr = dz = 0.f;
            if (p.rowslope) {
              by_distance = __builtin_fmaf(dz, distance, by_distance);
              distances = __builtin_fmaf(pr, distance, distances);
              rest += dz;
            }
            s[i] = capped ? dz * __builtin_fmaf(-bend, bend, 1.f) : dz;
          } else {
            s[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], factor, -lse)) * (dp[i] - sum);
            if (masked && n.doc[j] != own.doc) s[i] = 0.f;
          }
        }
        column_products<D>(kt, kb, s, dq, lane, T{});
      }
    }
    if (following < walk.end) note.keep(notes[buffer ^ 1]);
    t = following;
    masked = next_masked;
  }

  if (!busy) return;
  if (TERMS && p.rowslope) {
    by_distance = other_half_sum(by_distance);
    rest = other_half_sum(rest);
    distances = other_half_sum(distances);
    if (own.there && half == 0) {
      const size_t tokens = (size_t)p.B * p.Nq, plane = (size_t)p.H * tokens;
      float* to = p.rowslope + (size_t)split * 3 * plane + (size_t)own.head * tokens + (size_t)b * p.Nq + own.i;
      const bool pad = own.doc < 0;
      to[0] = pad ? 0.f : by_distance;
      to[plane] = pad ? 0.f : rest;
      to[2 * plane] = pad ? 0.f : distances;
    }
  }
  if (!own.there) return;
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int ch = 32 * db + 8 * e + 4 * half;
      if (ch < p.d) {
        float v[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) v[c] = own.doc < 0 ? 0.f : dq[db][4 * e + c] * p.grad_scale;
        if (p.part) store_piece<4>(p.part + ((size_t)split * p.B * p.Nq * p.H + own.at) * p.d + ch, v);
        else store_piece<4>((T*)p.dq + own.at * p.d + ch, v);
      }
    }
}

// Of a tile's rows: lse in units of log 2 (infinity for rows that are not there, see no key or are padding: their p is 0) and <dout,
// out>; place, slope and image.
template <int BN>
struct RowNotes {
  float lse[BN], sum[BN], x[BN], y[BN], slope[BN];
  int doc[BN];
};
template <int BN>
struct RowNote {
  float lse, sum, x, y, slope;
  int doc;
  __device__ __forceinline__ void fetch(const AttnParams& p, int b, int hk, int r0) {
    const int r = r0 + (int)threadIdx.x;
    lse = __builtin_inff();
    sum = x = y = slope = 0.f;
    doc = -2;
    if ((int)threadIdx.x < BN && r < p.rows) {
      const int i = exact_div(r, p.G, p.g_magic), head = hk * p.G + (r - i * p.G);
      const size_t token = (size_t)b * p.Nq + i, at = token * p.H + head;
      doc = 0;
      if (p.q_doc) {
        doc = p.q_doc[token];
        if (doc < 0) doc = -2;
      }
      if (p.slope && doc >= 0) {
        const float2 xy = reinterpret_cast<const float2*>(p.q_xy)[token];
        x = xy.x;
        y = xy.y;
        slope = p.slope[head] * kLog2e;
      }
      const float seen = p.lse[at];
      if (doc >= 0 && seen != -__builtin_inff()) {
        lse = seen * kLog2e;
        sum = p.rowsum[at];
      }
    }
  }
  __device__ __forceinline__ void keep(RowNotes<BN>& n, bool terms) const {
    if ((int)threadIdx.x < BN) {
      n.lse[threadIdx.x] = lse;
      n.sum[threadIdx.x] = sum;
      n.doc[threadIdx.x] = doc;
      if (terms) {
        n.x[threadIdx.x] = x;
        n.y[threadIdx.x] = y;
        n.slope[threadIdx.x] = slope;
      }
    }
  }
};

template <typename T, int D, bool TERMS>
__global__ __launch_bounds__(kAttnThreads, D == 128 || sizeof(T) == 4 ? 1 : 2) void attn_bwd_key_kernel(AttnParams p) {
  using R = TileRows<T, D>;
  constexpr int BN = R::BN;
  extern __shared__ __align__(16) char lds[];
  __shared__ RowNotes<BN> notes[2];
  const int work = xcd_contiguous_block(blockIdx.x, gridDim.x);
  if (work >= p.work) return;
  const int group = exact_div(work, p.blocks, p.blocks_magic), block = work - group * p.blocks;
  const int split = group / (p.B * p.Hk), bh = group - split * p.B * p.Hk, b = bh / p.Hk, hk = bh - b * p.Hk;
  const int lane = threadIdx.x & 63, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int block0 = block * kAttnRows, j0 = block0 + wave * 32;
  const bool busy = j0 < p.Nk;
  const int j = min(j0 + (lane & 31), p.Nk - 1);
  const bool there = j0 + (lane & 31) < p.Nk;
  const size_t token = (size_t)b * p.Nk + j, own_at = token * p.Hk + hk;
  float own_x = 0.f, own_y = 0.f;
  if (p.slope) {
    const float2 xy = reinterpret_cast<const float2*>(p.k_xy)[token];
    own_x = xy.x;
    own_y = xy.y;
  }
  const int own_doc = p.k_doc ? max(p.k_doc[token], -1) : 0;
  const Source<T, D, false> queries(p, p.q, b, hk), douts(p, p.dout, b, hk);
  Fixed<T, D> k, v;
  k.load((const char*)p.k + own_at * p.d * R::E, half, p.d * R::E, there);
  v.load((const char*)p.v + own_at * p.d * R::E, half, p.d * R::E, there);
  if (p.negate) {
#pragma unroll
    for (int s = 0; s < R::kSteps; ++s) k.x[s].negate();
  }
  const bool capped = TERMS && p.cap > 0.f;
  const float factor = capped ? p.scale / p.cap : p.scale * kLog2e;

  const int tiles = (p.rows + BN - 1) / BN;
  Walk walk;
  walk.spans = nullptr;
  walk.mixed = false;
  walk.end = min(tiles, (split + 1) * p.split_tiles);
  walk.tile_rows = BN; walk.G = p.G; walk.g_magic = p.g_magic;
  if (p.q_doc) {
    walk.spans = p.q_span + (size_t)b * ((p.Nq + kSpan - 1) / kSpan);
    walk.own(p.k_span + (size_t)b * ((p.Nk + kSpan - 1) / kSpan), block0, min(block0 + kAttnRows, p.Nk) - 1);
  }
  walk.start(split * p.split_tiles);

  const auto fetch = [&](int t, int buffer, RowNote<BN>& note, bool& masked) __attribute__((always_inline)) {
    char* dst = lds + buffer * 2 * R::kBytes;
    bool pads = false;
    masked = false;
    if (walk.spans) {
      const Span x = walk.of(t, p.rows);
      pads = __builtin_amdgcn_readfirstlane(x.pad);
      masked = walk.mixed || pads || __builtin_amdgcn_readfirstlane(x.lo) != walk.lo || __builtin_amdgcn_readfirstlane(x.hi) != walk.lo;
    }
    queries.load(dst, t * BN, pads);
    douts.load(dst + R::kBytes, t * BN, pads);
    note.fetch(p, b, hk, t * BN);
  };

  f32x16 dk[D / 32] = {}, dv[D / 32] = {};
  RowNote<BN> note = {};
  bool masked = false;
  int t = walk.next(p.rows);
  if (t < walk.end) {
    fetch(t, 0, note, masked);
    note.keep(notes[0], TERMS);
  }
  for (int buffer = 0; t < walk.end; buffer ^= 1) {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    const int following = walk.next(p.rows);
    bool next_masked = false;
    if (following < walk.end) fetch(following, buffer ^ 1, note, next_masked);
    const char* qt = lds + buffer * 2 * R::kBytes;
    const char* gt = qt + R::kBytes;
    if (busy) {
      const RowNotes<BN>& n = notes[buffer];
#pragma unroll
      for (int rb = 0; rb < R::kBlocks; ++rb) {
        f32x16 s = row_products<T, D>(qt, rb, k, lane);
        f32x16 dp = row_products<T, D>(gt, rb, v, lane);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int r = 32 * rb + 16 * (i >> 3) + 8 * half + (i & 7);
          float pr, bend = 0.f;
          if constexpr (TERMS) {
            float distance;
            pr = __builtin_amdgcn_exp2f(score<sizeof(T) == 4>(s[i], p, factor, n.x[r] - own_x, n.y[r] - own_y, n.slope[r], bend, distance) - n.lse[r]);
          } else {
            pr = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], factor, -n.lse[r]));
          }
          float ds = pr * (dp[i] - n.sum[r]);
          if (capped) ds *= __builtin_fmaf(-bend, bend, 1.f);
          if (masked && n.doc[r] != own_doc) pr = ds = 0.f;
          s[i] = pr;
          dp[i] = ds;
        }
        column_products<D>(gt, rb, s, dv, lane, T{});
        column_products<D>(qt, rb, dp, dk, lane, T{});
      }
    }
    if (following < walk.end) note.keep(notes[buffer ^ 1], TERMS);
    t = following;
    masked = next_masked;
  }

  if (!busy || !there) return;
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int ch = 32 * db + 8 * e + 4 * half;
      if (ch < p.d) {
        float a[4], c[4];
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          a[x] = own_doc < 0 ? 0.f : dk[db][4 * e + x] * p.grad_scale;
          c[x] = own_doc < 0 ? 0.f : dv[db][4 * e + x];
        }
        if (p.part) {
          const size_t to = ((size_t)split * p.B * p.Nk * p.Hk + own_at) * p.d + ch;
          store_piece<4>(p.part + to, a);
          store_piece<4>(p.part_v + to, c);
        } else {
          store_piece<4>((T*)p.dk + own_at * p.d + ch, a);
          store_piece<4>((T*)p.dv + own_at * p.d + ch, c);
        }
      }
    }
}

// Parts of splits added up, in their order: of dq, dk and dv, a blockIdx.y each
struct Joins {
  const float* part[3];
  void* out[3];
  int splits[3];
  size_t n[3];  // values, a multiple of 4
};
template <typename T>
__global__ __launch_bounds__(256) void attn_bwd_join_kernel(Joins j) {
  const int w = blockIdx.y;
  const float* part = w == 0 ? j.part[0] : w == 1 ? j.part[1] : j.part[2];
  T* out = (T*)(w == 0 ? j.out[0] : w == 1 ? j.out[1] : j.out[2]);
  const int splits = w == 0 ? j.splits[0] : w == 1 ? j.splits[1] : j.splits[2];
  const size_t n = w == 0 ? j.n[0] : w == 1 ? j.n[1] : j.n[2];
  for (size_t at = ((size_t)blockIdx.x * 256 + threadIdx.x) * 4; at < n; at += (size_t)gridDim.x * 1024) {
    float v[4] = {};
    for (int s = 0; s < splits; ++s) {
      float x[4];
      load_piece<4>(part + s * n + at, x);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] += x[e];
    }
    store_piece<4>(out + at, v);
  }
}

// dslope of a head, from every row's sums of dZ |x - y|, dZ and p |x - y|.  The kernel's D comes from the rounded output: where the exact
// one is D + e, the sum of the row's dZ is e, and its share of dslope lacks e times the sum of p |x - y|.
__global__ __launch_bounds__(1024) void attn_bwd_slope_kernel(const float* rows, int splits, int H, size_t tokens, float* dslope) {
  __shared__ float acc[16];
  const size_t plane = (size_t)H * tokens;
  const float* at = rows + (size_t)blockIdx.x * tokens;
  float total = 0.f;
  for (size_t i = threadIdx.x; i < tokens; i += 1024) {
    float a = 0.f, e = 0.f, c = 0.f;
    for (int s = 0; s < splits; ++s) {
      const float* x = at + (size_t)s * 3 * plane + i;
      a += x[0];
      e += x[plane];
      c += x[2 * plane];
    }
    total -= __builtin_fmaf(-e, c, a);
  }
  total = wave_sum(total);
  if ((threadIdx.x & 63) == 0) acc[threadIdx.x / kWave] = total;
  __syncthreads();
  if (threadIdx.x == 0) {
    float s = 0.f;
    for (int w = 0; w < 16; ++w) s += acc[w];
    dslope[blockIdx.x] = s;
  }
}

// Splits of the side that comes by: where the other one alone does not fill the chip, as many as do, of at least kLeast rows.
constexpr int kLeast = 256;
struct Side {
  int blocks, splits, split_tiles;
};
Side side(long long own, long long other, long long groups, int D, int el) {
  const int BN = D * el > 256 ? 32 : 64;
  Side s;
  s.blocks = (int)((own + kAttnRows - 1) / kAttnRows);
  const int tiles = (int)((other + BN - 1) / BN);
  groups *= s.blocks;
  const long long want = std::min<long long>((512 + groups - 1) / groups, std::max<long long>(1, other / kLeast));
  s.split_tiles = (int)((tiles + want - 1) / want);
  s.splits = (tiles + s.split_tiles - 1) / s.split_tiles;
  return s;
}
int width(int d) { return d <= 32 ? 32 : d <= 64 ? 64 : 128; }

struct Layout {
  Side query, key;
  size_t spans, rowsum, rowslope, part_q, part_k, part_v, total;  // places in the workspace
};
Layout layout(int B, int Nq, int Nk, int H, int Hk, int d, int dtype, bool docs, bool want_dslope) {
  Layout l;
  const int D = width(d), el = dtype == 1 ? 2 : 4;
  const long long rows = (long long)Nq * (H / Hk);
  l.query = side(rows, Nk, (long long)B * Hk, D, el);
  l.key = side(Nk, rows, (long long)B * Hk, D, el);
  size_t off = 0;
  const auto take = [&](size_t bytes) {
    const size_t at = off;
    off += attn_align(bytes);
    return at;
  };
  const size_t nq = (size_t)B * Nq * H, nk = (size_t)B * Nk * Hk;
  l.spans = take(docs ? attn_span_bytes(B, Nq, Nk) : 0);
  l.rowsum = take(nq * 4);
  l.rowslope = take(want_dslope ? (size_t)l.query.splits * 3 * nq * 4 : 0);
  l.part_q = take(l.query.splits > 1 ? (size_t)l.query.splits * nq * d * 4 : 0);
  l.part_k = take(l.key.splits > 1 ? (size_t)l.key.splits * nk * d * 4 : 0);
  l.part_v = take(l.key.splits > 1 ? (size_t)l.key.splits * nk * d * 4 : 0);
  l.total = off;
  return l;
}

template <typename T, int D, bool TERMS>
hipError_t launch(const AttnParams& pq, const AttnParams& pk, hipStream_t stream) {
  const size_t lds = 4 * TileRows<T, D>::kBytes;
  hipError_t e = hipFuncSetAttribute((const void*)attn_bwd_query_kernel<T, D, TERMS>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
  if (e != hipSuccess) return e;
  e = hipFuncSetAttribute((const void*)attn_bwd_key_kernel<T, D, TERMS>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
  if (e != hipSuccess) return e;
  AFFMAE_LAUNCH("attn_bwd_query_kernel", stream, (attn_bwd_query_kernel<T, D, TERMS>), dim3((pq.work + 7) / 8 * 8), dim3(kAttnThreads), lds, stream, pq);
  AFFMAE_LAUNCH("attn_bwd_key_kernel", stream, (attn_bwd_key_kernel<T, D, TERMS>), dim3((pk.work + 7) / 8 * 8), dim3(kAttnThreads), lds, stream, pk);
  return hipGetLastError();
}
template <typename T, bool TERMS>
hipError_t launch_width(const AttnParams& pq, const AttnParams& pk, hipStream_t stream) {
  switch (width(pq.d)) {
    case 32: return launch<T, 32, TERMS>(pq, pk, stream);
    case 64: return launch<T, 64, TERMS>(pq, pk, stream);
    default: return launch<T, 128, TERMS>(pq, pk, stream);
  }
}

}  // namespace

size_t attn_bwd_workspace_bytes(int B, int Nq, int Nk, int H, int Hk, int d, int dtype, bool docs, bool want_dslope) {
  return layout(B, Nq, Nk, H, Hk, d, dtype, docs, want_dslope).total;
}

hipError_t launch_attn_bwd(const AttnArgs& a, hipStream_t stream) {
  const Layout l = layout(a.B, a.Nq, a.Nk, a.H, a.Hk, a.d, a.dtype, a.q_doc != nullptr, a.dslope != nullptr);
  char* ws = static_cast<char*>(a.workspace);
  AttnParams p = attn_params(a, reinterpret_cast<Span*>(ws + l.spans));
  p.rowsum = reinterpret_cast<float*>(ws + l.rowsum);
  p.rowslope = a.dslope ? reinterpret_cast<float*>(ws + l.rowslope) : nullptr;
  p.grad_scale = a.scale;
  p.dq = a.dq; p.dk = a.dk; p.dv = a.dv;
  AttnParams pq = p, pk = p;
  pq.blocks = l.query.blocks; pq.splits = l.query.splits; pq.split_tiles = l.query.split_tiles;
  pk.blocks = l.key.blocks; pk.splits = l.key.splits; pk.split_tiles = l.key.split_tiles;
  for (AttnParams* x : {&pq, &pk}) {
    x->blocks_magic = div_magic(x->blocks);
    x->work = a.B * a.Hk * x->blocks * x->splits;
  }
  if (pq.splits > 1) pq.part = reinterpret_cast<float*>(ws + l.part_q);
  if (pk.splits > 1) pk.part = reinterpret_cast<float*>(ws + l.part_k), pk.part_v = reinterpret_cast<float*>(ws + l.part_v);
  hipError_t e = hipSuccess;
  if (a.q_doc) e = launch_attn_spans(a, const_cast<Span*>(p.q_span), const_cast<Span*>(p.k_span), stream);
  if (e != hipSuccess) return e;
  const bool terms = a.cap > 0.f || a.slope;
  if (a.dtype == 1) e = terms ? launch_width<bf16_t, true>(pq, pk, stream) : launch_width<bf16_t, false>(pq, pk, stream);
  else e = terms ? launch_width<float, true>(pq, pk, stream) : launch_width<float, false>(pq, pk, stream);
  if (e != hipSuccess) return e;
  Joins j = {};
  int parts = 0;
  const auto join = [&](const float* part, void* out, int splits, size_t n) {
    j.part[parts] = part; j.out[parts] = out; j.splits[parts] = splits; j.n[parts] = n;
    ++parts;
  };
  if (pq.splits > 1) join(pq.part, a.dq, pq.splits, (size_t)a.B * a.Nq * a.H * a.d);
  if (pk.splits > 1) {
    join(pk.part, a.dk, pk.splits, (size_t)a.B * a.Nk * a.Hk * a.d);
    join(pk.part_v, a.dv, pk.splits, (size_t)a.B * a.Nk * a.Hk * a.d);
  }
  if (parts) {
    const size_t most = *std::max_element(j.n, j.n + parts);
    const dim3 grid((unsigned)std::min<size_t>((most / 4 + 255) / 256, 4096), parts);
    if (a.dtype == 1) AFFMAE_LAUNCH("attn_bwd_join_kernel", stream, attn_bwd_join_kernel<bf16_t>, grid, dim3(256), 0, stream, j);
    else AFFMAE_LAUNCH("attn_bwd_join_kernel", stream, attn_bwd_join_kernel<float>, grid, dim3(256), 0, stream, j);
  }
  if (a.dslope)
    AFFMAE_LAUNCH("attn_bwd_slope_kernel", stream, attn_bwd_slope_kernel, dim3(a.H), dim3(1024), 0, stream, p.rowslope, pq.splits, a.H, (size_t)a.B * a.Nq, a.dslope);
  return hipGetLastError();
}

}  // namespace affmae
