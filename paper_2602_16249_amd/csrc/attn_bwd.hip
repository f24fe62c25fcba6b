// Attention between all tokens, backward.  With p = exp(z - lse) worked out again and g = dout, per image and head (attn_fwd.hip has z):
//     dP_ij = <g_i, v_j>,  D_i = <g_i, out_i>,  dZ_ij = p_ij (dP_ij - D_i),  dS_ij = dZ_ij (1 - tanh^2),
//     dq_i = scale sum_j dS_ij k_j,  dk_j = scale sum_i dS_ij q_i,  dv_j = sum_i p_ij g_i,  dslope_h = -sum_ij dZ_ij |x_i - y_j|.
// Two kernels, one that keeps queries and lets keys come by (dq, D, dslope; this file) and one the other way round (dk, dv; attn_bwd_key.hip):
// seven products of two of a pair's vectors instead of five, and nothing is added up by atomics: the results are the same in every
// run, and grouped heads' gradients add up in registers.
//
// Bound by the vector ALU with 32 channels (16 x 1024 tokens, 8 heads, distances: 90 us, key kernel 85), by matrix instructions with 128 (8 x 4096, 6
// heads: 756 to 776 us, 1063 to 1091 TFLOP/s, near the rate of a large library product; key kernel 808 to 838 us, 984 to 1020); 48 x 2048 tokens, 6
// heads of 64: 638 us, key kernel 693.
//
// D from the bf16 out is off by what out was rounded by, which counts where few keys share a row's weight, in a row of any length (500
// queries near the sum of two keys, of 2 of 64 channels or of 1024 of 128: dq off by 0.0049 and 0.0060 of its size, dk by 0.0029 and
// 0.0055, rows with one key in front by all of their own).  The row's dZ sum to 0 if D is right, so their sum is what D lacks: the key kernel
// gets it, and dq is put right at the end by as much of sum_j p_ij k_j, one more product (dq 0.0025, dk at most 0.0025).  How many keys
// share a row's weight is not known beforehand, so every bf16 row has it.  With 128 channels that product is not hidden behind the
// exponentials (8 x 4096 tokens, 6 heads: 546 us without it), and its sums take registers: the forms of 128 channels spill, 6 to 87 of them.  Room for
// one wave a SIMD, where nothing spills, is worse all the same (885 us instead of 776 on the same day), but for images with distances
// (96 x 1024 tokens of one head, both kernels: 322 us, 307 with one wave; capped 446, 364).
#include "attn_common.h"
#include "timing.h"

#include <algorithm>

namespace affmae {
namespace {

template <typename T, int D, int TERMS, bool DOCS, bool ALONE>
__global__ __launch_bounds__(kAttnThreads, (kAttnWaves<T, D>)) void attn_bwd_query_kernel(AttnParams p) {
  using R = TileRows<T, D, ALONE>;
  constexpr int BN = R::BN, kTogether = D == 128 ? 1 : 2;  // blocks of a tile that are worked on together
  constexpr bool REST = sizeof(T) == 2;  // D is put right
  extern __shared__ __align__(16) char lds[];
  __shared__ KeyNotes notes[ALONE ? 4 : 2];
  const int work = xcd_contiguous_block(blockIdx.x, gridDim.x);
  if (work >= p.work) return;
  const int group = exact_div(work, p.blocks, p.blocks_magic), block = work - group * p.blocks;
  const int split = group / (p.B * p.Hk), bh = group - split * p.B * p.Hk, b = bh / p.Hk, hk = bh - b * p.Hk;
  const int lane = threadIdx.x & 63, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  constexpr int kRows = ALONE ? 32 : kAttnRows;
  const int block0 = block * kRows, r0 = ALONE ? block0 : block0 + wave * 32;
  const bool busy = r0 < p.rows;
  Row own = own_row(p, b, hk, r0);
  const Source<T, D, true> keys(p, p.k, b, hk), values(p, p.v, b, hk);
  Fixed<T, D> q, g;
  if (own.there) {
    q.load((const char*)p.q + own.at * p.d * R::E, half, p.d * R::E);
    g.load((const char*)p.dout + own.at * p.d * R::E, half, p.d * R::E);
  } else {
    q.zero();
    g.zero();
  }
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
  const float seen = own.there ? p.lse[own.at] : 0.f;
  float lse = seen == -__builtin_inff() ? __builtin_inff() : seen * kLog2e;  // (no key: every p is 0)

  const int tiles = (p.Nk + BN - 1) / BN;
  Walk walk;
  walk.spans = nullptr;
  walk.mixed = false;
  walk.end = min(tiles, (split + 1) * p.split_tiles);
  walk.tile_rows = BN; walk.G = 1; walk.g_magic = 0u;
  if constexpr (DOCS) {
    walk.spans = p.k_span + (size_t)b * ((p.Nk + kSpan - 1) / kSpan);
    walk.own(p.q_span + (size_t)b * ((p.Nq + kSpan - 1) / kSpan), exact_div(block0, p.G, p.g_magic), exact_div(min(block0 + kRows, p.rows) - 1, p.G, p.g_magic));
  }
  walk.start(split * p.split_tiles);

  const KeySource about(p, b, TERMS & kDistance, DOCS);
  const auto fetch = [&](int t, int buffer, bool& masked) __attribute__((always_inline)) {
    char* dst = lds + (ALONE ? wave : buffer) * 2 * R::kBytes;
    bool pads = false;
    masked = t * BN + BN > p.Nk;
    if constexpr (DOCS) {
      pads = walk.padded(t);
      masked = masked || walk.hides(t);
    }
    keys.template load<ALONE>(dst, t * BN, pads);
    values.template load<ALONE>(dst + R::kBytes, t * BN, pads);
    about.load<TERMS, DOCS, ALONE>(notes[ALONE ? wave : buffer], t * BN, wave, lane);
  };

  q.arrive();
  g.arrive();
  arrive(own);
  arrive(lse);
  arrive(sum);
  f32x16 dq[D / 32] = {}, keys_seen[REST ? D / 32 : 1] = {};  // sums of dS k, and of what multiplies D in dS
  float by_distance = 0.f, rest = 0.f, distances = 0.f;  // sums of dZ |x - y|, of dZ, of p |x - y|
  bool masked = false;
  int t = walk.skip(p.Nk, ALONE ? wave : 0);
  if (t < walk.end) fetch(t, 0, masked);
  for (int buffer = 0; t < walk.end; buffer ^= ALONE ? 0 : 1) {
    // the tile has arrived, and (with a barrier) every wave has read what the next one will be written over
    if constexpr (ALONE) asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    const int following = walk.skip(p.Nk, ALONE ? 3 : 0);
    bool next_masked = false;
    if (!ALONE && following < walk.end) fetch(following, buffer ^ 1, next_masked);
    const char* kt = lds + (ALONE ? wave : buffer) * 2 * R::kBytes;
    const char* vt = kt + R::kBytes;
    if (busy) {
      const int left = p.Nk - t * BN - 8 * half;  // keys of the tile that are there, from the lane's first one on
      const KeyNotes& n = notes[ALONE ? wave : buffer];
#pragma unroll kTogether
      for (int kb = 0; kb < R::kBlocks; ++kb) {
        f32x16 s, dp;
        row_products<T, D>(kt, kb, q, s, lane, p.d);
        row_products<T, D>(vt, kb, g, dp, lane, p.d);
        const auto slopes = [&](auto near, auto hides) __attribute__((always_inline)) {
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int j = 32 * kb + 16 * (i >> 3) + 8 * half + (i & 7);
            float bend, distance, dx = 0.f, dy = 0.f;
            if constexpr (TERMS & kDistance) dx = own.x - n.x[j], dy = own.y - n.y[j];
            const float z = score<T, TERMS, near>(s[i], p, dx, dy, own.slope, lse, bend, distance);
            float pr = __builtin_amdgcn_exp2f(z);
            float dz = pr * (dp[i] - sum);
            if constexpr (hides) {  // (keys behind the last one, too: their p, exp(0 - lse), may not fit 32 bits)
              const bool off = j - 8 * half >= left || (DOCS && n.doc[j] != own.doc);
              pr = off ? 0.f : pr;
              dz = off ? 0.f : dz;
              if constexpr (DOCS && (TERMS & kDistance)) distance = off ? 0.f : distance;  // (padding may have any place)
            }
            if constexpr (REST || (TERMS & kDistance)) rest += dz;
            if constexpr (TERMS & kDistance) {
              by_distance = __builtin_fmaf(dz, distance, by_distance);
              distances = __builtin_fmaf(pr, distance, distances);
            }
            if constexpr (TERMS & kCap) {
              const float bends = bend_slope(bend, p);
              dz *= bends;
              if constexpr (REST) pr *= bends;
            }
            s[i] = dz;
            dp[i] = pr;
          }
        };
        using yes = std::true_type;
        using no = std::false_type;
        bool near = false;
        if constexpr ((TERMS & kCap) && D < 128) near = all_near(s, p.near);
        if (masked || D == 128) {  // (one way through where two would not fit the registers)
          if (near) slopes(yes{}, yes{});
          else slopes(no{}, yes{});
        } else {
          if (near) slopes(yes{}, no{});
          else slopes(no{}, no{});
        }
        const Weights<T> w(s);
        if constexpr (REST) {
          const Weights<T> wp(dp);
          column_products<D, 2>(kt, kb, {&w, &wp}, {dq, keys_seen}, lane, p.d);
        } else {
          column_products<D, 1>(kt, kb, {&w}, {dq}, lane, p.d);
        }
      }
    }
    if (ALONE && following < walk.end) {
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // (the tile has been read)
      fetch(following, buffer, next_masked);
    }
    t = following;
    masked = next_masked;
  }

  rest = other_half_sum(rest);
  if constexpr (TERMS & kDistance) {
    by_distance = other_half_sum(by_distance);
    distances = other_half_sum(distances);
  }
  if constexpr (ALONE) {
    __syncthreads();  // (the last tiles have been read)
    add_waves<D>(lds, wave, lane, dq);
    if constexpr (REST) {
      __syncthreads();
      add_waves<D>(lds, wave, lane, keys_seen);
    }
    if constexpr (REST || (TERMS & kDistance)) {
      float* at = reinterpret_cast<float*>(lds) + lane;
      __syncthreads();
      at[wave * 64] = rest;
      at[256 + wave * 64] = by_distance;
      at[512 + wave * 64] = distances;
      __syncthreads();
      rest = (at[0] + at[64]) + (at[128] + at[192]);
      by_distance = (at[256] + at[320]) + (at[384] + at[448]);
      distances = (at[512] + at[576]) + (at[640] + at[704]);
    }
  }
  if (!busy) return;
  const bool pad = own.doc < 0, first = half == 0 && (!ALONE || wave == 0);
  if (pad) rest = by_distance = distances = 0.f;  // (padding may hold anything)
  if (own.there && first) {
    const size_t row = (size_t)bh * p.rows + own.r;
    const bool none = pad || lse == __builtin_inff();
    if (split == 0) {
      p.rowlse[row] = none ? __builtin_inff() : lse;
      p.rowsum[row] = none ? 0.f : sum + (REST && p.splits == 1 ? rest : 0.f);
    }
    if (REST && p.splits > 1) p.rowrest[(size_t)split * p.B * p.Nq * p.H + row] = none ? 0.f : rest;
  }
  if constexpr (TERMS & kDistance) {
    if (p.rowslope && own.there && first) {
      const size_t tokens = (size_t)p.B * p.Nq, plane = (size_t)p.H * tokens;
      float* to = p.rowslope + (size_t)split * 3 * plane + (size_t)own.head * tokens + (size_t)b * p.Nq + own.i;
      to[0] = by_distance;
      to[plane] = rest;
      to[2 * plane] = distances;
    }
  }
  if (!own.there) return;
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int ch = 32 * db + 8 * e + 4 * half;
      if (ch < p.d && (!ALONE || e == wave)) {
        float v[4], u[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          v[c] = pad ? 0.f : dq[db][4 * e + c];
          u[c] = !REST || pad ? 0.f : keys_seen[REST ? db : 0][4 * e + c];
        }
        if (p.part) {
          const size_t to = ((size_t)split * p.B * p.Nq * p.H + own.at) * p.d + ch;
          store_piece<4>(p.part + to, v);
          if (REST) store_piece<4>(p.part_v + to, u);
        } else {
#pragma unroll
          for (int c = 0; c < 4; ++c) v[c] = __builtin_fmaf(-rest, u[c], v[c]) * p.grad_scale;
          store_piece<4>((T*)p.dq + own.at * p.d + ch, v);
        }
      }
    }
}

template <typename T, int D, int TERMS, bool DOCS, bool ALONE>
hipError_t launch_kernel(const AttnParams& p, hipStream_t stream) {
  const size_t lds = (ALONE ? 8 : 4) * TileRows<T, D, ALONE>::kBytes;
  const hipError_t e = hipFuncSetAttribute((const void*)attn_bwd_query_kernel<T, D, TERMS, DOCS, ALONE>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
  if (e != hipSuccess) return e;
  AFFMAE_LAUNCH("attn_bwd_query_kernel", stream, (attn_bwd_query_kernel<T, D, TERMS, DOCS, ALONE>), dim3((p.work + 7) / 8 * 8), dim3(kAttnThreads), lds, stream, p);
  return hipGetLastError();
}
template <typename T, int D, int TERMS>
hipError_t launch(const AttnParams& p, hipStream_t stream) {
  if (p.q_doc) return p.alone ? launch_kernel<T, D, TERMS, true, true>(p, stream) : launch_kernel<T, D, TERMS, true, false>(p, stream);
  return p.alone ? launch_kernel<T, D, TERMS, false, true>(p, stream) : launch_kernel<T, D, TERMS, false, false>(p, stream);
}
template <typename T, int TERMS>
hipError_t launch_width(const AttnParams& p, hipStream_t stream) {
  switch (attn_width(p.d)) {
    case 32: return launch<T, 32, TERMS>(p, stream);
    case 64: return launch<T, 64, TERMS>(p, stream);
    default: return launch<T, 128, TERMS>(p, stream);
  }
}
template <typename T>
hipError_t launch_query(const AttnParams& p, hipStream_t stream) {
  if (p.cap > 0.f) return p.slope ? launch_width<T, kCap | kDistance>(p, stream) : launch_width<T, kCap>(p, stream);
  return p.slope ? launch_width<T, kDistance>(p, stream) : launch_width<T, 0>(p, stream);
}

// Parts of splits added up, in their order: of dq, or of dk and dv, a blockIdx.y each.  With `rest`, whose sum is what D lacks in a row of d
// values, as much of `seen` is taken off, and D gets it; the whole times `scale`.
struct Join {
  const float *part, *seen, *rest;
  float* sum;  // with rest: D, which it is added to
  void* out;
  int splits, d;
  size_t n;  // values, a multiple of 4
  float scale;
  int rows, H, G;  // with rest: part's rows are (query, head) in [B,Nq,H], rest's and sum's [B,Hk,rows]
};
struct Joins {
  Join of[2];
};
template <typename T>
__global__ __launch_bounds__(256) void attn_bwd_join_kernel(Joins all) {
  const Join j = blockIdx.y == 0 ? all.of[0] : all.of[1];
  for (size_t at = ((size_t)blockIdx.x * 256 + threadIdx.x) * 4; at < j.n; at += (size_t)gridDim.x * 1024) {
    float v[4] = {}, u[4] = {}, rest = 0.f;
    const size_t all_rows = j.n / j.d, at_row = at / j.d;
    size_t row = 0;
    if (j.rest) {
      const int head = (int)(at_row % j.H), Nq = j.rows / j.G;
      const size_t token = at_row / j.H, b = token / Nq, i = token - b * Nq;
      row = (b * (j.H / j.G) + head / j.G) * j.rows + i * j.G + head % j.G;
    }
    for (int s = 0; s < j.splits; ++s) {
      float x[4];
      load_piece<4>(j.part + s * j.n + at, x);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] += x[e];
      if (j.rest) {
        load_piece<4>(j.seen + s * j.n + at, x);
#pragma unroll
        for (int e = 0; e < 4; ++e) u[e] += x[e];
        rest += j.rest[s * all_rows + row];
      }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = __builtin_fmaf(-rest, u[e], v[e]) * j.scale;
    store_piece<4>((T*)j.out + at, v);
    if (j.rest && at % j.d == 0) j.sum[row] += rest;
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

struct Layout {
  AttnSide query, key;
  size_t spans, rowsum, rowlse, rowrest, rowslope, part_q, seen_q, part_k, part_v, total;  // places in the workspace
  bool rest;  // D is put right
};
Layout layout(int B, int Nq, int Nk, int H, int Hk, int d, int dtype, bool docs, bool want_dslope) {
  Layout l;
  const int D = attn_width(d), el = dtype == 1 ? 2 : 4;
  const long long rows = (long long)Nq * (H / Hk);
  l.query = attn_side(rows, Nk, (long long)B * Hk, D, el, docs);
  l.key = attn_side(Nk, rows, (long long)B * Hk, D, el, docs);
  size_t off = 0;
  const auto take = [&](size_t bytes) {
    const size_t at = off;
    off += attn_align(bytes);
    return at;
  };
  const size_t nq = (size_t)B * Nq * H, nk = (size_t)B * Nk * Hk;
  l.spans = take(docs ? attn_span_bytes(B, Nq, Nk) : 0);
  l.rest = dtype == 1;
  l.rowsum = take(nq * 4);
  l.rowlse = take(nq * 4);
  l.rowrest = take(l.rest && l.query.splits > 1 ? (size_t)l.query.splits * nq * 4 : 0);
  l.rowslope = take(want_dslope ? (size_t)l.query.splits * 3 * nq * 4 : 0);
  l.part_q = take(l.query.splits > 1 ? (size_t)l.query.splits * nq * d * 4 : 0);
  l.seen_q = take(l.query.splits > 1 && l.rest ? (size_t)l.query.splits * nq * d * 4 : 0);
  l.part_k = take(l.key.splits > 1 ? (size_t)l.key.splits * nk * d * 4 : 0);
  l.part_v = take(l.key.splits > 1 ? (size_t)l.key.splits * nk * d * 4 : 0);
  l.total = off;
  return l;
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
  p.rowlse = reinterpret_cast<float*>(ws + l.rowlse);
  p.rowrest = reinterpret_cast<float*>(ws + l.rowrest);
  p.grad_scale = a.scale;
  p.dq = a.dq; p.dk = a.dk; p.dv = a.dv;
  AttnParams pq = p, pk = p;
  pq.alone = l.query.alone; pq.blocks = l.query.blocks; pq.splits = l.query.splits; pq.split_tiles = l.query.split_tiles;
  pk.alone = l.key.alone; pk.blocks = l.key.blocks; pk.splits = l.key.splits; pk.split_tiles = l.key.split_tiles;
  for (AttnParams* x : {&pq, &pk}) {
    x->blocks_magic = div_magic(x->blocks);
    x->work = a.B * a.Hk * x->blocks * x->splits;
  }
  if (pq.splits > 1) pq.part = reinterpret_cast<float*>(ws + l.part_q), pq.part_v = reinterpret_cast<float*>(ws + l.seen_q);
  if (pk.splits > 1) pk.part = reinterpret_cast<float*>(ws + l.part_k), pk.part_v = reinterpret_cast<float*>(ws + l.part_v);
  hipError_t e = hipSuccess;
  if (a.q_doc) e = launch_attn_spans(a, const_cast<Span*>(p.q_span), const_cast<Span*>(p.k_span), stream);
  if (e != hipSuccess) return e;
  e = a.dtype == 1 ? launch_query<bf16_t>(pq, stream) : launch_query<float>(pq, stream);
  if (e != hipSuccess) return e;
  const size_t nq = (size_t)a.B * a.Nq * a.H * a.d, nk = (size_t)a.B * a.Nk * a.Hk * a.d;
  const auto join = [&](const Joins& j, int parts) {
    const dim3 grid((unsigned)std::min<size_t>((j.of[0].n / 4 + 255) / 256, 4096), parts);
    if (a.dtype == 1) AFFMAE_LAUNCH("attn_bwd_join_kernel", stream, attn_bwd_join_kernel<bf16_t>, grid, dim3(256), 0, stream, j);
    else AFFMAE_LAUNCH("attn_bwd_join_kernel", stream, attn_bwd_join_kernel<float>, grid, dim3(256), 0, stream, j);
  };
  if (pq.splits > 1) join({{{pq.part, pq.part_v, l.rest ? p.rowrest : nullptr, p.rowsum, a.dq, pq.splits, a.d, nq, a.scale, p.rows, a.H, p.G}}}, 1);
  e = launch_attn_bwd_key(pk, a.dtype, stream);
  if (e != hipSuccess) return e;
  if (pk.splits > 1)
    join({{{pk.part, nullptr, nullptr, nullptr, a.dk, pk.splits, a.d, nk, 1.f}, {pk.part_v, nullptr, nullptr, nullptr, a.dv, pk.splits, a.d, nk, 1.f}}}, 2);
  if (a.dslope)
    AFFMAE_LAUNCH("attn_bwd_slope_kernel", stream, attn_bwd_slope_kernel, dim3(a.H), dim3(1024), 0, stream, p.rowslope, pq.splits, a.H, (size_t)a.B * a.Nq, a.dslope);
  return hipGetLastError();
}

}  // namespace affmae
