// Attention between all tokens, forward: per image, head h and query i
//     z_j = scale <q_i, k_j>,  z_j = cap tanh(z_j / cap),  z_j -= slope_h |x_i - y_j|,  hidden where the images of i and j differ,
//     out_i = sum_j p_j v_j,  p = softmax(z),  lse_i = log sum_j exp z_j,
// in one pass over the keys with a running reference and sum of every row (attn_common.h: the tiles and their layout).
//
// Bound by the vector ALU up to 64 channels (a product, an exponential that takes the time of two, a sum and half a conversion a
// pair, beside 8 cycles of matrix instructions for 64 channels), by both with 128: 8 x 4096 tokens, 6 heads of 64 a call of 240 us (859 TFLOP/s), of 128
// 410 to 420 us (982 to 1005); 48 x 2048, 6 heads of 64 375 us; 16 x 1024, 8 heads of 32 with distances 66 to 68 us.  Two rows of 8001 tokens of 11
// images each, capped, 4 heads of 32: 50 us.  One query of 12 heads on 3, 4 x 16384 keys of 64: 14.5 us (3.5 TB/s) and 5.6 for the join.
#include "attn_common.h"
#include "timing.h"

#include <algorithm>

namespace affmae {
namespace {

// The four waves' running maximum, sum and output of the same rows, joined: every wave gets the maximum and the sum (of both halves), and
// wave w the sums of registers 4 w .. 4 w + 3 of each block of channels, which it stores.
template <int D>
__device__ __forceinline__ void join_waves(char* lds, int wave, int lane, f32x16 (&o)[D / 32], float& m, float& l) {
  l = other_half_sum(l);
  float* tops = reinterpret_cast<float*>(lds);
  __syncthreads();  // (the last tiles have been read)
  tops[wave * 64 + lane] = m;
  tops[256 + wave * 64 + lane] = l;
  __syncthreads();
  float top = m;
#pragma unroll
  for (int w = 0; w < 4; ++w) top = fmaxf(top, tops[w * 64 + lane]);
  const float from = top == -__builtin_inff() ? 0.f : top;
  float sum = 0.f;
#pragma unroll
  for (int w = 0; w < 4; ++w) sum += tops[256 + w * 64 + lane] * __builtin_amdgcn_exp2f(tops[w * 64 + lane] - from);
  const float mine = __builtin_amdgcn_exp2f(m - from);
#pragma unroll
  for (int db = 0; db < D / 32; ++db) o[db] *= mine;
  __syncthreads();
  add_waves<D>(lds, wave, lane, o);
  m = top;
  l = sum;
}

// Registers: bf16 heads of 32 channels leave room for four waves a SIMD (packed images 50 us and distances 66; three 55 and 69, five spill, 133 and
// 215; a chip that is not full gains by three, as the forms of blocks of 32 rows with images spill up to 14 registers under four: 16 x 1024 tokens of one
// head 19.2 us, 16.8 under three), of 64 for three (255 us; two 292, four spill, 1229), in blocks of 32 rows for two (one query 14.5 us; three
// spill, 16.3), as everything else.
template <typename T, int D, int TERMS, bool DOCS, bool ALONE>
__global__ __launch_bounds__(kAttnThreads, (sizeof(T) == 4 ? kAttnWaves<T, D> : D == 32 ? 4 : D == 64 && !ALONE ? 3 : 2)) void attn_fwd_kernel(AttnParams p) {
  using R = TileRows<T, D, ALONE>;
  constexpr int BN = R::BN;
  extern __shared__ __align__(16) char lds[];
  __shared__ KeyNotes notes[ALONE ? 4 : 2];
  const int work = xcd_contiguous_block(blockIdx.x, gridDim.x);
  if (work >= p.work) return;
  const int group = exact_div(work, p.blocks, p.blocks_magic), block = work - group * p.blocks;  // group: (split, image, key head)
  const int split = group / (p.B * p.Hk), bh = group - split * p.B * p.Hk, b = bh / p.Hk, hk = bh - b * p.Hk;
  const int lane = threadIdx.x & 63, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  constexpr int kRows = ALONE ? 32 : kAttnRows;
  const int block0 = block * kRows, r0 = ALONE ? block0 : block0 + wave * 32;
  const bool busy = r0 < p.rows;
  const Source<T, D, true> keys(p, p.k, b, hk), values(p, p.v, b, hk);
  Row own = own_row(p, b, hk, r0);
  Fixed<T, D> q;
  if (own.there) q.load((const char*)p.q + own.at * p.d * R::E, half, p.d * R::E);
  else q.zero();
  if (p.negate) {
#pragma unroll
    for (int s = 0; s < R::kSteps; ++s) q.x[s].negate();
  }

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
  arrive(own);
  f32x16 o[D / 32] = {};
  // The exponentials are taken from a score of the row that lies within 2^12 of the largest one (in p) so far: m.  It is found in the row's
  // first tile, and again where the sum over a tile says that a score lies above it, which hardly ever happens: floating
  // values lose nothing by being larger than 1, and the maximum of every tile took a tenth of the vector instructions.
  float m = -__builtin_inff(), l = 0.f;
  if (DOCS && own.doc < 0) m = 0.f;  // (padding: nothing to find)
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
      f32x16 s[R::kBlocks];
#pragma unroll
      for (int kb = 0; kb < R::kBlocks; ++kb) row_products<T, D>(kt, kb, q, s[kb], lane, p.d);
      const KeyNotes& about_key = notes[ALONE ? wave : buffer];
      const int left = p.Nk - t * BN - 8 * half;  // keys of the tile that are there, from the lane's first one on
      // s becomes score - from, hidden ones -infinity
      const auto scores = [&](auto near, auto hides, float from) __attribute__((always_inline)) {
#pragma unroll
        for (int kb = 0; kb < R::kBlocks; ++kb)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int j = 32 * kb + 16 * (i >> 3) + 8 * half + (i & 7);
            float bend, distance, dx = 0.f, dy = 0.f;
            if constexpr (TERMS & kDistance) dx = own.x - about_key.x[j], dy = own.y - about_key.y[j];
            float z = score<T, TERMS, near>(s[kb][i], p, dx, dy, own.slope, from, bend, distance);
            if constexpr (hides) z = j - 8 * half >= left || (DOCS && about_key.doc[j] != own.doc) ? -__builtin_inff() : z;
            s[kb][i] = z;
          }
      };
      const auto exponentials = [&]() __attribute__((always_inline)) {
        float sum = 0.f;
#pragma unroll
        for (int kb = 0; kb < R::kBlocks; ++kb)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            s[kb][i] = __builtin_amdgcn_exp2f(s[kb][i]);
            sum += s[kb][i];
          }
        return sum;
      };
      using yes = std::true_type;
      using no = std::false_type;
      const auto is_near = [&]() __attribute__((always_inline)) {
        bool near = true;
#pragma unroll
        for (int kb = 0; kb < R::kBlocks; ++kb) near = near && all_near(s[kb], p.near);
        return near;
      };
      bool search = masked || __any(m == -__builtin_inff()), near = false;
      if constexpr (TERMS & kCap) {
        near = is_near();
        search = search || !near;
      }
      if (!search) {
        scores(yes{}, no{}, m);
        const float sum = exponentials();
        search = __any(!(sum < 4096.f));
        if (search) {
#pragma unroll
          for (int kb = 0; kb < R::kBlocks; ++kb) row_products<T, D>(kt, kb, q, s[kb], lane, p.d);
        } else {
          l += sum;
        }
      }
      if (search) {
        if (masked) {
          if (near) scores(yes{}, yes{}, 0.f);
          else scores(no{}, yes{}, 0.f);
        } else {
          if (near) scores(yes{}, no{}, 0.f);
          else scores(no{}, no{}, 0.f);
        }
        float top = -__builtin_inff();
#pragma unroll
        for (int kb = 0; kb < R::kBlocks; ++kb)
#pragma unroll
          for (int i = 0; i < 16; ++i) top = fmaxf(top, s[kb][i]);
        top = other_half_max(top);
        if (__any(top > m)) {
          const float before = m;
          m = fmaxf(m, top);
          const float shrink = m == -__builtin_inff() ? 1.f : __builtin_amdgcn_exp2f(before - m);
          l *= shrink;
#pragma unroll
          for (int db = 0; db < D / 32; ++db) o[db] *= shrink;
        }
        const float from = m == -__builtin_inff() ? 0.f : m;
#pragma unroll
        for (int kb = 0; kb < R::kBlocks; ++kb)
#pragma unroll
          for (int i = 0; i < 16; ++i) s[kb][i] -= from;
        l += exponentials();
      }
#pragma unroll
      for (int kb = 0; kb < R::kBlocks; ++kb) {
        const Weights<T> w(s[kb]);
        column_products<D, 1>(vt, kb, {&w}, {o}, lane, p.d);
      }
    }
    if (ALONE && following < walk.end) {
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // (the tile has been read)
      fetch(following, buffer, next_masked);
    }
    t = following;
    masked = next_masked;
  }

  if constexpr (ALONE) join_waves<D>(lds, wave, lane, o, m, l);
  if (!busy) return;
  const float seen = ALONE ? l : other_half_sum(l), sum = DOCS && own.doc < 0 ? 0.f : seen;
  const bool none = sum == 0.f;  // (a NaN stays one)
  const float part = 1.f / sum;
  const float lse = none ? -__builtin_inff() : __builtin_fmaf(m, kLn2, __logf(sum));
  if (!own.there) return;
  const size_t all = (size_t)p.B * p.Nq * p.H;
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int ch = 32 * db + 8 * g + 4 * half;
      if (ch < p.d && (!ALONE || g == wave)) {
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = none ? 0.f : o[db][4 * g + e] * part;
        if (p.part) store_piece<4>(p.part + ((size_t)split * all + own.at) * p.d + ch, v);
        else store_piece<4>((T*)p.o + own.at * p.d + ch, v);
      }
    }
  if (half == 0 && (!ALONE || wave == 0)) (p.part ? p.part + (size_t)p.splits * all * p.d + (size_t)split * all : p.lse_out)[own.at] = lse;
}

// out = sum over splits of exp(lse_s - lse) out_s, lse = log sum exp lse_s.  A thread takes four channels of a (query, head) for every `lanes`th
// split, and the first of the lanes adds up, in their order.  (A thread for all splits waited for one after the other: 24 us for 43.)
template <typename T>
__global__ __launch_bounds__(256) void attn_join_kernel(const float* part, int splits, int lanes, size_t all, int d, T* out, float* lse) {
  __shared__ float sums[256][5];
  const int quarters = d / 4, per = quarters * lanes, rows = 256 / per;
  const int slot = (int)threadIdx.x / per, in_row = (int)threadIdx.x - slot * per, lane = in_row / quarters, ch = (in_row - lane * quarters) * 4;
  const size_t row = (size_t)blockIdx.x * rows + slot;
  const bool there = slot < rows && row < all;
  const float* ls = part + (size_t)splits * all * d + row;
  float top = -__builtin_inff(), sum = 0.f, v[4] = {};
  if (there) {
#pragma unroll 8
    for (int s = 0; s < splits; ++s) top = fmaxf(top, ls[s * all]);
    const float from = top == -__builtin_inff() ? 0.f : top;
    for (int s = lane; s < splits; s += lanes) {
      const float w = __expf(ls[s * all] - from);
      float x[4];
      load_piece<4>(part + (s * all + row) * d + ch, x);
      sum += w;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = __builtin_fmaf(w, x[e], v[e]);
    }
    top = from;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) sums[threadIdx.x][e] = v[e];
  sums[threadIdx.x][4] = sum;
  __syncthreads();
  if (!there || lane > 0) return;
  for (int i = 1; i < lanes; ++i) {
    const float* x = sums[threadIdx.x + i * quarters];
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] += x[e];
    sum += x[4];
  }
  const float inv = sum > 0.f ? 1.f / sum : (sum == sum ? 0.f : sum);
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] *= inv;
  store_piece<4>(out + row * d + ch, v);
  if (ch == 0) lse[row] = sum > 0.f ? top + __logf(sum) : (sum == sum ? -__builtin_inff() : sum);
}

__global__ __launch_bounds__(256) void attn_spans_kernel(const int32_t* q_doc, const int32_t* k_doc, int Nq, int Nk, int q_spans, int k_spans, int images, Span* to_q, Span* to_k) {
  const int at = (int)blockIdx.x * 4 + (int)(threadIdx.x / kWave), lane = threadIdx.x & 63;
  const int of_q = images * q_spans;
  if (at >= of_q + images * k_spans) return;
  const bool q = at < of_q;
  const int n = q ? at : at - of_q, spans = q ? q_spans : k_spans, N = q ? Nq : Nk;
  const int b = n / spans, i = (n - b * spans) * kSpan + lane;
  int lo = 0x7fffffff, hi = -1, pad = 0;
  if (i < N) {
    const int id = (q ? q_doc : k_doc)[(size_t)b * N + i];
    if (id < 0) pad = 1;
    else lo = hi = id;
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    lo = min(lo, __shfl_xor(lo, o));
    hi = max(hi, __shfl_xor(hi, o));
  }
  pad = __any(pad);
  if (lane == 0) (q ? to_q : to_k)[n] = Span{lo, hi, pad, 0};
}

template <typename T, int D, int TERMS, bool DOCS, bool ALONE>
hipError_t launch_kernel(const AttnParams& p, hipStream_t stream) {
  const size_t lds = (ALONE ? 8 : 4) * TileRows<T, D, ALONE>::kBytes;
  const hipError_t e = hipFuncSetAttribute((const void*)attn_fwd_kernel<T, D, TERMS, DOCS, ALONE>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
  if (e != hipSuccess) return e;
  AFFMAE_LAUNCH("attn_fwd_kernel", stream, (attn_fwd_kernel<T, D, TERMS, DOCS, ALONE>), dim3((p.work + 7) / 8 * 8), dim3(kAttnThreads), lds, stream, p);
  return hipGetLastError();
}
template <typename T, int D, int TERMS>
hipError_t launch(const AttnParams& p, hipStream_t stream) {
  const hipError_t e = p.q_doc ? (p.alone ? launch_kernel<T, D, TERMS, true, true>(p, stream) : launch_kernel<T, D, TERMS, true, false>(p, stream))
                               : (p.alone ? launch_kernel<T, D, TERMS, false, true>(p, stream) : launch_kernel<T, D, TERMS, false, false>(p, stream));
  if (e != hipSuccess || !p.part) return e;
  const size_t all = (size_t)p.B * p.Nq * p.H;
  const int lanes = std::min(p.splits, 256 / (p.d / 4)), rows = 256 / (lanes * (p.d / 4));
  AFFMAE_LAUNCH("attn_join_kernel", stream, attn_join_kernel<T>, dim3((unsigned)((all + rows - 1) / rows)), dim3(256), 0, stream, p.part, p.splits, lanes, all, p.d, (T*)p.o, p.lse_out);
  return hipGetLastError();
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
hipError_t launch_terms(const AttnParams& p, hipStream_t stream) {
  if (p.cap > 0.f) return p.slope ? launch_width<T, kCap | kDistance>(p, stream) : launch_width<T, kCap>(p, stream);
  return p.slope ? launch_width<T, kDistance>(p, stream) : launch_width<T, 0>(p, stream);
}

AttnSide side(int B, int Nq, int Nk, int H, int Hk, int d, int dtype, bool docs) {
  return attn_side((long long)Nq * (H / Hk), Nk, (long long)B * Hk, attn_width(d), dtype == 1 ? 2 : 4, docs);
}

}  // namespace

AttnParams attn_params(const AttnArgs& a, Span* spans) {
  AttnParams p = {};
  p.q = a.q; p.k = a.k; p.v = a.v; p.out = a.out; p.dout = a.dout; p.lse = a.lse;
  p.q_xy = a.q_xy; p.k_xy = a.k_xy; p.slope = a.slope; p.q_doc = a.q_doc; p.k_doc = a.k_doc;
  if (a.q_doc) {
    p.q_span = spans;
    p.k_span = spans + attn_align((size_t)a.B * attn_spans(a.Nq) * sizeof(Span)) / sizeof(Span);
  }
  p.B = a.B; p.Nq = a.Nq; p.Nk = a.Nk; p.H = a.H; p.Hk = a.Hk; p.G = a.H / a.Hk; p.d = a.d;
  p.rows = a.Nq * p.G;
  p.g_magic = div_magic(p.G);
  p.negate = a.scale < 0.f;
  p.scale = p.negate ? -a.scale : a.scale;
  p.cap = a.cap;
  const double log2e = 1.4426950408889634;
  p.factor = (float)(a.cap > 0.f ? (double)p.scale / a.cap : p.scale * log2e);
  if (a.cap > 0.f) {
    const double f = (double)p.scale / a.cap, c = p.scale * log2e;
    p.cap2 = (float)(a.cap * log2e);
    p.cap2_inv = (float)(1.0 / (a.cap * log2e));
    double power = c;
    bool fits = true;
    p.bend[0] = (float)c;
    for (int k = 0; k < 5; ++k) {
      power *= f * f;
      p.bend[k + 1] = (float)(power * (a.dtype == 1 ? kBend16 : kBend32)[k]);
      fits = fits && power < 1e30;
    }
    p.near = fits ? (float)(kNear / std::max(f, 1e-30)) : 0.f;
  }
  return p;
}

hipError_t launch_attn_spans(const AttnArgs& a, Span* q_span, Span* k_span, hipStream_t stream) {
  const int qs = attn_spans(a.Nq), ks = attn_spans(a.Nk);
  AFFMAE_LAUNCH("attn_spans_kernel", stream, attn_spans_kernel, dim3((unsigned)(((long long)a.B * (qs + ks) + 3) / 4)), dim3(256), 0, stream, a.q_doc, a.k_doc, a.Nq, a.Nk, qs, ks, a.B,
                q_span, k_span);
  return hipGetLastError();
}

size_t attn_fwd_workspace_bytes(int B, int Nq, int Nk, int H, int Hk, int d, int dtype, bool docs) {
  const AttnSide l = side(B, Nq, Nk, H, Hk, d, dtype, docs);
  return (docs ? attn_span_bytes(B, Nq, Nk) : 0) + (l.splits > 1 ? (size_t)l.splits * B * Nq * H * (d + 1) * sizeof(float) : 0);
}

hipError_t launch_attn_fwd(const AttnArgs& a, hipStream_t stream) {
  AttnParams p = attn_params(a, static_cast<Span*>(a.workspace));
  p.o = a.out;
  p.lse_out = a.lse;
  const AttnSide l = side(a.B, a.Nq, a.Nk, a.H, a.Hk, a.d, a.dtype, a.q_doc != nullptr);
  p.alone = l.alone; p.blocks = l.blocks; p.splits = l.splits; p.split_tiles = l.split_tiles;
  if (p.splits > 1) p.part = reinterpret_cast<float*>(static_cast<char*>(a.workspace) + (a.q_doc ? attn_span_bytes(a.B, a.Nq, a.Nk) : 0));
  p.blocks_magic = div_magic(p.blocks);
  p.work = a.B * a.Hk * p.blocks * p.splits;
  if (a.q_doc) {
    const hipError_t e = launch_attn_spans(a, const_cast<Span*>(p.q_span), const_cast<Span*>(p.k_span), stream);
    if (e != hipSuccess) return e;
  }
  return a.dtype == 1 ? launch_terms<bf16_t>(p, stream) : launch_terms<float>(p, stream);
}

}  // namespace affmae
