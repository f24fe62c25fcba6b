// Attention between all tokens, backward by keys: dk and dv (attn_bwd.hip has the formulas).  A workgroup keeps 128 keys of an image and key
// head with their values; the rows that may see them, of all the head's queries, come by with their dout, lse and D.
// With 128 channels the keys, values and both gradients of 32 keys take 192 of a lane's 256 registers (two waves a SIMD; with one wave and twice
// the registers 8 x 4096 tokens of 6 heads take 960 us instead of 838, less being hidden behind the other wave), and a tile's two blocks are taken in turn.
#include "attn_common.h"
#include "timing.h"

namespace affmae {
namespace {

// Rows of a tile, as they are in memory (attn_common.h: KeyNotes): lse and D (zeros behind the last one, whose vectors are zeros too), place,
// slope and image.
struct RowNotes {
  float lse[64], sum[64], x[64], y[64], slope[64];
  int doc[64];
};
struct RowSource {
  i32x4 lse, sum, xy, slope, doc;
  int rows, G;
  uint32_t g_magic;
  __device__ __forceinline__ RowSource(const AttnParams& p, int b, int hk, bool places, bool images) : rows(p.rows), G(p.G), g_magic(p.g_magic) {
    const size_t at = ((size_t)b * p.Hk + hk) * p.rows;
    lse = uniform(buffer_of((const char*)(p.rowlse + at), 4ll * p.rows));
    sum = uniform(buffer_of((const char*)(p.rowsum + at), 4ll * p.rows));
    if (places) {
      xy = uniform(buffer_of((const char*)(p.q_xy + 2 * (size_t)b * p.Nq), 8ll * p.Nq));
      slope = uniform(buffer_of((const char*)(p.slope + hk * p.G), 4ll * p.G));
    }
    if (images) doc = uniform(buffer_of((const char*)(p.q_doc + (size_t)b * p.Nq), 4ll * p.Nq));
  }
  // of 64 rows, whatever a tile has (KeySource::load)
  template <int TERMS, bool DOCS, bool ALONE>
  __device__ __forceinline__ void load(RowNotes& n, int r0, int wave, int lane) const {
    const int r = r0 + lane;
    const bool there = r < rows;
    if (ALONE || wave == 0) lds_load<4>(lds_at(n.lse), lse, there ? (uint32_t)r * 4u : kNowhere);
    if (ALONE || wave == 1) lds_load<4>(lds_at(n.sum), sum, there ? (uint32_t)r * 4u : kNowhere);
    if constexpr (DOCS || (TERMS & kDistance)) {
      const int i = exact_div(r, G, g_magic);
      if constexpr (TERMS & kDistance) {
        if (ALONE || wave == 2) {
          const uint32_t at = there ? (uint32_t)i * 8u : kNowhere;
          lds_load<4>(lds_at(n.x), xy, at);
          lds_load<4>(lds_at(n.y), xy, at + 4);
        }
        if (ALONE || wave == 3) lds_load<4>(lds_at(n.slope), slope, there ? (uint32_t)(r - i * G) * 4u : kNowhere);
      }
      if constexpr (DOCS)
        if (ALONE || wave == 0) lds_load<4>(lds_at(n.doc), doc, there ? (uint32_t)i * 4u : kNowhere);
    }
  }
};

template <typename T, int D, int TERMS, bool DOCS, bool ALONE>
__global__ __launch_bounds__(kAttnThreads, (sizeof(T) == 4 && D > 32 ? 1 : 2)) void attn_bwd_key_kernel(AttnParams p) {
  using R = TileRows<T, D, ALONE>;
  constexpr int BN = R::BN, kTogether = D == 128 ? 1 : 2;  // blocks of a tile that are worked on together
  extern __shared__ __align__(16) char lds[];
  __shared__ RowNotes notes[ALONE ? 4 : 2];
  const int work = xcd_contiguous_block(blockIdx.x, gridDim.x);
  if (work >= p.work) return;
  const int group = exact_div(work, p.blocks, p.blocks_magic), block = work - group * p.blocks;
  const int split = group / (p.B * p.Hk), bh = group - split * p.B * p.Hk, b = bh / p.Hk, hk = bh - b * p.Hk;
  const int lane = threadIdx.x & 63, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  constexpr int kRows = ALONE ? 32 : kAttnRows;
  const int block0 = block * kRows, j0 = ALONE ? block0 : block0 + wave * 32;
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
  int own_doc = DOCS ? max(p.k_doc[token], -1) : 0;
  const Source<T, D, false> queries(p, p.q, b, hk), douts(p, p.dout, b, hk);
  Fixed<T, D> k, v;
  const int own_bytes = there ? p.d * R::E : 0;  // (a branch around the loads: 92 us instead of 85 with 32 channels and distances)
  k.load((const char*)p.k + own_at * p.d * R::E, half, own_bytes);
  v.load((const char*)p.v + own_at * p.d * R::E, half, own_bytes);
  if (p.negate) {
#pragma unroll
    for (int s = 0; s < R::kSteps; ++s) k.x[s].negate();
  }

  const int tiles = (p.rows + BN - 1) / BN;
  Walk walk;
  walk.spans = nullptr;
  walk.mixed = false;
  walk.end = min(tiles, (split + 1) * p.split_tiles);
  walk.tile_rows = BN; walk.G = p.G; walk.g_magic = p.g_magic;
  if constexpr (DOCS) {
    walk.spans = p.q_span + (size_t)b * ((p.Nq + kSpan - 1) / kSpan);
    walk.own(p.k_span + (size_t)b * ((p.Nk + kSpan - 1) / kSpan), block0, min(block0 + kRows, p.Nk) - 1);
  }
  walk.start(split * p.split_tiles);

  const RowSource about(p, b, hk, TERMS & kDistance, DOCS);
  const auto fetch = [&](int t, int buffer, bool& masked) __attribute__((always_inline)) {
    char* dst = lds + (ALONE ? wave : buffer) * 2 * R::kBytes;
    bool pads = false;
    masked = false;
    if constexpr (DOCS) {
      pads = walk.padded(t);
      masked = walk.hides(t);
    }
    queries.template load<ALONE>(dst, t * BN, pads);
    douts.template load<ALONE>(dst + R::kBytes, t * BN, pads);
    about.load<TERMS, DOCS, ALONE>(notes[ALONE ? wave : buffer], t * BN, wave, lane);
  };

  k.arrive();
  v.arrive();
  arrive(own_x);
  arrive(own_y);
  arrive(own_doc);
  f32x16 dk[D / 32] = {}, dv[D / 32] = {};
  bool masked = false;
  int t = walk.skip(p.rows, ALONE ? wave : 0);
  if (t < walk.end) fetch(t, 0, masked);
  for (int buffer = 0; t < walk.end; buffer ^= ALONE ? 0 : 1) {
    // the tile has arrived, and (with a barrier) every wave has read what the next one will be written over
    if constexpr (ALONE) asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    const int following = walk.skip(p.rows, ALONE ? 3 : 0);
    bool next_masked = false;
    if (!ALONE && following < walk.end) fetch(following, buffer ^ 1, next_masked);
    const char* qt = lds + (ALONE ? wave : buffer) * 2 * R::kBytes;
    const char* gt = qt + R::kBytes;
    if (busy) {
      const RowNotes& n = notes[ALONE ? wave : buffer];
#pragma unroll kTogether
      for (int rb = 0; rb < R::kBlocks; ++rb) {
        f32x16 s, dp;
        row_products<T, D>(qt, rb, k, s, lane, p.d);
        row_products<T, D>(gt, rb, v, dp, lane, p.d);
        const auto slopes = [&](auto near, auto hides) __attribute__((always_inline)) {
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int r = 32 * rb + 16 * (i >> 3) + 8 * half + (i & 7);
            float bend, distance, dx = 0.f, dy = 0.f, slope = 0.f;
            if constexpr (TERMS & kDistance) dx = n.x[r] - own_x, dy = n.y[r] - own_y, slope = n.slope[r] * kLog2e;
            const float z = score<T, TERMS, near>(s[i], p, dx, dy, slope, n.lse[r], bend, distance);
            float pr = __builtin_amdgcn_exp2f(z), ds = pr * (dp[i] - n.sum[r]);
            if constexpr (TERMS & kCap) ds *= bend_slope(bend, p);
            if constexpr (hides) {
              const bool off = n.doc[r] != own_doc;
              pr = off ? 0.f : pr;
              ds = off ? 0.f : ds;
            }
            s[i] = pr;
            dp[i] = ds;
          }
        };
        using yes = std::true_type;
        using no = std::false_type;
        bool near = false;
        if constexpr ((TERMS & kCap) && D < 128) near = all_near(s, p.near);
        if (DOCS && (D == 128 || masked)) {  // (one way through where two would not fit the registers)
          if (near) slopes(yes{}, yes{});
          else slopes(no{}, yes{});
        } else {
          if (near) slopes(yes{}, no{});
          else slopes(no{}, no{});
        }
        const Weights<T> wp(s), ws(dp);
        column_products<D, 1>(gt, rb, {&wp}, {dv}, lane, p.d);
        column_products<D, 1>(qt, rb, {&ws}, {dk}, lane, p.d);
      }
    }
    if (ALONE && following < walk.end) {
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // (the tile has been read)
      fetch(following, buffer, next_masked);
    }
    t = following;
    masked = next_masked;
  }

  if constexpr (ALONE) {
    __syncthreads();  // (the last tiles have been read)
    add_waves<D>(lds, wave, lane, dk);
    __syncthreads();
    add_waves<D>(lds, wave, lane, dv);
  }
  if (!busy || !there) return;
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int ch = 32 * db + 8 * e + 4 * half;
      if (ch < p.d && (!ALONE || e == wave)) {
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

template <typename T, int D, int TERMS, bool DOCS, bool ALONE>
hipError_t launch_kernel(const AttnParams& p, hipStream_t stream) {
  const size_t lds = (ALONE ? 8 : 4) * TileRows<T, D, ALONE>::kBytes;
  const hipError_t e = hipFuncSetAttribute((const void*)attn_bwd_key_kernel<T, D, TERMS, DOCS, ALONE>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
  if (e != hipSuccess) return e;
  AFFMAE_LAUNCH("attn_bwd_key_kernel", stream, (attn_bwd_key_kernel<T, D, TERMS, DOCS, ALONE>), dim3((p.work + 7) / 8 * 8), dim3(kAttnThreads), lds, stream, p);
  return hipGetLastError();
}
template <typename T, int D, int TERMS, bool DOCS>
hipError_t launch_docs(const AttnParams& p, hipStream_t stream) {
  return p.alone ? launch_kernel<T, D, TERMS, DOCS, true>(p, stream) : launch_kernel<T, D, TERMS, DOCS, false>(p, stream);
}
template <typename T, int D, int TERMS>
hipError_t launch(const AttnParams& p, hipStream_t stream) {
  return p.q_doc ? launch_docs<T, D, TERMS, true>(p, stream) : launch_docs<T, D, TERMS, false>(p, stream);
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

}  // namespace

hipError_t launch_attn_bwd_key(const AttnParams& p, int dtype, hipStream_t stream) {
  return dtype == 1 ? launch_terms<bf16_t>(p, stream) : launch_terms<float>(p, stream);
}

}  // namespace affmae
