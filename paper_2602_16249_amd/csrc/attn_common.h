// What the kernels of attention between all tokens share (attn_fwd.hip, attn_bwd.hip).
//
// With G = H / Hk query heads to a key head, the Nq G (query, head) pairs that meet the same keys are the rows of one problem, row r =
// query r / G, head hk G + r % G, so that grouped heads share the keys on the chip and small calls of many heads fill their tiles.
// A workgroup of four waves keeps 128 rows (or keys) in registers, 32 to a wave, and lets tiles of the other side come through LDS, the
// next one on its way while one is used.  Where that makes too few workgroups (ALONE), it keeps 32 rows, the same in all four waves; each wave takes
// every fourth tile, fetched by itself, and the waves' results are joined at the end.
//
// Products are matrix instructions of 32 x 32.  The side in registers lies along the columns (a lane's column is lane % 32, in both
// halves), the side in LDS along the rows: a lane then holds 16 scores of one row of the softmax, whose sums need one exchange with
// the other half, and the scores are at once the second operand of the next product.  For that LDS rows are taken in the order
// that puts 8 consecutive ones into the lane's first 8 registers: place m of an instruction is row perm(m), bits 2 and 3 swapped.
#pragma once

#include "launch.h"

#include "cluster_common.h"
#include "dense_common.h"
#include "direct_lds.h"

#include <algorithm>

namespace affmae {

typedef __attribute__((ext_vector_type(16))) float f32x16;

constexpr int kAttnThreads = 256;
constexpr int kAttnRows = 128;  // of a workgroup
constexpr int kSpan = 64;       // tokens whose images are summed up beforehand
constexpr float kLog2e = 1.44269504f, kLn2 = 0.693147181f;

// Images of kSpan consecutive tokens: the lowest and highest one, and whether there is padding (id < 0) among them; lo > hi: nothing else.
struct Span {
  int lo, hi, pad, unused;
};

struct AttnParams {
  const void *q, *k, *v, *out, *dout;
  const float* lse;
  const float *q_xy, *k_xy, *slope;
  const int32_t *q_doc, *k_doc;
  const Span *q_span, *k_span;  // [B][spans of Nq], [B][spans of Nk], null without images
  int B, Nq, Nk, H, Hk, G, d, rows;
  uint32_t g_magic;
  float scale;   // at least 0: a negative one is taken off the queries
  bool negate;
  float cap;
  float factor;             // scale / cap, without a cap scale log2 e
  float cap2, cap2_inv;     // cap log2 e
  float near, bend[6];      // products below `near` are bent by s q(s^2)
  // workgroups: `blocks` of rows (or keys), `splits` of the other side, `split_tiles` tiles each
  int blocks, splits, split_tiles, work;
  bool alone;
  uint32_t blocks_magic;
  // forward
  void* o;
  float* lse_out;
  float* part;      // [splits][B,Nq,H][d + 1], the last one lse; null: no splits
  // backward
  float* rowsum;    // [B,Hk,rows] D: <dout, out>, and what that lacks
  float* rowlse;    // [B,Hk,rows] lse in units of log 2; infinity for rows that see no key or are padding: their p is 0
  float* rowrest;   // [splits][B,Hk,rows] what <dout, out> lacks of D, with splits
  float* rowslope;  // [splits][3][H][B,Nq] parts of dslope, or null
  float* part_v;    // (part: dq, or dk: [splits][...][d]; part_v: what D's rest takes from dq, or dv)
  float grad_scale; // scale, sign and all
  void *dq, *dk, *dv;
};

// A tile's rows in LDS, 16-byte pieces.  A piece's place is XORed with bits of its row so that the lanes of a read meet different
// banks: 16 consecutive rows at the same piece, and (bf16) 64 bytes of each of four consecutive rows.
template <typename T, int D, bool ALONE = false>
struct TileRows {
  static constexpr int E = sizeof(T), RB = D * E, PR = RB / 16;
  static constexpr int BN = RB > 256 || (ALONE && RB > 128) ? 32 : 64;  // rows of a tile (ALONE has four of each side in a CU's LDS at least twice)
  static constexpr int kBytes = BN * RB;
  static constexpr int kSteps = PR / 2;  // pairs of pieces of a row: a product's steps over channels
  static constexpr int kBlocks = BN / 32;
  static_assert(kBytes % (16 * kAttnThreads) == 0);
  static __device__ __forceinline__ int mix(int row) {
    if constexpr (E == 4) return (RB == 128 ? row >> 1 : row) & (PR - 1) & 31;
    else if constexpr (RB == 64) return (row >> 2) & 3;
    else if constexpr (RB == 128) return ((row >> 1) & 1) << 2 | ((row >> 2) & 3);
    else return (row & 3) << 2 | ((row >> 2) & 3);
  }
};

// Waves that a kernel's registers are to leave room for on a SIMD: two, but where the vectors of a lane's row alone fill them.
template <typename T, int D>
constexpr int kAttnWaves = sizeof(T) == 4 && D == 128 ? 1 : 2;
// Whether `blocks` workgroups of 128 rows are too few: below one a CU, and with images, whose blocks see more or fewer tiles, below two.
// us of blocks of 128 / of 32, forward and backward, bf16, rows of 1024 tokens: 32 channels 22 / 15 and 51 / 40 with 248 blocks, 22 / 21 and
// 56 / 55 with 384; 64 channels 32 / 25 and 75 / 68 with 248, 27 / 30 and 75 / 83 with 288; 128 channels 42 / 39 and 127 / 140 with 248, 39 / 51
// and 139 / 182 with 288.  With images it depends on their lengths, which the host does not see; rows of 2048 tokens, 496 blocks: 3 images
// 89 / 54 and 163 / 111 (32 channels), 8 images 44 / 34 and 82 / 67 (32) or 51 / 57 and 104 / 130 (64), 24 images 28 / 28 and 52 / 53 (32) or
// 30 / 43 and 63 / 97 (64).  Blocks of 128 win from 288 blocks on where images are many and short, from more than 640 where they are few.
inline bool attn_alone(long long blocks, bool docs) { return blocks < (docs ? 512 : 256); }
inline int attn_tile_rows(int D, int el, bool alone) { return D * el > 256 || (alone && D * el > 128) ? 32 : 64; }
inline int attn_width(int d) { return d <= 32 ? 32 : d <= 64 ? 64 : 128; }  // channels that a kernel is built for

// Blocks of `own` rows (or keys), of 128 or of 32 whose waves share the `other` side out; where these do not fill the chip's 256 CUs twice, the other
// side is split over workgroups too, kAttnLeast of it each at least.
constexpr int kAttnLeast = 256;
struct AttnSide {
  bool alone;
  int blocks, splits, split_tiles;
};
inline AttnSide attn_side(long long own, long long other, long long heads, int D, int el, bool docs) {
  AttnSide s;
  s.alone = attn_alone((own + kAttnRows - 1) / kAttnRows * heads, docs);
  const int BN = attn_tile_rows(D, el, s.alone);
  const int per = s.alone ? 32 : kAttnRows;
  s.blocks = (int)((own + per - 1) / per);
  const int tiles = (int)((other + BN - 1) / BN);
  const long long groups = heads * s.blocks;
  const long long want = std::max(1ll, std::min(512 / groups, other / kAttnLeast));
  s.split_tiles = (int)((tiles + want - 1) / want);
  s.splits = (tiles + s.split_tiles - 1) / s.split_tiles;
  return s;
}

__device__ __forceinline__ int swap23(int m) { return (m & ~12) | (m & 4) << 1 | (m & 8) >> 1; }

// One side's tensor [B,N,heads,d] as the rows of an image and key head.  KEYS: a row is a token; else a (query, head) pair.
template <typename T, int D, bool KEYS>
struct Source {
  using R = TileRows<T, D>;
  const char* first;  // row 0, channel 0
  long long bytes;    // from there to the tensor's end
  uint32_t stride;    // bytes from token to token
  int rows, G, row_bytes;
  uint32_t g_magic;
  const int32_t* doc;  // of the image, or null

  __device__ __forceinline__ Source(const AttnParams& p, const void* tensor, int b, int hk) {
    const int N = KEYS ? p.Nk : p.Nq, heads = KEYS ? p.Hk : p.H, head = KEYS ? hk : hk * p.G;
    const long long skip = (((long long)b * N) * heads + head) * p.d * R::E;
    first = (const char*)tensor + skip;
    bytes = (long long)p.B * N * heads * p.d * R::E - skip;
    stride = (uint32_t)heads * p.d * R::E;
    rows = KEYS ? p.Nk : p.rows;
    G = KEYS ? 1 : p.G;
    g_magic = KEYS ? 0u : p.g_magic;
    row_bytes = p.d * R::E;
    const int32_t* ids = KEYS ? p.k_doc : p.q_doc;
    doc = ids ? ids + (long long)b * N : nullptr;
  }
  __device__ __forceinline__ int token(int r) const { return KEYS ? r : exact_div(r, G, g_magic); }
  // rows r0 .. r0 + BN - 1 into LDS at `dst`, by the workgroup or by a wave; what is not there, and with `pads` rows of padding, as
  // zeros
  template <bool ALONE>
  __device__ __forceinline__ void load(char* dst, int r0, bool pads) const {
    constexpr int kThreads = ALONE ? kWave : kAttnThreads, kTurns = TileRows<T, D, ALONE>::kBytes / 16 / kThreads;
    const int tid = ALONE ? (int)(threadIdx.x & 63) : (int)threadIdx.x;
    const int i0 = token(r0);
    const long long skip = (long long)i0 * stride;
    const i32x4 rsrc = uniform(buffer_of(first + skip, bytes - skip));
    const uint32_t at0 = lds_at(dst) + (ALONE ? 0u : (uint32_t)(__builtin_amdgcn_readfirstlane(threadIdx.x / kWave) * kWave * 16));
    uint32_t off[kTurns];
#pragma unroll
    for (int t = 0; t < kTurns; ++t) {
      const int at = t * kThreads + tid, row = at / R::PR, piece = (at % R::PR) ^ R::mix(row);
      const int r = r0 + row, i = token(r);
      bool there = r < rows && piece * 16 < row_bytes;
      if (pads && there) there = doc[i] >= 0;
      off[t] = there ? (uint32_t)(i - i0) * stride + (uint32_t)((KEYS ? 0 : r - i * G) * row_bytes + piece * 16) : kNowhere;
    }
#pragma unroll
    for (int t = 0; t < kTurns; ++t) lds_load<16>(at0 + t * kThreads * 16, rsrc, off[t]);
  }
};

// 16 bytes of a row: an operand of kSteps steps of a product over channels
template <typename T>
struct Piece;
template <>
struct Piece<bf16_t> {
  bf16x8 x;
  __device__ __forceinline__ void zero() { x = bf16x8{}; }
  __device__ __forceinline__ void negate() {
    u32x4 u = __builtin_bit_cast(u32x4, x);
    u ^= 0x80008000u;
    x = __builtin_bit_cast(bf16x8, u);
  }
  static __device__ __forceinline__ float dot(const Piece& a, const Piece& b) {
    float s = 0.f;
    const u32x4 u = __builtin_bit_cast(u32x4, a.x), w = __builtin_bit_cast(u32x4, b.x);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      s = __builtin_fmaf(__uint_as_float(u[e] << 16), __uint_as_float(w[e] << 16), s);
      s = __builtin_fmaf(__uint_as_float(u[e] & 0xffff0000u), __uint_as_float(w[e] & 0xffff0000u), s);
    }
    return s;
  }
};
template <>
struct Piece<float> {
  f32x4 x;
  __device__ __forceinline__ void zero() { x = f32x4{}; }
  __device__ __forceinline__ void negate() { x = -x; }
  static __device__ __forceinline__ float dot(const Piece& a, const Piece& b) {
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) s = __builtin_fmaf(a.x[e], b.x[e], s);
    return s;
  }
};
__device__ __forceinline__ f32x16 multiply(const Piece<bf16_t>& a, const Piece<bf16_t>& b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.x, b.x, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 multiply(const Piece<float>& a, const Piece<float>& b, f32x16 c) {
#pragma unroll
  for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.x[e], b.x[e], c, 0, 0, 0);
  return c;
}

// The lane's row of the side in registers: piece 2 s + half of step s.
template <typename T, int D>
struct Fixed {
  using R = TileRows<T, D>;
  Piece<T> x[R::kSteps];
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int s = 0; s < R::kSteps; ++s) x[s].zero();
  }
  __device__ __forceinline__ void load(const char* row, int half, int row_bytes) {
#pragma unroll
    for (int s = 0; s < R::kSteps; ++s) {
      x[s].zero();
      const int at = (2 * s + half) * 16;
      if (at < row_bytes) __builtin_memcpy(&x[s], row + at, 16);
    }
  }
  // Waits for them.  (The compiler would wait where they are first used, inside the loop, in every turn of it, and so for the next tile.)
  __device__ __forceinline__ void arrive() {
#pragma unroll
    for (int s = 0; s < R::kSteps; ++s) asm volatile("" : "+v"(x[s].x));
  }
};

// s[m] = <row perm(m) of block `block` in LDS, the row of the lane's column>
template <typename T, int D>
__device__ __forceinline__ void row_products(const char* tile, int block, const Fixed<T, D>& fixed, f32x16& s, int lane, int d) {
  using R = TileRows<T, D>;
  const int row = swap23(lane & 31);
  const char* at = tile + block * 32 * R::RB + row * R::RB;
  const int m = (R::mix(row) ^ (lane >> 5)) << 4;
  s = f32x16{};
#pragma unroll
  for (int step = 0; step < R::kSteps; ++step) {
    if (sizeof(T) == 4 && step > 0 && step * 8 >= d) break;  // (256 cycles a step; of bf16 it is 32, less than a branch between the reads costs)
    Piece<T> a;
    __builtin_memcpy(&a, at + (m ^ (step << 5)), 16);
    s = multiply(a, fixed.x[step], s);
  }
}

// Weights of a block's 32 rows by the lane's column as row_products leaves them (registers i: rows 16 (i / 8) + 8 (lane / 32) + i % 8), as
// the second operand of a product over those rows.
template <typename T>
struct Weights;
template <>
struct Weights<bf16_t> {  // (off by at most 2^-8 of each, what the matrix instructions take; products of bf16 values are exact and sums 32-bit)
  Frag8 w[2];
  __device__ __forceinline__ Weights(const f32x16& x) {
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i >> 2].u[i & 3] = pack_bf16x2(x[2 * i], x[2 * i + 1]);
  }
};
template <>
struct Weights<float> {
  f32x16 w;
  __device__ __forceinline__ Weights(const f32x16& x) : w(x) {}
};

// c[j][column][ch] += sum over the block's rows of tile[row][ch] w[j][column][row], for M sets of weights that share the reads of the tile
template <int D, int M>
__device__ __forceinline__ void column_products(const char* tile, int block, const Weights<bf16_t>* const (&w)[M], f32x16* const (&c)[M], int lane, int) {
  using R = TileRows<bf16_t, D>;
  const int r = lane & 15, half = lane >> 5;
  const int row = 8 * half + (r >> 2);  // + 4 e + 16 t
  const char* at = tile + (block * 32 + row) * R::RB + (r & 1) * 8;
  const int m = (R::mix(row) ^ (2 * ((lane >> 4) & 1) + ((r & 3) >> 1))) << 4;
#pragma unroll
  for (int t = 0; t < 2; ++t)
#pragma unroll
    for (int db = 0; db < D / 32; ++db) {
      Frag8 a;
#pragma unroll
      for (int e = 0; e < 2; ++e) a.u2[e] = lds_read_tr(at + (16 * t + 4 * e) * R::RB + (m ^ (db << 6) ^ (e << 4)));  // (mix has bit 2 of the row in bit 0)
#pragma unroll
      for (int j = 0; j < M; ++j) c[j][db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.v, w[j]->w[t].v, c[j][db], 0, 0, 0);
    }
}
template <int D, int M>
__device__ __forceinline__ void column_products(const char* tile, int block, const Weights<float>* const (&w)[M], f32x16* const (&c)[M], int lane, int d) {
  using R = TileRows<float, D>;
  const int ch = lane & 31, half = lane >> 5;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int row = 16 * (i >> 3) + 8 * half + (i & 7);
    const char* at = tile + (block * 32 + row) * R::RB + (ch & 3) * 4;
#pragma unroll
    for (int db = 0; db < D / 32; ++db) {
      if (db > 0 && 32 * db >= d) break;
      const float a = *reinterpret_cast<const float*>(at + (((8 * db + (ch >> 2)) ^ R::mix(row)) << 4));
#pragma unroll
      for (int j = 0; j < M; ++j) c[j][db] = __builtin_amdgcn_mfma_f32_32x32x2f32(a, w[j]->w[i], c[j][db], 0, 0, 0);
    }
  }
}

// Terms of the scores that a kernel is built for.
enum { kCap = 1, kDistance = 2 };
// tanh x up to |x| = kNear is x times a polynomial of x^2, fitted by least squares to a relative error of 5e-8 (4e-9 for fp32 tensors), beyond
// it 1 - 2 / (exp(2 x) + 1), of which the 1 is most there (near 0 it would leave an error of 1e-7, times the cap).  Caps are many
// times the usual score, so that as a rule no lane of a wave is beyond: then cap tanh(scale s / cap) log2 e is s q(s^2) with the constants
// in q's coefficients, and the second form is not worked out.
constexpr float kNear = 0.55f;
constexpr double kBend16[5] = {-0.33332926, 0.13320038, -0.05261931, 0.01632615, 0.0};
constexpr double kBend32[5] = {-0.33333316, 0.13332534, -0.05384533, 0.02103814, -0.0062211};
template <typename T>
__device__ __forceinline__ float bent_near(float s, const float (&q)[6]) {  // q(s^2)
  const float t = s * s;
  float c = sizeof(T) == 4 ? __builtin_fmaf(t, q[5], q[4]) : q[4];
  c = __builtin_fmaf(t, c, q[3]);
  c = __builtin_fmaf(t, c, q[2]);
  c = __builtin_fmaf(t, c, q[1]);
  return __builtin_fmaf(t, c, q[0]);
}
// no lane has a product of `limit` or more
__device__ __forceinline__ bool all_near(const f32x16& s, float limit) {
  float top = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) top = fmaxf(top, fabsf(s[i]));
  return !__any(!(top < limit));
}
// Score in units of log 2 from a product s, less `from`; bend: the part of it that the cap bends (NEAR: no lane of the wave is beyond).
template <typename T, int TERMS, bool NEAR>
__device__ __forceinline__ float score(float s, const AttnParams& p, float dx, float dy, float slope, float from, float& bend, float& distance) {
  float rest = -from;
  if constexpr (TERMS & kDistance) {
    distance = __builtin_amdgcn_sqrtf(__builtin_fmaf(dx, dx, dy * dy));
    if constexpr (sizeof(T) == 4) {  // (`from` last: it takes most of the value away, and what is left is exact)
      float z = s * p.factor;
      if constexpr (TERMS & kCap) {
        score<T, kCap, NEAR>(s, p, 0.f, 0.f, 0.f, 0.f, bend, z);
        z = bend;
      }
      return __builtin_fmaf(-slope, distance, z) - from;
    }
    rest = __builtin_fmaf(-slope, distance, rest);
  }
  if constexpr (!(TERMS & kCap)) return __builtin_fmaf(s, p.factor, rest);
  const float near = bent_near<T>(s, p.bend);
  if constexpr (NEAR) {
    bend = s * near;
    return __builtin_fmaf(s, near, rest);
  } else {
    const float x = s * p.factor;  // scale / cap
    const float far = p.cap2 - 2.f * p.cap2 * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(x * (2.f * kLog2e)));
    bend = fabsf(s) < p.near ? s * near : far;
    return bend + rest;
  }
}
// 1 - tanh^2, from the bent score
__device__ __forceinline__ float bend_slope(float bend, const AttnParams& p) {
  const float t = bend * p.cap2_inv;
  return __builtin_fmaf(-t, t, 1.f);
}

__device__ __forceinline__ float other_half_max(float x) { return fmaxf(x, __uint_as_float(lane_xor_u32<32>(__float_as_uint(x), threadIdx.x & 63))); }
__device__ __forceinline__ float other_half_sum(float x) { return x + __uint_as_float(lane_xor_u32<32>(__float_as_uint(x), threadIdx.x & 63)); }

// Sums over the four waves: wave w gets those of registers 4 w .. 4 w + 3 of each block of channels.
template <int D>
__device__ __forceinline__ void add_waves(char* lds, int wave, int lane, f32x16 (&c)[D / 32]) {
  f32x4* at = reinterpret_cast<f32x4*>(lds) + lane;  // [wave][block][4][64]
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int g = 0; g < 4; ++g) at[((wave * (D / 32) + db) * 4 + g) * 64] = f32x4{c[db][4 * g], c[db][4 * g + 1], c[db][4 * g + 2], c[db][4 * g + 3]};
  __syncthreads();
#pragma unroll
  for (int db = 0; db < D / 32; ++db) {
    f32x4 s = {};
#pragma unroll
    for (int w = 0; w < 4; ++w) s += at[((w * (D / 32) + db) * 4 + wave) * 64];
#pragma unroll
    for (int g = 0; g < 4; ++g)
      if (g == wave) {
#pragma unroll
        for (int e = 0; e < 4; ++e) c[db][4 * g + e] = s[e];
      }
  }
}

// What a workgroup's own rows (or keys) see of the other side's tiles: all of them, or those that hold a token of one of its images.
struct Walk {
  const Span* spans;  // of the other side's image
  int lo, hi;         // own images
  bool mixed;         // own tokens are not all of one image
  int end, tile_rows, G;
  uint32_t g_magic;
  uint64_t bits;
  int base;
  int tile_lo, tile_hi, tile_pad;  // of tile base + lane

  // own tokens i0 .. i1
  __device__ __forceinline__ void own(const Span* s, int i0, int i1) {
    lo = 0x7fffffff; hi = -1;
    int pad = 0;
    for (int t = i0 / kSpan; t <= i1 / kSpan; ++t) {
      const Span x = s[t];
      lo = min(lo, x.lo);
      hi = max(hi, x.hi);
      pad |= x.pad;
    }
    lo = __builtin_amdgcn_readfirstlane(lo);
    hi = __builtin_amdgcn_readfirstlane(hi);
    mixed = __builtin_amdgcn_readfirstlane((lo != hi || pad) ? 1 : 0);
  }
  // the images of tile t's tokens, rows t tile_rows ... (a tile of at most 64 rows lies in at most two spans)
  __device__ __forceinline__ Span of(int t, int rows) const {
    const int r0 = t * tile_rows, r1 = min(r0 + tile_rows, rows) - 1;
    const int a = exact_div(r0, G, g_magic) / kSpan, b = exact_div(r1, G, g_magic) / kSpan;
    Span x = spans[a];
    if (b != a) {
      const Span y = spans[b];
      x.lo = min(x.lo, y.lo);
      x.hi = max(x.hi, y.hi);
      x.pad |= y.pad;
    }
    return x;
  }
  // whether the tile that next() gave last holds padding, and whether some of its tokens are hidden from some of the own ones
  __device__ __forceinline__ bool padded(int t) const { return __builtin_amdgcn_readlane(tile_pad, t - base); }
  __device__ __forceinline__ bool hides(int t) const {
    return mixed || padded(t) || __builtin_amdgcn_readlane(tile_lo, t - base) != lo || __builtin_amdgcn_readlane(tile_hi, t - base) != lo;
  }
  __device__ __forceinline__ void start(int t) {
    bits = 0;
    base = t - 64;
  }
  // the tile that matters `more` after the next one
  __device__ __forceinline__ int skip(int rows, int more) {
    int t = next(rows);
    for (int i = 0; i < more && t < end; ++i) t = next(rows);
    return t;
  }
  // the next tile that matters, after the one that it gave last; `end`: none
  __device__ __forceinline__ int next(int rows) {
    while (!bits) {
      if (base + 64 >= end) return end;  // (asked again behind the last one, too)
      base += 64;
      const int t = base + (int)(threadIdx.x & 63);
      bool hit = t < end;
      if (spans) {
        tile_lo = 0x7fffffff;
        tile_hi = -1;
        tile_pad = 0;
        if (hit) {
          const Span x = of(t, rows);
          tile_lo = x.lo;
          tile_hi = x.hi;
          tile_pad = x.pad;
          hit = x.lo <= hi && x.hi >= lo;
        }
      }
      bits = __ballot(hit);
    }
    const int at = __builtin_ctzll(bits);
    bits &= bits - 1;
    return base + at;
  }
};

// A wave's 32 rows of the image's problem, one to a lane of either half.
struct Row {
  int r, i, head;   // clamped to the last one
  bool there;
  size_t at;        // (query, head) in [B,Nq,H]
  float x, y, slope;  // slope in units of log 2
  int doc;          // -1: padding
};
__device__ __forceinline__ Row own_row(const AttnParams& p, int b, int hk, int r0) {
  Row w;
  const int r = r0 + (int)(threadIdx.x & 31);
  w.there = r < p.rows;
  w.r = min(r, p.rows - 1);
  w.i = exact_div(w.r, p.G, p.g_magic);
  w.head = hk * p.G + (w.r - w.i * p.G);
  const size_t token = (size_t)b * p.Nq + w.i;
  w.at = token * p.H + w.head;
  w.x = w.y = w.slope = 0.f;
  if (p.slope) {
    const float2 xy = reinterpret_cast<const float2*>(p.q_xy)[token];
    w.x = xy.x;
    w.y = xy.y;
    w.slope = p.slope[w.head] * kLog2e;
  }
  w.doc = p.q_doc ? max(p.q_doc[token], -1) : 0;
  return w;
}

__device__ __forceinline__ void arrive(float& x) { asm volatile("" : "+v"(x)); }
__device__ __forceinline__ void arrive(int& x) { asm volatile("" : "+v"(x)); }
__device__ __forceinline__ void arrive(Row& w) {
  arrive(w.x);
  arrive(w.y);
  arrive(w.slope);
  arrive(w.doc);
}

// Tokens of a tile: places and images, as they are in memory (zeros behind the last one).  They come by loads that the compiler does not
// see, like the tile: behind a load that it sees it would wait for everything on its way, the next tile too, before it uses anything.
struct KeyNotes {
  float x[64], y[64];
  int doc[64];
};
struct KeySource {
  i32x4 xy, doc;
  int rows;
  __device__ __forceinline__ KeySource(const AttnParams& p, int b, bool places, bool images) : rows(p.Nk) {
    if (places) xy = uniform(buffer_of((const char*)(p.k_xy + 2 * (size_t)b * p.Nk), 8ll * p.Nk));
    if (images) doc = uniform(buffer_of((const char*)(p.k_doc + (size_t)b * p.Nk), 4ll * p.Nk));
  }
  // of 64 tokens, whatever a tile has, by one wave, or by waves 0 (places) and 1 (images) of a workgroup.  (All lanes: at the end of a region for a
  // tile's 32 the compiler has put copies of registers where the other lanes were still off, in a kernel that uses all its registers.)
  template <int TERMS, bool DOCS, bool ALONE>
  __device__ __forceinline__ void load(KeyNotes& n, int k0, int wave, int lane) const {
    const int j = k0 + lane;
    if constexpr (TERMS & kDistance)
      if (ALONE || wave == 0) {
        const uint32_t at = j < rows ? (uint32_t)j * 8u : kNowhere;
        lds_load<4>(lds_at(n.x), xy, at);
        lds_load<4>(lds_at(n.y), xy, at + 4);
      }
    if constexpr (DOCS)
      if (ALONE || wave == 1) lds_load<4>(lds_at(n.doc), doc, j < rows ? (uint32_t)j * 4u : kNowhere);
  }
};

hipError_t launch_attn_spans(const AttnArgs& a, Span* q_span, Span* k_span, hipStream_t stream);

inline int attn_spans(int N) { return (N + kSpan - 1) / kSpan; }
inline size_t attn_align(size_t n) { return (n + 255) / 256 * 256; }
inline size_t attn_span_bytes(int B, int Nq, int Nk) { return attn_align((size_t)B * attn_spans(Nq) * sizeof(Span)) + attn_align((size_t)B * attn_spans(Nk) * sizeof(Span)); }

AttnParams attn_params(const AttnArgs& a, Span* spans);
hipError_t launch_attn_bwd_key(const AttnParams& p, int dtype, hipStream_t stream);

}  // namespace affmae
