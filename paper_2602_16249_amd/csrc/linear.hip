// Dense layer of the tokens: out = residual + dropout(act(x W^T + bias)), and its gradients dx = dz W, dW = dz^T x,
// dbias = sum of dz, with dz = dropout(dout) act'(pre).
//
// All three are products c[m][n] = sum_k a(m, k) b(n, k) of one tiled kernel; they differ in which operands lie along k in memory:
//   forward  a = x  [rows,Cin]  (along k)     b = W [Cout,Cin] (along k)
//   dx       a = dz [rows,Cout] (along k)     b = W [Cout,Cin] (across: a row of W is one k)
//   dW       a = dz [rows,Cout] (across)      b = x [rows,Cin] (across), k = rows: split over workgroups, parts added by a second launch
// dz is written once, rounded to the tensors' type: bf16 operands are what the matrix instructions take, and an operand in two bf16 parts
// would double both products (16384 x 768 -> 2304 behind gelu: dx and dW 112 of 167 us).  What that costs there: dx and dW are off by 0.00235 of
// their size, with dz unrounded by 0.00166, the rounding of the results.  dbias adds the values before they are rounded.
#include "launch.h"
#include "timing.h"

#include "cluster_common.h"
#include "dense_common.h"
#include "linear_plan.h"

#include <algorithm>

namespace affmae {
namespace {

typedef __attribute__((ext_vector_type(4))) int i32x4;

int cdiv(long long a, long long b) { return (int)((a + b - 1) / b); }

constexpr uint32_t kNowhere = 0x80000000u;  // beyond every buffer: such loads bring 0

// A buffer of at most 2^31 - 1 bytes from `base` on: what lies beyond reads as 0.
__device__ __forceinline__ i32x4 buffer_of(const char* base, long long bytes) {
  const uint64_t p = (uint64_t)base;
  const int n = (int)(bytes < 0 ? 0 : bytes < 0x7fffffffll ? bytes : 0x7fffffffll);
  return i32x4{(int)(uint32_t)p, (int)((uint32_t)(p >> 32) & 0xffffu), n, 0x00020000};
}
__device__ __forceinline__ i32x4 uniform(i32x4 v) {
  return i32x4{__builtin_amdgcn_readfirstlane(v.x), __builtin_amdgcn_readfirstlane(v.y), __builtin_amdgcn_readfirstlane(v.z), __builtin_amdgcn_readfirstlane(v.w)};
}

// From a buffer straight into LDS (lane l's bytes land at dst + W l).  By hand: for the compiler every LDS read might read what
// such a load still writes, and it would wait for what is on its way before it reads what is there.  (The waits: m0 for the load, and five
// states between a vector instruction that writes a scalar of `rsrc` and the load, which the compiler does not see in here.)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"  // (m0 is reserved: written only for the next instruction, never held)
template <int W>
__device__ __forceinline__ void lds_load(uint32_t dst, i32x4 rsrc, uint32_t off) {
  if constexpr (W == 16)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(dst), "v"(off), "s"(rsrc) : "m0", "memory");
  else
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(dst), "v"(off), "s"(rsrc) : "m0", "memory");
}
#pragma clang diagnostic pop
__device__ __forceinline__ uint32_t lds_at(const void* p) { return (uint32_t)(size_t)(__attribute__((address_space(3))) const char*)p; }

template <typename T>
constexpr int kSlice = kSliceBytes / (int)sizeof(T);

// An operand's slice of BX rows in LDS, 16-byte pieces.  ALONG: BX lines of 128 bytes, a line per row; else a line of BX values per k.
// A piece's place in its line is XORed with bits of the line's number, so that the lanes of a read, which take the same piece of
// several lines, meet different banks.
template <typename T, bool ALONG, int BX>
struct SliceLayout {
  static constexpr int kLine = ALONG ? kSliceBytes : BX * (int)sizeof(T);
  static constexpr int kBytes = BX * kSliceBytes;
  static __device__ __forceinline__ int mix(int line) {
    if constexpr (ALONG)
      return line & 7;  // a read takes one piece of 8 lines at a time
    else if constexpr (sizeof(T) == 4)
      return ((line >> 2) & 3) << 2;  // 64 bytes of each of the lines 4 g + j, g = 0..3
    else if constexpr (kLine % 256 == 0)
      return ((line & 3) | ((line >> 3) & 1) << 2) << 1;  // 32 bytes of each of four lines, of lines 8 apart beside them
    else
      return (((line >> 1) & 1) | ((line >> 3) & 1) << 1) << 1;  // (lines of 128 bytes: odd ones are in the other half of the banks)
  }
};

// Brings slices of an operand into LDS.  W: bytes a lane brings at a time.  Rows beyond the operand's and k beyond the last read as 0.
template <typename T, bool ALONG, int BX, int W, int THREADS>
struct Stager {
  using L = SliceLayout<T, ALONG, BX>;
  static constexpr int kTurns = L::kBytes / (W < 4 ? 16 : W) / THREADS;
  static_assert(kTurns * THREADS * (W < 4 ? 16 : W) == L::kBytes);
  const char* first;  // of the tile, k = 0
  long long bytes;    // from there to the end of the operand
  uint32_t ld;
  int x_left;  // rows of the operand from the tile's first on
  uint32_t off[kTurns];

  // which bytes of its line the thread's turn brings, and the line
  static __device__ __forceinline__ void place(int turn, int& line, int& in_line) {
    constexpr int U = W < 4 ? 16 : W;
    const int at = (turn * THREADS + (int)threadIdx.x) * U;
    line = at / L::kLine;
    const int rest = at - line * L::kLine;
    in_line = (((rest >> 4) ^ L::mix(line)) << 4) | (rest & 15);
  }
  __device__ __forceinline__ Stager(const void* p, uint32_t ld_, long long total, int x0, int X) : ld(ld_) {
    const long long skip = ALONG ? (long long)x0 * ld : (long long)x0 * sizeof(T);
    first = (const char*)p + skip;
    bytes = total - skip;
    x_left = X - x0;
#pragma unroll
    for (int t = 0; t < kTurns; ++t) {
      int line, in_line;
      place(t, line, in_line);
      const bool there = ALONG ? line < x_left : in_line < x_left * (int)sizeof(T);
      off[t] = there ? (uint32_t)line * ld + in_line : kNowhere;
    }
  }
  __device__ __forceinline__ long long skip(int k0) const { return ALONG ? (long long)k0 * sizeof(T) : (long long)k0 * ld; }
  // slice of k0 .. k0 + kSlice - 1, `left` of them there, into `dst`
  __device__ __forceinline__ void load(char* dst, int k0, int left) const {
    const i32x4 rsrc = uniform(buffer_of(first + skip(k0), bytes - skip(k0)));
    const uint32_t base = lds_at(dst) + (uint32_t)(__builtin_amdgcn_readfirstlane(threadIdx.x / kWave) * kWave * W);
    if (left >= kSlice<T>) {
#pragma unroll
      for (int t = 0; t < kTurns; ++t) lds_load<W>(base + t * THREADS * W, rsrc, off[t]);
    } else {
#pragma unroll
      for (int t = 0; t < kTurns; ++t) {
        int line, in_line;
        place(t, line, in_line);
        const bool there = ALONG ? in_line < left * (int)sizeof(T) : line < left;
        lds_load<W>(base + t * THREADS * W, rsrc, there ? off[t] : kNowhere);
      }
    }
  }
  // The same through registers, for operands whose rows do not start on 4 bytes: whole pieces wherever they start, value by value where a
  // piece is cut off.  Along k only the last slice has such pieces: the others ask for none of it (17381 x 1725 -> 55, bf16: 38 us, with the
  // checks in every slice 56).
  __device__ __forceinline__ void load_values(char* dst, int k0, int left) const {
    const char* from = first + skip(k0);
    uint4* to = reinterpret_cast<uint4*>(dst) + threadIdx.x;
    const int lines = ALONG ? x_left : left, row = (ALONG ? left : x_left) * (int)sizeof(T);  // there: lines, bytes of each
    const auto some_of = [&](int line, int in_line) {
      T some[kPiece<T>];
#pragma unroll
      for (int e = 0; e < kPiece<T>; ++e)
        some[e] = line < lines && in_line + e * (int)sizeof(T) < row ? reinterpret_cast<const T*>(from + (size_t)line * ld + in_line)[e] : T(0);
      uint4 v;
      __builtin_memcpy(&v, some, 16);
      return v;
    };
    if (ALONG && row < L::kLine) {
#pragma unroll 1
      for (int t = 0; t < kTurns; ++t) {
        int line, in_line;
        place(t, line, in_line);
        to[t * THREADS] = some_of(line, in_line);
      }
      return;
    }
    uint4 v[kTurns];
#pragma unroll
    for (int t = 0; t < kTurns; ++t) {
      int line, in_line;
      place(t, line, in_line);
      v[t] = make_uint4(0u, 0u, 0u, 0u);
      if (line >= lines || in_line >= row) continue;
      if (ALONG || in_line + 16 <= row)
        __builtin_memcpy(&v[t], from + (size_t)line * ld + in_line, 16);
      else
        v[t] = some_of(line, in_line);
    }
#pragma unroll
    for (int t = 0; t < kTurns; ++t) to[t * THREADS] = v[t];
  }
};

// What lane (r = lane % 16, g = lane / 16) hands to the matrix instruction for row r of 16: bf16 k = 8 g .. 8 g + 7 of a step of 32;
// fp32 k = 4 g .. 4 g + 3 of a step of 16, value j to the j-th of four instructions (which k meets which instruction is free as long
// as both operands agree).  (The instructions of 32 x 32 values are faster alone, 2.0 PFLOP/s against 1.26 in bf16, 152 TFLOP/s against 139
// in fp32, but not in these tiles: 16384 x 768 -> 2304 75 us against 67, dx 57 against 55, dW of 16384 x 256 -> 768 in fp32 81 against 73.)
template <typename T>
struct Frag;
template <>
struct Frag<bf16_t> {
  union {
    uint4 u4;
    uint2 u2[2];
    bf16x8 v;
  };
};
template <>
struct Frag<float> {
  union {
    uint4 u4;
    float f[4];
  };
};
__device__ __forceinline__ f32x4 multiply(const Frag<bf16_t>& a, const Frag<bf16_t>& b, f32x4 c, int) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v, b.v, c, 0, 0, 0);
}
// the h-th of the instructions of a step
template <typename T>
constexpr int kStepParts = sizeof(T) == 2 ? 1 : 4;
__device__ __forceinline__ f32x4 multiply(const Frag<float>& a, const Frag<float>& b, f32x4 c, int h) {
  return __builtin_amdgcn_mfma_f32_16x16x4f32(a.f[h], b.f[h], c, 0, 0, 0);
}
template <typename T, bool ALONG, int BX>
__device__ __forceinline__ Frag<T> read_frag(const char* slice, int row0, int step, int r, int g) {
  using L = SliceLayout<T, ALONG, BX>;
  Frag<T> f;
  if constexpr (ALONG) {
    f.u4 = *reinterpret_cast<const uint4*>(slice + (row0 + r) * kSliceBytes + (((4 * step + g) ^ (r & 7)) << 4));
  } else if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int k = 16 * step + 4 * g + j;
      f.f[j] = *reinterpret_cast<const float*>(slice + k * L::kLine + ((((row0 + r) >> 2) ^ (g << 2)) << 4) + (r & 3) * 4);
    }
  } else {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int k = 32 * step + 8 * g + 4 * h + (r >> 2);
      f.u2[h] = lds_read_tr(slice + k * L::kLine + ((((row0 >> 3) + ((r & 3) >> 1)) ^ L::mix(k)) << 4) + (r & 1) * 8);
    }
  }
  return f;
}

struct Operand {
  const void* p;
  uint32_t ld;      // bytes between its lines
  long long bytes;  // of the whole operand
};
struct Product {
  Operand a, b;
  int M, N, K;
  int tiles_n, tiles, splits, split_slices;  // tiles of c; workgroups that share a tile's k, slices of each
  int buffers;  // 1: the next slice comes into a second place in LDS while one is multiplied, 0: into the same, afterwards
};
struct Epilogue {
  const void *bias, *residual;
  void *out, *pre;
  int act;
  Dropout d;
};
struct GradEpilogue {
  void* out;      // [M,N], times alpha
  void* bias;     // [M]: alpha times the sums of a over k, or null
  float* part;    // with splits: [splits][M][part_ld] fp32 instead of out, [splits][M] behind it instead of bias
  int part_ld;
  float alpha;
};

// the first `some` of E values from column n on of a row, the first of them value `at` of the tensor; `even`: rows are whole blocks of 4
template <typename T, int E>
__device__ __forceinline__ void finish(const Epilogue& e, const RngKey& key, float (&v)[E], int some, int n, size_t at, bool even) {
  float r[E];
  if (e.residual) load_some<E>((const T*)e.residual + at, some, r);
  if (e.bias) {
    float b[E];
    load_some<E>((const T*)e.bias + n, some, b);
#pragma unroll
    for (int i = 0; i < E; ++i) v[i] += b[i];
  }
  if (e.pre) store_some<E>((T*)e.pre + at, some, v);
  act_values<sizeof(T) == 2, E>(v, e.act);
  if (e.d.rng) drop<E>(v, e.d, key, at, even);
  if (e.residual) {
#pragma unroll
    for (int i = 0; i < E; ++i) v[i] += r[i];
  }
  store_some<E>((T*)e.out + at, some, v);
}

template <int BM, int BN>
constexpr int kStageBytes = (BM + BN) * kSliceBytes;

// What a wave puts into LDS at a tile's end: strips of 16 rows, all or half of them.
template <int BM, int BN, int WM, int WN>
struct Batch {
  static constexpr int kLd = BN / WN + 4, kAll = BM / WM / 16;
  static constexpr int kStrips = WM * WN * kAll * 16 * kLd * 4 <= 40 * 1024 ? kAll : kAll / 2;
  static constexpr int kFloats = kStrips * 16 * kLd;
  static constexpr int kBytes = WM * WN * kFloats * 4;
};

// BM x BN values of c by WM x WN waves, a slice of both operands in LDS at a time, with p.buffers the next one on its way beside it.
// The products are c^T tiles (b's rows along the instruction's rows), so that a lane holds four consecutive columns of c.
template <typename T, bool AA, bool BA, int W, int BM, int BN, int WM, int WN, typename Ep>
__global__ __launch_bounds__(WM* WN* kWave, 2) void linear_kernel(Product p, Ep e) {
  extern __shared__ __align__(16) char lds[];
  constexpr int kThreads = WM * WN * kWave, TM = BM / WM, TN = BN / WN, IM = TM / 16, IN = TN / 16;
  constexpr bool kGrad = std::is_same_v<Ep, GradEpilogue>, kSums = kGrad && !AA;  // (a's sums: the weights' gradient)
  const int work = xcd_contiguous_block(blockIdx.x, gridDim.x);
  if (work >= p.tiles * p.splits) return;
  const int split = work / p.tiles, tile = work - split * p.tiles;
  const int mt = tile / p.tiles_n, nt = tile - mt * p.tiles_n;
  const int m0 = mt * BM, n0 = nt * BN;
  const int k_begin = split * p.split_slices * kSlice<T>;
  const int k_end = min(p.K, k_begin + p.split_slices * kSlice<T>);
  const int slices = (k_end - k_begin + kSlice<T> - 1) / kSlice<T>;
  const int lane = threadIdx.x & (kWave - 1), r = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), wm = wave / WN, wn = wave % WN;
  const Stager<T, AA, BM, W, kThreads> sa(p.a.p, p.a.ld, p.a.bytes, m0, p.M);
  const Stager<T, BA, BN, W, kThreads> sb(p.b.p, p.b.ld, p.b.bytes, n0, p.N);
  const auto stage = [&](int s) {
    char* dst = lds + (s & p.buffers) * kStageBytes<BM, BN>;
    const int k0 = k_begin + s * kSlice<T>;
    if constexpr (W >= 4) {
      sa.load(dst, k0, k_end - k0);
      sb.load(dst + BM * kSliceBytes, k0, k_end - k0);
    } else {
      sa.load_values(dst, k0, k_end - k0);
      sb.load_values(dst + BM * kSliceBytes, k0, k_end - k0);
    }
  };
  f32x4 c[IM][IN] = {}, sums[kSums ? IM : 1] = {};
  bool want_sums = false;
  if constexpr (kSums) want_sums = e.bias && nt == 0 && wn == 0;
  stage(0);
  for (int s = 0; s < slices; ++s) {
    // slice s has arrived, and every wave has read what the next one will be written over
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    if (p.buffers && s + 1 < slices) stage(s + 1);
    const char* as = lds + (s & p.buffers) * kStageBytes<BM, BN>;
    const char* bs = as + BM * kSliceBytes;
#pragma unroll
    for (int step = 0; step < 2; ++step) {
      Frag<T> a[IM], b[IN];
#pragma unroll
      for (int i = 0; i < IM; ++i) a[i] = read_frag<T, AA, BM>(as, wm * TM + 16 * i, step, r, g);
#pragma unroll
      for (int j = 0; j < IN; ++j) b[j] = read_frag<T, BA, BN>(bs, wn * TN + 16 * j, step, r, g);
#pragma unroll
      for (int h = 0; h < kStepParts<T>; ++h)  // (instructions that add to the same registers far from each other)
#pragma unroll
        for (int i = 0; i < IM; ++i)
#pragma unroll
          for (int j = 0; j < IN; ++j) c[i][j] = multiply(b[j], a[i], c[i][j], h);
      if constexpr (kSums) {
        if (want_sums) {  // a's sums over k: its products with ones
          Frag<T> ones;
          ones.u4 = sizeof(T) == 2 ? make_uint4(0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u)
                                   : make_uint4(0x3f800000u, 0x3f800000u, 0x3f800000u, 0x3f800000u);
#pragma unroll
          for (int h = 0; h < kStepParts<T>; ++h)
#pragma unroll
            for (int i = 0; i < IM; ++i) sums[i] = multiply(ones, a[i], sums[i], h);
        }
      }
    }
    if (!p.buffers && s + 1 < slices) {
      asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
      stage(s + 1);
    }
  }
  // A wave's values go through LDS, a batch of strips of 16 rows at a time, and leave as pieces in the order of memory, by a loop that is
  // not unrolled: with the epilogue's code once for every strip, 65536 x 256 -> 256 took 30.6 us with gelu and 24.8 with relu, so it takes
  // 27.4 and 23.1.
  __syncthreads();
  using B = Batch<BM, BN, WM, WN>;
  float* batch = reinterpret_cast<float*>(lds) + wave * B::kFloats;
  if constexpr (kSums) {
    if (want_sums) {
#pragma unroll
      for (int i = 0; i < IM; ++i) {
        const int m = m0 + wm * TM + 16 * i + r;
        if (g != 0 || m >= p.M) continue;
        if (e.part)
          e.part[(size_t)p.splits * p.M * e.part_ld + (size_t)split * p.M + m] = sums[i][0];
        else
          Elem<T>::store((T*)e.bias + m, sums[i][0] * e.alpha);
      }
    }
  }
#pragma unroll
  for (int first = 0; first < IM; first += B::kStrips) {
    const int m = m0 + wm * TM + 16 * first, n = n0 + wn * TN;
    if (m >= p.M || n >= p.N) break;
    wave_lds_sync();
#pragma unroll
    for (int i = 0; i < B::kStrips; ++i)
#pragma unroll
      for (int j = 0; j < IN; ++j) *reinterpret_cast<f32x4*>(batch + (16 * i + r) * B::kLd + 16 * j + 4 * g) = c[first + i][j];
    wave_lds_sync();
    // f(row and column in the batch) for the lane's pieces of E values inside M x N
    const auto pieces = [&](auto piece, int N, auto f) __attribute__((always_inline)) {
      constexpr int E = decltype(piece)::value, kRow = TN / E;
      const int all = min(16 * B::kStrips, p.M - m) * kRow;
#pragma unroll 1
      for (int q = lane; q < all; q += kWave) {
        const int row = q / kRow, col = q % kRow * E;
        if (n + col < N) f(row, col);
      }
    };
    using std::integral_constant;
    constexpr int E = kPiece<T>;
    if constexpr (kGrad) {
      // `whole`: rows are whole pieces
      const auto put = [&](auto* out, auto piece, int N, auto whole) __attribute__((always_inline)) {
        constexpr int E = decltype(piece)::value;
        pieces(piece, N, [&](int row, int col) {
          float v[E];
          load_row<E>(batch + row * B::kLd + col, v);
#pragma unroll
          for (int x = 0; x < E; ++x) v[x] *= e.alpha;
          store_some<E>(out + (size_t)(m + row) * N + n + col, whole ? E : min(E, N - n - col), v);
        });
      };
      if (e.part)  // (alpha is 1)
        put(e.part + (size_t)split * p.M * e.part_ld, integral_constant<int, 4>(), e.part_ld, std::true_type());
      else if (p.N % E == 0)
        put((T*)e.out, integral_constant<int, E>(), p.N, std::true_type());
      else
        put((T*)e.out, integral_constant<int, E>(), p.N, std::false_type());
    } else {
      RngKey key = {};
      if (e.d.rng) key = rng_key(e.d.rng);
      const auto put = [&](auto whole) __attribute__((always_inline)) {
        pieces(integral_constant<int, E>(), p.N, [&](int row, int col) {
          float v[E];
          load_row<E>(batch + row * B::kLd + col, v);
          finish<T, E>(e, key, v, whole ? E : min(E, p.N - n - col), n + col, (size_t)(m + row) * p.N + n + col, whole || p.N % 4 == 0);
        });
      };
      if (p.N % E == 0)
        put(std::true_type());
      else
        put(std::false_type());
    }
  }
}

// Forward products of few rows and columns: 16 x 16 values of c a workgroup, the waves share k between them, operands straight from
// memory into registers.  A tile of 64 x 64 would leave most of the chip without work and walk k alone, one round trip to memory per
// slice: 64 rows, 2304 -> 768 in bf16, 27.6 us with tiles of 128 x 128, 7.3 so.
constexpr int kSlim = 16, kSlimWaves = 8;
template <typename T>
__global__ __launch_bounds__(kSlimWaves* kWave) void linear_slim_kernel(Product p, Epilogue e) {
  __shared__ __align__(16) float parts[kSlimWaves][kSlim * kSlim];
  constexpr int kStep = kSlice<T> / 2;
  const int mt = blockIdx.x / p.tiles_n, nt = blockIdx.x - mt * p.tiles_n;
  const int lane = threadIdx.x & (kWave - 1), r = lane & 15, g = lane >> 4, wave = threadIdx.x / kWave;
  // (rows beyond the last repeat it: their values go nowhere)
  const char* a = (const char*)p.a.p + (size_t)min(mt * kSlim + r, p.M - 1) * p.a.ld;
  const char* b = (const char*)p.b.p + (size_t)min(nt * kSlim + r, p.N - 1) * p.b.ld;
  const int begin = min(p.K, wave * p.split_slices * kStep), end = min(p.K, begin + p.split_slices * kStep);
  f32x4 c = {};
  constexpr int kAhead = 6;  // steps on their way at a time
  for (int k0 = begin; k0 < end; k0 += kAhead * kStep) {
    Frag<T> fa[kAhead], fb[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int k = k0 + i * kStep + g * kPiece<T>;
      fa[i].u4 = fb[i].u4 = make_uint4(0u, 0u, 0u, 0u);
      if (k < end) {  // (lines are whole pieces)
        fa[i].u4 = *reinterpret_cast<const uint4*>(a + (size_t)k * sizeof(T));
        fb[i].u4 = *reinterpret_cast<const uint4*>(b + (size_t)k * sizeof(T));
      }
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
#pragma unroll
      for (int h = 0; h < kStepParts<T>; ++h) c = multiply(fb[i], fa[i], c, h);
  }
  *reinterpret_cast<f32x4*>(&parts[wave][r * kSlim + 4 * g]) = c;
  __syncthreads();
  if (threadIdx.x >= kSlim * kSlim) return;
  float v[1] = {0.f};
#pragma unroll
  for (int w = 0; w < kSlimWaves; ++w) v[0] += parts[w][threadIdx.x];
  const int m = mt * kSlim + threadIdx.x / kSlim, n = nt * kSlim + threadIdx.x % kSlim;
  if (m >= p.M || n >= p.N) return;
  const size_t at = (size_t)m * p.N + n;
  RngKey key = {};
  if (e.d.rng) key = rng_key(e.d.rng);
  finish<T, 1>(e, key, v, 1, n, at, true);
}

// out[i] = alpha * (part[0][i] + part[1][i] + ...), rows of N in part_ld, LANES threads a piece of four; the last workgroups: bias
// likewise, of bias_part.  (A thread that adds all parts of its piece waits for them one after another where there are many: 94 parts of 301 x 100 took
// 27 us.)
template <typename T, int LANES>
__global__ __launch_bounds__(256) void linear_join_kernel(GradEpilogue e, int M, int N, int splits, float alpha, int bias_blocks, const float* bias_part,
                                                          int bias_parts) {
  constexpr int kPieces = 256 / LANES;
  __shared__ float4 sums[LANES > 1 ? 256 : 1];
  const int blocks = gridDim.x - bias_blocks;
  if ((int)blockIdx.x >= blocks) {  // 16 values a workgroup, 16 threads each
    const int m = (blockIdx.x - blocks) * 16 + (threadIdx.x & 15), run = threadIdx.x >> 4;
    float s = 0.f;
    if (m < M) {
#pragma unroll 8
      for (int k = run; k < bias_parts; k += 16) s += bias_part[(size_t)k * M + m];
    }
    __shared__ float all[16][17];
    all[run][threadIdx.x & 15] = s;
    __syncthreads();
    if (run != 0 || m >= M) return;
    s = 0.f;
#pragma unroll
    for (int k = 0; k < 16; ++k) s += all[k][threadIdx.x];
    Elem<T>::store((T*)e.bias + m, s * alpha);
    return;
  }
  const size_t all = (size_t)M * e.part_ld;
  const int run = threadIdx.x / kPieces;
  for (size_t first = (size_t)blockIdx.x * kPieces * 4; first < all; first += (size_t)blocks * kPieces * 4) {
    const size_t i = first + threadIdx.x % kPieces * 4;
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    if (i < all) {
#pragma unroll 4
      for (int k = run; k < splits; k += LANES) {
        const float4 v = *reinterpret_cast<const float4*>(e.part + k * all + i);
        s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
      }
    }
    if constexpr (LANES > 1) {
      __syncthreads();
      sums[threadIdx.x] = s;
      __syncthreads();
      if (run != 0) continue;
#pragma unroll
      for (int k = 1; k < LANES; ++k) {
        const float4 v = sums[k * kPieces + threadIdx.x];
        s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
      }
    }
    if (i >= all) continue;
    const size_t m = i / (unsigned)e.part_ld;
    const int n = (int)(i - m * e.part_ld);
    T* out = (T*)e.out + m * N + n;
    const float v[4] = {s.x * alpha, s.y * alpha, s.z * alpha, s.w * alpha};
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (n + j < N) Elem<T>::store(out + j, v[j]);
  }
}

// dz / factor = (kept? dout : 0) act'(pre), rows of C in lines of `ld` values whose rest is 0.  A thread takes a piece of dout in the
// order of memory, whatever rows it is part of, so that odd rows cost neither wide loads nor blocks of the generator.  EVEN: C is a
// multiple of a piece, hence ld.  (Without pre and mask: a copy in such lines.)
template <typename T, bool EVEN>
__global__ __launch_bounds__(256) void linear_dz_kernel(const T* __restrict__ dout, const T* __restrict__ pre, int rows, int C, int ld, uint32_t magic, int act,
                                                        Dropout d, T* __restrict__ dz) {
  constexpr int E = kPiece<T>;
  RngKey key = {};
  if (d.rng) key = rng_key(d.rng);
  d.factor = 1.f;
  const long long all = (long long)rows * C;
  for (long long first = (long long)blockIdx.x * 256 * E; first < all; first += (long long)gridDim.x * 256 * E) {
    const long long i = first + threadIdx.x * E;
    const int n = (int)std::min<long long>(all - i, E);
    if (n <= 0) break;
    float v[E], z[E];
    load_some<E>(dout + i, n, v);
    if (pre) load_some<E>(pre + i, n, z);
    if (d.rng) drop<E>(v, d, key, (uint64_t)i, true);
    if (pre) act_slopes<sizeof(T) == 2, E>(v, z, act);
    if constexpr (EVEN) {
      store_piece<E>(dz + i, v);
    } else {
      const long long row0 = first / C;  // (of the workgroup: one long division, short ones from there)
      const int from = (int)(first - row0 * C) + (int)threadIdx.x * E;
      int row = exact_div(from, C, magic), col = from - row * C;
      T* to = dz + (size_t)(row0 + row) * ld;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        if (e >= n) break;
        Elem<T>::store(to + col, v[e]);
        if (++col == C) {
          for (int x = C; x < ld; ++x) Elem<T>::store(to + x, 0.f);
          to += ld;
          col = 0;
        }
      }
    }
  }
}

// The same for bf16 with the sums of dz over a run of rows, part [runs][C]: of the values before they are rounded for the products, since the
// bias' gradient is the only one that adds them up bare (1024 x 64 -> 192: off by 0.0029 of its size with rounded ones, by 0.0017 so).  A
// thread takes one column of pieces, `lanes` of them over each other, every lanes-th row.
struct Runs {
  int cols, lanes, blocks;  // columns of a workgroup, threads of one, workgroups of a row
  int rows, count;          // of a run, runs
};
template <bool EVEN>
__global__ __launch_bounds__(256) void linear_dz_sums_kernel(const bf16_t* __restrict__ dout, const bf16_t* __restrict__ pre, int rows, int C, int ld, Runs k,
                                                             uint32_t cols_magic, int act, Dropout d, bf16_t* __restrict__ dz, float* __restrict__ part) {
  constexpr int E = kPiece<bf16_t>;
  __shared__ float sums[256 * E];
  RngKey key = {};
  if (d.rng) key = rng_key(d.rng);
  d.factor = 1.f;
  const int run = blockIdx.x / k.blocks, block = blockIdx.x - run * k.blocks;
  const int lane = exact_div(threadIdx.x, k.cols, cols_magic), col = threadIdx.x - lane * k.cols;
  const int c0 = block * k.cols * E, c = c0 + col * E, n = C - c, some = EVEN ? E : n;
  const int end = std::min(rows, (run + 1) * k.rows);
  float db[E] = {};
  if (lane < k.lanes && n > 0) {
#pragma unroll 4
    for (int row = run * k.rows + lane; row < end; row += k.lanes) {
      const long long at = (long long)row * C + c;
      float v[E], z[E];
      load_some<E>(dout + at, some, v);
      if (pre) load_some<E>(pre + at, some, z);
      if (d.rng) drop<E>(v, d, key, (uint64_t)at, EVEN || C % 4 == 0);
      if (pre) act_slopes<true, E>(v, z, act);
#pragma unroll
      for (int e = 0; e < E; ++e) db[e] += v[e];
      store_piece<E>(dz + (size_t)row * ld + c, v);
    }
  }
#pragma unroll
  for (int e = 0; e < E; ++e) sums[threadIdx.x * E + e] = db[e];
  __syncthreads();
  for (int i = threadIdx.x; i < k.cols * E && c0 + i < C; i += 256) {
    float s = 0.f;
    for (int l = 0; l < k.lanes; ++l) s += sums[l * k.cols * E + i];
    part[(size_t)run * C + c0 + i] = s;
  }
}
// Columns in blocks of at most 32 pieces, which fill a workgroup (blocks of 144, of 256 threads 112 idle: 63 us of 16384 x 2304 instead of 45);
// about 6144 workgroups, of at least four turns.
Runs runs_of(int rows, int C) {
  Runs k;
  const int pieces = cdiv(C, kPiece<bf16_t>);
  k.blocks = cdiv(pieces, 32);
  k.cols = cdiv(pieces, k.blocks);
  k.blocks = cdiv(pieces, k.cols);
  k.lanes = 256 / k.cols;
  k.rows = std::max(4 * k.lanes, cdiv(rows, std::max(1, 6144 / k.blocks)));
  k.count = cdiv(rows, k.rows);
  return k;
}

// what a lane may bring at a time, by where an operand's lines start
int line_bytes(const Operand& o) {
  const uintptr_t all = reinterpret_cast<uintptr_t>(o.p) | o.ld;
  return all % 16 == 0 ? 16 : all % 4 == 0 ? 4 : 2;
}

template <typename T, bool AA, bool BA, int W, int BM, int BN, int WM, int WN, typename Ep>
hipError_t run_tiles(Product p, const Ep& e, hipStream_t stream) {
  p.tiles_n = cdiv(p.N, BN);
  p.tiles = cdiv(p.M, BM) * p.tiles_n;
  const int slices = cdiv(p.K, kSlice<T>);
  p.split_slices = cdiv(slices, p.splits);
  // A second place for a slice hides its way from memory; without it twice the workgroups fit a CU and hide each other's.  The latter
  // pays in forward products that have several for every CU and are not deep: 65536 x 256 -> 256 20.0 us against 23.1, 16384 x 768 -> 2304
  // 67 against 74, but 16384 x 2304 -> 768 63 against 61, 4096 x 768 -> 768 13.5 against 12.5, dx of 16384 x 768 -> 2304 59 against 55; fp32: no difference.
  const bool crowded = std::is_same_v<Ep, Epilogue> && sizeof(T) == 2 && p.split_slices <= 16 && p.tiles >= 2 * kCus;
  p.buffers = p.split_slices > 1 && (!crowded || W < 4);
  const auto kernel = linear_kernel<T, AA, BA, W, BM, BN, WM, WN, Ep>;
  const size_t lds = (size_t)std::max((1 + p.buffers) * kStageBytes<BM, BN>, Batch<BM, BN, WM, WN>::kBytes);
  if (lds > 64 * 1024) {
    const hipError_t rc = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (rc != hipSuccess) return rc;
  }
  const unsigned grid = (unsigned)cdiv((long long)p.tiles * p.splits, 8) * 8;
  [[maybe_unused]] constexpr const char* name = std::is_same_v<Ep, Epilogue> ? "linear_fwd_kernel" : AA ? "linear_dx_kernel" : "linear_dweight_kernel";
  AFFMAE_LAUNCH(name, stream, kernel, dim3(grid), dim3(WM * WN * kWave), lds, stream, p, e);
  return hipGetLastError();
}

template <typename T>
hipError_t run_slim(Product p, const Epilogue& e, hipStream_t stream) {
  p.tiles_n = cdiv(p.N, kSlim);
  p.split_slices = cdiv(cdiv(p.K, kSlice<T> / 2), kSlimWaves);  // (steps of a wave)
  AFFMAE_LAUNCH("linear_slim_kernel", stream, linear_slim_kernel<T>, dim3(cdiv(p.M, kSlim) * p.tiles_n), dim3(kSlimWaves * kWave), 0, stream, p, e);
  return hipGetLastError();
}

template <typename T, bool AA, bool BA, typename Ep>
hipError_t run_product(Product p, int shape, const Ep& e, hipStream_t stream) {
  const int w = std::min(line_bytes(p.a), line_bytes(p.b));
  if (w == 16) {
    if constexpr (std::is_same_v<Ep, Epilogue>) {
      if (shape == kSlimTile) return run_slim<T>(p, e, stream);
    }
    if constexpr (sizeof(T) == 2) {
      if (shape == k128x192) return run_tiles<T, AA, BA, 16, 128, 192, 2, 2>(p, e, stream);
      if (shape == k128x128) return run_tiles<T, AA, BA, 16, 128, 128, 2, 2>(p, e, stream);
    }
    if (shape == k128x64) return run_tiles<T, AA, BA, 16, 128, 64, 2, 2>(p, e, stream);
    return run_tiles<T, AA, BA, 16, 64, 64, 2, 2>(p, e, stream);
  }
  if constexpr (sizeof(T) == 2) {
    if (w == 4 && shape == k128x128) return run_tiles<T, AA, BA, 4, 128, 128, 2, 2>(p, e, stream);
    if (w == 2) {
      if (shape == k128x128) return run_tiles<T, AA, BA, 2, 128, 128, 2, 2>(p, e, stream);
      return shape == k128x64 ? run_tiles<T, AA, BA, 2, 128, 64, 2, 2>(p, e, stream) : run_tiles<T, AA, BA, 2, 64, 64, 2, 2>(p, e, stream);
    }
  }
  return shape == k128x64 ? run_tiles<T, AA, BA, 4, 128, 64, 2, 2>(p, e, stream) : run_tiles<T, AA, BA, 4, 64, 64, 2, 2>(p, e, stream);
}

int part_ld(int N) { return cdiv(N, 4) * 4; }
size_t part_bytes(int splits, int M, int N, bool bias) {
  return splits > 1 ? ((size_t)splits * M * part_ld(N) + (bias ? (size_t)splits * M : 0)) * sizeof(float) : 0;
}
size_t up256(size_t n) { return (n + 255) / 256 * 256; }

template <typename T>
hipError_t gradient(bool dx, Operand a, Operand b, int M, int N, int K, void* out, void* bias, const float* bias_part, int bias_parts, float alpha,
                    float* part, hipStream_t stream) {
  const Plan plan = plan_product(M, N, K, sizeof(T), std::min(line_bytes(a), line_bytes(b)), false);
  Product p = {};
  p.a = a; p.b = b; p.M = M; p.N = N; p.K = K; p.splits = plan.splits;
  GradEpilogue e = {out, bias_part ? nullptr : bias, p.splits > 1 ? part : nullptr, part_ld(N), p.splits > 1 ? 1.f : alpha};
  hipError_t rc = dx ? run_product<T, true, false>(p, plan.shape, e, stream) : run_product<T, false, false>(p, plan.shape, e, stream);
  if (rc != hipSuccess || (p.splits == 1 && !bias_part)) return rc;
  const int bias_blocks = bias ? cdiv(M, 16) : 0;
  if (!bias_part) {
    bias_part = part + (size_t)p.splits * M * e.part_ld;
    bias_parts = p.splits;
  }
  e.bias = bias;
  const long long pieces = p.splits > 1 ? (long long)M * (part_ld(N) / 4) : 0;
  const auto join = [&](auto lanes) {
    constexpr int L = decltype(lanes)::value;
    const int blocks = (int)std::min<long long>(cdiv(pieces * L, 256), 4096);
    AFFMAE_LAUNCH("linear_join_kernel", stream, (linear_join_kernel<T, L>), dim3(blocks + bias_blocks), dim3(256), 0, stream, e, M, N, p.splits, alpha, bias_blocks,
                  bias_part, bias_parts);
  };
  if (pieces <= 8192 && p.splits > 16)
    join(std::integral_constant<int, 16>());
  else if (pieces <= 32768 && p.splits > 4)
    join(std::integral_constant<int, 4>());
  else
    join(std::integral_constant<int, 1>());
  return hipGetLastError();
}

template <typename T>
hipError_t fwd(const LinearArgs& a, hipStream_t stream) {
  const uint32_t ld = (uint32_t)a.Cin * sizeof(T);
  Product p = {};
  p.a = {a.x, ld, (long long)a.rows * ld};
  p.b = {a.weight, ld, (long long)a.Cout * ld};
  p.M = a.rows; p.N = a.Cout; p.K = a.Cin; p.splits = 1;
  const Epilogue e = {a.bias, a.residual, a.out, a.pre_out, a.act, make_dropout(a.p, a.rng)};
  const Plan plan = plan_product(p.M, p.N, p.K, sizeof(T), std::min(line_bytes(p.a), line_bytes(p.b)), true);
  return run_product<T, true, true>(p, plan.shape, e, stream);
}

size_t copy_bytes(int rows, int C, int el) { return up256((size_t)rows * padded(C, el) * el); }

template <typename T>
hipError_t bwd(const LinearArgs& a, hipStream_t stream) {
  const Dropout d = make_dropout(a.p, a.rng);
  constexpr int el = sizeof(T), E = kPiece<T>;
  const auto operand = [](const void* p, int rows, int ld) { return Operand{p, (uint32_t)ld * el, (long long)rows * ld * el}; };
  Operand dz = operand(a.dout, a.rows, a.Cout), x = operand(a.x, a.rows, a.Cin), weight = operand(a.weight, a.Cout, a.Cin);
  char* ws = static_cast<char*>(a.workspace);
  const auto write = [&](Operand& o, const void* from, const void* pre, int rows, int C, int act, Dropout drop) {
    const int ld = padded(C, el);
    const auto kernel = C % E == 0 ? linear_dz_kernel<T, true> : linear_dz_kernel<T, false>;
    const dim3 grid((unsigned)std::min<long long>(cdiv((long long)rows * C, 256 * E), kMaxBlocks));
    AFFMAE_LAUNCH("linear_dz_kernel", stream, kernel, grid, dim3(256), 0, stream, (const T*)from, (const T*)pre, rows, C, ld, div_magic(C), act, drop, (T*)ws);
    o = operand(ws, rows, ld);
    ws += copy_bytes(rows, C, el);
  };
  const Copies c = copies(a.rows, a.Cin, a.Cout, a.act != kActNone || d.rng, a.dx != nullptr, a.dweight != nullptr, el);
  const Dropout none = make_dropout(0.f, nullptr);
  const void* pre = a.act != kActNone ? a.pre : nullptr;
  const float* sums = nullptr;
  int runs = 0;
  if (sizeof(T) == 2 && (pre || d.rng) && a.dbias) {
    const Runs k = runs_of(a.rows, a.Cout);
    const int ld = padded(a.Cout, el);
    float* to = reinterpret_cast<float*>(ws + copy_bytes(a.rows, a.Cout, el));
    const auto kernel = a.Cout % E == 0 ? linear_dz_sums_kernel<true> : linear_dz_sums_kernel<false>;
    AFFMAE_LAUNCH("linear_dz_kernel", stream, kernel, dim3((unsigned)k.count * k.blocks), dim3(256), 0, stream, (const bf16_t*)a.dout,
                  (const bf16_t*)pre, a.rows, a.Cout, ld, k, div_magic(k.cols), a.act, d, (bf16_t*)ws, to);
    dz = operand(ws, a.rows, ld);
    sums = to;
    runs = k.count;
    ws += copy_bytes(a.rows, a.Cout, el) + up256((size_t)runs * a.Cout * sizeof(float));
  } else if (c.dz) {
    write(dz, a.dout, pre, a.rows, a.Cout, a.act, d);
  }
  if (c.x) write(x, a.x, nullptr, a.rows, a.Cin, kActNone, none);
  if (c.weight) write(weight, a.weight, nullptr, a.Cout, a.Cin, kActNone, none);
  const hipError_t launched = hipGetLastError();
  if (launched != hipSuccess) return launched;
  float* part = reinterpret_cast<float*>(ws);
  if (a.dx) {
    const hipError_t rc = gradient<T>(true, dz, weight, a.rows, a.Cin, a.Cout, a.dx, nullptr, nullptr, 0, d.factor, part, stream);
    if (rc != hipSuccess) return rc;
  }
  if (a.dweight)
    return gradient<T>(false, dz, x, a.Cout, a.Cin, a.rows, a.dweight, a.dbias, sums, runs, d.factor, part, stream);
  return hipSuccess;
}

}  // namespace

size_t linear_bwd_workspace_bytes(int rows, int Cin, int Cout, int act, bool drops, int dtype, bool want_dx, bool want_dweight) {
  const int el = dtype == 1 ? 2 : 4;
  const bool made = act != kActNone || drops;
  const Copies c = copies(rows, Cin, Cout, made, want_dx, want_dweight, el);
  const size_t sums = el == 2 && made && want_dweight ? up256((size_t)runs_of(rows, Cout).count * Cout * sizeof(float)) : 0;
  const size_t written = sums + (c.dz ? copy_bytes(rows, Cout, el) : 0) + (c.x ? copy_bytes(rows, Cin, el) : 0) + (c.weight ? copy_bytes(Cout, Cin, el) : 0);
  // (which tile a call takes, hence how it splits, depends on its tensors' alignment)
  const auto parts = [&](int M, int N, int K, bool bias) {
    return std::max(part_bytes(plan_product(M, N, K, el, 16, false).splits, M, N, bias), part_bytes(plan_product(M, N, K, el, 2, false).splits, M, N, bias));
  };
  const size_t dx = want_dx ? parts(rows, Cin, Cout, false) : 0;
  const size_t dw = want_dweight ? parts(Cout, Cin, rows, true) : 0;
  return written + std::max(dx, dw);  // (the parts of one are joined before the other's are written)
}
hipError_t launch_linear_fwd(const LinearArgs& a, hipStream_t stream) { return a.dtype == 1 ? fwd<bf16_t>(a, stream) : fwd<float>(a, stream); }
hipError_t launch_linear_bwd(const LinearArgs& a, hipStream_t stream) { return a.dtype == 1 ? bwd<bf16_t>(a, stream) : bwd<float>(a, stream); }

}  // namespace affmae
