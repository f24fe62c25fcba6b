// Rotary positions of queries and keys from the tokens' coordinates, on up to three axes: the pair c of every head's channels turns by
// the angle theta(b,n,c) = sum_a coords[b,n,a] freq[c,a],
//     y0 = x0 cos theta - x1 sin theta,  y1 = x0 sin theta + x1 cos theta,
// and, backward, by -theta; d<dy, y> / d theta = y0 dy1 - y1 dy0, which summed over heads and pairs times freq gives dcoords.
//
// Bound by memory: three operations a value.  A thread holds P pairs of a token, works their sines and cosines out once and
// turns those pairs of all the heads, of the queries and of the keys.  131072 tokens of (2 + 2) x 32 bf16 12.1 us (68 MB, 5.6 TB/s, part of it in the
// last-level cache), backward of 98304 x 6 x 64 with dcoords 44 us (228 MB, 5.2 TB/s).
#include "launch.h"
#include "timing.h"

#include "dense_common.h"

#include <algorithm>

namespace affmae {
namespace {

constexpr int kThreads = 256;
constexpr long long kMaxBlocks = 1 << 16;  // (a block takes several turns beyond)

struct RotaryParams {
  const void *q, *k;  // what is turned: the forward's inputs, the gradients of its outputs
  const void *q_out, *k_out;  // backward, for dcoords: the forward's outputs
  const float *coords, *freq;
  void *to_q, *to_k;
  float* dcoords;
  long long tokens;
  int H, Hk, d, A;
  int per;     // threads of a token
  int at_once; // tokens of a block
};

// sin and cos of theta.  A far token's angle does not fit 32 bits (at 10^6 an fp32 angle is off by 0.06): the sum and its
// remainder after quarter turns are 64-bit, pi / 2 in two parts, so that the error of that is theta 2^-53; the rest of at most pi / 4 goes
// through the Taylor series in 32 bits (the terms left out are below 2e-9 and 2.5e-9).
__device__ __forceinline__ void sin_cos(double theta, float& s, float& c) {
  constexpr double kHalfPi = 1.5707963267948966, kRest = 6.123233995736766e-17;  // pi / 2 = 1.57079632679489661923132...
  const double n = __builtin_rint(theta * 0.6366197723675814);
  const float r = (float)__builtin_fma(-n, kRest, __builtin_fma(-n, kHalfPi, theta));
  const int quarter = (int)(n - 4.0 * __builtin_floor(n * 0.25));
  const float z = r * r;
  float p = __builtin_fmaf(z, 2.7557319e-6f, -1.9841270e-4f);
  p = __builtin_fmaf(z, p, 8.3333333e-3f);
  p = __builtin_fmaf(z, p, -1.6666667e-1f);
  const float sr = __builtin_fmaf(r * z, p, r);
  float e = __builtin_fmaf(z, -2.7557319e-7f, 2.4801587e-5f);
  e = __builtin_fmaf(z, e, -1.3888889e-3f);
  e = __builtin_fmaf(z, e, 4.1666667e-2f);
  e = __builtin_fmaf(z, e, -0.5f);
  const float cr = __builtin_fmaf(z, e, 1.f);
  const float a = quarter & 1 ? cr : sr, b = quarter & 1 ? sr : cr;
  s = quarter & 2 ? -a : a;
  c = (quarter + 1) & 2 ? -b : b;
}

// P pairs of a head: beside each other in memory (2 P values), or P values each of the head's two halves
template <bool HALVES, int P, typename T>
__device__ __forceinline__ void load_pairs(const T* p, int half, float (&x)[2 * P]) {
  if constexpr (HALVES) {
    float a[P], b[P];
    load_piece<P>(p, a);
    load_piece<P>(p + half, b);
#pragma unroll
    for (int i = 0; i < P; ++i) x[2 * i] = a[i], x[2 * i + 1] = b[i];
  } else {
    load_piece<2 * P>(p, x);
  }
}
template <bool HALVES, int P, typename T>
__device__ __forceinline__ void store_pairs(T* p, int half, const float (&x)[2 * P]) {
  if constexpr (HALVES) {
    float a[P], b[P];
#pragma unroll
    for (int i = 0; i < P; ++i) a[i] = x[2 * i], b[i] = x[2 * i + 1];
    store_piece<P>(p, a);
    store_piece<P>(p + half, b);
  } else {
    store_piece<2 * P>(p, x);
  }
}

// BWD: turned back.  SPIN: dcoords too.
template <typename T, bool HALVES, int P, bool BWD, bool SPIN>
__global__ __launch_bounds__(kThreads) void rotary_kernel(RotaryParams p) {
  constexpr int U = SPIN ? 2 : 4;  // heads on their way at a time
  __shared__ float part[SPIN ? 3 * kThreads : 1];
  const int slot = (int)threadIdx.x / p.per, c0 = ((int)threadIdx.x - slot * p.per) * P;
  const int half = p.d / 2, first = HALVES ? c0 : 2 * c0, heads = p.H + p.Hk;
  for (long long t0 = (long long)blockIdx.x * p.at_once; t0 < p.tokens; t0 += (long long)gridDim.x * p.at_once) {
    const long long token = t0 + slot;
    const bool there = slot < p.at_once && token < p.tokens;
    float spin[P] = {};
    if (there) {
      double theta[P] = {};
      for (int a = 0; a < p.A; ++a) {
        const double x = (double)p.coords[token * p.A + a];
#pragma unroll
        for (int i = 0; i < P; ++i) theta[i] = __builtin_fma(x, (double)p.freq[(c0 + i) * p.A + a], theta[i]);
      }
      float sn[P], cs[P];
#pragma unroll
      for (int i = 0; i < P; ++i) {
        sin_cos(theta[i], sn[i], cs[i]);
        if (BWD) sn[i] = -sn[i];
      }
      const T* q = (const T*)p.q + token * p.H * p.d + first;
      const T* k = (const T*)p.k + token * p.Hk * p.d + first;
      const T* qo = (const T*)p.q_out + token * p.H * p.d + first;
      const T* ko = (const T*)p.k_out + token * p.Hk * p.d + first;
      T* to_q = (T*)p.to_q + token * p.H * p.d + first;
      T* to_k = (T*)p.to_k + token * p.Hk * p.d + first;
      for (int h0 = 0; h0 < heads; h0 += U) {
        float x[U][2 * P], y[SPIN ? U : 1][2 * P];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int h = h0 + u;
          if (h < heads) {
            load_pairs<HALVES, P>(h < p.H ? q + h * p.d : k + (h - p.H) * p.d, half, x[u]);
            if constexpr (SPIN) load_pairs<HALVES, P>(h < p.H ? qo + h * p.d : ko + (h - p.H) * p.d, half, y[u]);
          }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int h = h0 + u;
          if (h < heads) {
            float o[2 * P];
#pragma unroll
            for (int i = 0; i < P; ++i) {
              const float a = x[u][2 * i], b = x[u][2 * i + 1];
              o[2 * i] = __builtin_fmaf(-b, sn[i], a * cs[i]);
              o[2 * i + 1] = __builtin_fmaf(b, cs[i], a * sn[i]);
              if constexpr (SPIN) spin[i] += __builtin_fmaf(y[u][2 * i], b, -(y[u][2 * i + 1] * a));
            }
            store_pairs<HALVES, P>(h < p.H ? to_q + h * p.d : to_k + (h - p.H) * p.d, half, o);
          }
        }
      }
    }
    if constexpr (SPIN) {  // over the token's threads, in their order
      for (int a = 0; a < p.A; ++a) {
        float s = 0.f;
        if (there) {
#pragma unroll
          for (int i = 0; i < P; ++i) s = __builtin_fmaf(spin[i], p.freq[(c0 + i) * p.A + a], s);
        }
        part[a * kThreads + threadIdx.x] = s;
      }
      __syncthreads();
      const int left = (int)std::min<long long>(p.at_once, p.tokens - t0) * p.A;
      for (int i = threadIdx.x; i < left; i += kThreads) {
        const int at = i / p.A, a = i - at * p.A;
        float s = 0.f;
        for (int j = 0; j < p.per; ++j) s += part[a * kThreads + at * p.per + j];
        p.dcoords[t0 * p.A + i] = s;
      }
      __syncthreads();
    }
  }
}

template <typename T, bool HALVES, int P>
hipError_t launch(const RotaryParams& given, bool backward, hipStream_t stream) {
  RotaryParams p = given;
  p.per = p.d / 2 / P;
  p.at_once = kThreads / p.per;
  const dim3 grid((unsigned)std::min((p.tokens + p.at_once - 1) / p.at_once, kMaxBlocks));
  if (!backward)
    AFFMAE_LAUNCH("rotary_kernel", stream, (rotary_kernel<T, HALVES, P, false, false>), grid, dim3(kThreads), 0, stream, p);
  else if (!p.dcoords)
    AFFMAE_LAUNCH("rotary_bwd_kernel", stream, (rotary_kernel<T, HALVES, P, true, false>), grid, dim3(kThreads), 0, stream, p);
  else
    AFFMAE_LAUNCH("rotary_bwd_kernel", stream, (rotary_kernel<T, HALVES, P, true, true>), grid, dim3(kThreads), 0, stream, p);
  return hipGetLastError();
}

// The widest pieces that a head's pairs divide into, of 16 bytes at most.
template <typename T, bool HALVES>
hipError_t launch_pieces(const RotaryParams& p, bool backward, hipStream_t stream) {
  constexpr int kMost = HALVES ? kPiece<T> : kPiece<T> / 2;
  const int pairs = p.d / 2;
  if constexpr (kMost == 8)
    if (pairs % 8 == 0) return launch<T, HALVES, 8>(p, backward, stream);
  if constexpr (kMost >= 4)
    if (pairs % 4 == 0) return launch<T, HALVES, 4>(p, backward, stream);
  if (pairs % 2 == 0) return launch<T, HALVES, 2>(p, backward, stream);
  return launch<T, HALVES, 1>(p, backward, stream);
}

template <typename T>
hipError_t launch_type(const RotaryParams& p, bool halves, bool backward, hipStream_t stream) {
  return halves ? launch_pieces<T, true>(p, backward, stream) : launch_pieces<T, false>(p, backward, stream);
}

}  // namespace

hipError_t launch_rotary(const RotaryArgs& a, hipStream_t stream) {
  RotaryParams p = {};
  p.q = a.q; p.k = a.k; p.q_out = a.q_out; p.k_out = a.k_out;
  p.coords = a.coords; p.freq = a.freq;
  p.to_q = a.to_q; p.to_k = a.to_k; p.dcoords = a.dcoords;
  p.tokens = (long long)a.B * a.N;
  p.H = a.H; p.Hk = a.Hk; p.d = a.d; p.A = a.axes;
  return a.dtype == 1 ? launch_type<bf16_t>(p, a.halves, a.backward, stream) : launch_type<float>(p, a.halves, a.backward, stream);
}

}  // namespace affmae
