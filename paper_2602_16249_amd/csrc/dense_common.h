// What the dense operators share (linear.hip, norm.hip, dropout.hip): storage of 16-byte pieces, activations, and the
// counter-based generator behind dropout.
#pragma once

#include "device_util.h"

#include <type_traits>

namespace affmae {

enum Act { kActNone = 0, kActRelu = 1, kActGelu = 2, kActSilu = 3 };

// Phi(z) and phi(z) of the normal distribution.  Phi(-|z|) exp(z^2 / 2) is smooth and nearly algebraic in |z|: t = 1 / (1 + c |z|) times a
// polynomial in t, fitted by least squares weighted towards the largest relative error up to |z| = 14.5, where exp(-z^2 / 2) is below the
// least fp32.  The error is relative, also in the tail, where the published short forms of erf have an absolute one (1.5e-7: gelu(-5)
// off by 1.6e-3 of itself).
//   ten terms (c = 3/8): 4e-8 with coefficients of fp32; an error of t counts 2.1 times near 0.  Against 64 bits, z of spread 1.1, root mean square:
//   gelu 3.5e-8, its slope 5.1e-8 (a library's erf: 3.8e-8 and 4.1e-8).  A second step of the reciprocal changes neither.
//   BRIEF, eight terms (c = 5/16): 2.3e-7, for bf16 tensors (half a step: 3.9e-3).  131072 x 64 -> 192 with gelu 26.9 us, with ten terms 27.5; layer
//   norm of 65536 x 256 with gelu 21.2 and 21.7, backward 31.2 and 32.1 (dgamma off by 1.9e-7 either way, from its sums).
template <bool BRIEF>
__device__ __forceinline__ void normal_cdf(float z, float& cdf, float& density) {
  const float e = __expf(-0.5f * z * z);
  const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(BRIEF ? 0.3125f : 0.375f, fabsf(z), 1.f));
  float s;
  if constexpr (BRIEF) {
    s = __builtin_fmaf(0.035328057f, t, -0.1358021f);
    s = __builtin_fmaf(s, t, 0.14035626f);
    s = __builtin_fmaf(s, t, -0.004521572f);
    s = __builtin_fmaf(s, t, 0.10540111f);
    s = __builtin_fmaf(s, t, 0.109672695f);
    s = __builtin_fmaf(s, t, 0.1249033f);
    s = __builtin_fmaf(s, t, 0.12466235f);
  } else {
    s = __builtin_fmaf(0.02089967f, t, -0.13400264f);
    s = __builtin_fmaf(s, t, 0.3448391f);
    s = __builtin_fmaf(s, t, -0.42401287f);
    s = __builtin_fmaf(s, t, 0.21556622f);
    s = __builtin_fmaf(s, t, -0.056159656f);
    s = __builtin_fmaf(s, t, 0.10811007f);
    s = __builtin_fmaf(s, t, 0.125283f);
    s = __builtin_fmaf(s, t, 0.14988403f);
    s = __builtin_fmaf(s, t, 0.14959307f);
  }
  const float tail = s * t * e;
  cdf = z < 0.f ? tail : 1.f - tail;
  density = 0.39894228040143268f * e;
}
__device__ __forceinline__ float sigmoid(float z) { return __builtin_amdgcn_rcpf(1.f + __expf(-z)); }

// z becomes its activation (one branch for all of them, not one for each); BRIEF: of bf16 tensors
template <bool BRIEF, int E>
__device__ __forceinline__ void act_values(float (&z)[E], int act) {
  if (act == kActRelu) {
#pragma unroll
    for (int e = 0; e < E; ++e) z[e] = z[e] < 0.f ? 0.f : z[e];  // (a NaN stays one)
  } else if (act == kActGelu) {
#pragma unroll
    for (int e = 0; e < E; ++e) {
      float cdf, density;
      normal_cdf<BRIEF>(z[e], cdf, density);
      z[e] *= cdf;
    }
  } else if (act == kActSilu) {
#pragma unroll
    for (int e = 0; e < E; ++e) z[e] *= sigmoid(z[e]);
  }
}
// g becomes g act'(z)
template <bool BRIEF, int E>
__device__ __forceinline__ void act_slopes(float (&g)[E], const float (&z)[E], int act) {
  if (act == kActRelu) {
#pragma unroll
    for (int e = 0; e < E; ++e) g[e] = z[e] > 0.f ? g[e] : 0.f;
  } else if (act == kActGelu) {
#pragma unroll
    for (int e = 0; e < E; ++e) {
      float cdf, density;
      normal_cdf<BRIEF>(z[e], cdf, density);
      g[e] *= __builtin_fmaf(z[e], density, cdf);
    }
  } else if (act == kActSilu) {
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const float s = sigmoid(z[e]);
      g[e] *= s * __builtin_fmaf(z[e], 1.f - s, 1.f);
    }
  }
}

// Dropout of probability p.  Element i stays where word i % 4 of the generator's block i / 4 is at least `least` = floor(p 2^32);
// kept values are multiplied by `factor` = 1 / (1 - p), dropped ones are replaced by 0, whatever they were.
struct Dropout {
  const int64_t* rng;  // device memory: seed, call number; null: nothing is dropped
  uint32_t least;
  float factor;
};
inline Dropout make_dropout(float p, const int64_t* rng) {
  Dropout d = {nullptr, 0u, 1.f};
  if (p > 0.f) {
    d.rng = rng;
    d.least = (uint32_t)((double)p * 4294967296.0);
    d.factor = (float)(1.0 / (1.0 - (double)p));
  }
  return d;
}

struct RngKey {
  uint32_t k0, k1, c2, c3;
};
__device__ __forceinline__ RngKey rng_key(const int64_t* rng) {
  const uint64_t seed = (uint64_t)rng[0], call = (uint64_t)rng[1];
  return {(uint32_t)seed, (uint32_t)(seed >> 32), (uint32_t)call, (uint32_t)(call >> 32)};
}
// Philox 4x32 with ten rounds (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011): key = the seed,
// counter = (block, call number).  A pure function of the element's place: forward and backward work it out again instead of
// storing a mask, and any kernel may take any part of a tensor.
__device__ __forceinline__ uint32_t xor3(uint32_t a, uint32_t b, uint32_t c) { return __builtin_amdgcn_bitop3_b32(a, b, c, 0x96); }
__device__ __forceinline__ uint4 rng_words(const RngKey& key, uint64_t block) {
  uint32_t c0 = (uint32_t)block, c1 = (uint32_t)(block >> 32), c2 = key.c2, c3 = key.c3, k0 = key.k0, k1 = key.k1;
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
    c0 = xor3((uint32_t)(b >> 32), c1, k0);
    c1 = (uint32_t)b;
    c2 = xor3((uint32_t)(a >> 32), c3, k1);
    c3 = (uint32_t)a;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return make_uint4(c0, c1, c2, c3);
}
__device__ __forceinline__ uint32_t rng_word(const RngKey& key, uint64_t element) {
  const uint4 w = rng_words(key, element >> 2);
  const int i = (int)(element & 3);
  return i == 0 ? w.x : i == 1 ? w.y : i == 2 ? w.z : w.w;
}
// v[0..E) are elements first .. first + E - 1; `even`: first is a multiple of 4, that is, of the generator's blocks.
template <int E>
__device__ __forceinline__ void drop(float (&v)[E], const Dropout& d, const RngKey& key, uint64_t first, bool even) {
  if constexpr (E == 1) {
    v[0] = rng_word(key, first) >= d.least ? v[0] * d.factor : 0.f;
  } else {
    static_assert(E % 4 == 0);
    const uint64_t block = first >> 2;
    uint4 w[E / 4 + 1];
#pragma unroll
    for (int q = 0; q < E / 4; ++q) w[q] = rng_words(key, block + q);
    const auto keep = [&](float& x, uint32_t word) __attribute__((always_inline)) { x = word >= d.least ? x * d.factor : 0.f; };
    if (even) {
#pragma unroll
      for (int q = 0; q < E / 4; ++q) {
        keep(v[4 * q], w[q].x);
        keep(v[4 * q + 1], w[q].y);
        keep(v[4 * q + 2], w[q].z);
        keep(v[4 * q + 3], w[q].w);
      }
    } else {  // one block more, and the words from where the piece begins
      w[E / 4] = rng_words(key, block + E / 4);
      const bool odd = first & 1, two = first & 2;
#pragma unroll
      for (int q = 0; q < E / 4; ++q) {
        const uint32_t a = two ? w[q].z : w[q].x, b = two ? w[q].w : w[q].y, c = two ? w[q + 1].x : w[q].z, e = two ? w[q + 1].y : w[q].w,
                       f = two ? w[q + 1].z : w[q + 1].x;
        keep(v[4 * q], odd ? b : a);
        keep(v[4 * q + 1], odd ? c : b);
        keep(v[4 * q + 2], odd ? e : c);
        keep(v[4 * q + 3], odd ? f : e);
      }
    }
  }
}

// A piece of E consecutive values in memory: 16 bytes (E = 4 for fp32, 8 for bf16), wherever a value may start, or one value.  (Loads and
// stores of 16 bytes need no alignment on this hardware; a piece that crosses a line takes two.)
template <typename T>
constexpr int kPiece = 16 / (int)sizeof(T);

__device__ __forceinline__ uint32_t pack2_bf16(float lo, float hi) {
  typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
  typedef __attribute__((ext_vector_type(2))) float f32x2;
  const f32x2 f = {lo, hi};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2));
}
template <int E>
__device__ __forceinline__ void load_piece(const float* p, float (&v)[E]) {
  __builtin_memcpy(v, p, sizeof(v));
}
template <int E>
__device__ __forceinline__ void load_piece(const bf16_t* p, float (&v)[E]) {
  if constexpr (E == 1) {
    v[0] = bf16_to_f32(*p);
  } else {
    uint32_t w[E / 2];
    __builtin_memcpy(w, p, sizeof(w));
#pragma unroll
    for (int e = 0; e < E / 2; ++e) {
      v[2 * e] = __uint_as_float(w[e] << 16);
      v[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
    }
  }
}
template <int E>
__device__ __forceinline__ void store_piece(float* p, const float (&v)[E]) {
  __builtin_memcpy(p, v, sizeof(v));
}
template <int E>
__device__ __forceinline__ void store_piece(bf16_t* p, const float (&v)[E]) {
  if constexpr (E == 1) {
    *p = f32_to_bf16(v[0]);
  } else {
    uint32_t w[E / 2];
#pragma unroll
    for (int e = 0; e < E / 2; ++e) w[e] = pack2_bf16(v[2 * e], v[2 * e + 1]);
    __builtin_memcpy(p, w, sizeof(w));
  }
}
// the first n of a piece's values (the others read as 0)
template <int E, typename T>
__device__ __forceinline__ void load_some(const T* p, int n, float (&v)[E]) {
  if (n >= E) {
    load_piece<E>(p, v);
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = e < n ? Elem<T>::load(p + e) : 0.f;
  }
}
template <int E, typename T>
__device__ __forceinline__ void store_some(T* p, int n, const float (&v)[E]) {
  if (n >= E) {
    store_piece<E>(p, v);
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (e < n) Elem<T>::store(p + e, v[e]);
  }
}

}  // namespace affmae
