// Dropout from a counter-based generator (dense_common.h): out = residual + dropout(x), and its gradient, which is the same
// product with the same mask.  Nothing is stored between the two: the mask is a function of (seed, call number, place).
#include "launch.h"
#include "timing.h"

#include "dense_common.h"

#include <algorithm>

namespace affmae {
namespace {

constexpr int kThreads = 256;
constexpr long long kMaxBlocks = 1ll << 23;  // (the runtime counts the threads of a launch in 32 bits; further elements in further turns)

// A thread takes a piece of 16 bytes, the generator's words for it in one or two blocks, wherever the tensors start.
template <typename T>
__global__ __launch_bounds__(kThreads) void dropout_kernel(const T* x, const T* residual, long long n, Dropout d, T* out) {
  constexpr int E = kPiece<T>;
  RngKey key = {};
  if (d.rng) key = rng_key(d.rng);
  for (long long i = ((long long)blockIdx.x * kThreads + threadIdx.x) * E; i < n; i += (long long)gridDim.x * kThreads * E) {
    const auto piece = [&](int some) __attribute__((always_inline)) {
      float v[E], r[E];
      load_some<E>(x + i, some, v);
      if (residual) load_some<E>(residual + i, some, r);
      if (d.rng) drop<E>(v, d, key, (uint64_t)i, true);
      if (residual) {
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] += r[e];
      }
      store_some<E>(out + i, some, v);
    };
    if (n - i >= E)
      piece(E);
    else
      piece((int)(n - i));
  }
}

template <typename T>
hipError_t launch(const void* x, const void* residual, long long n, const Dropout& d, void* out, hipStream_t stream) {
  const long long per = (long long)kThreads * kPiece<T>;
  const dim3 grid((unsigned)std::min((n + per - 1) / per, kMaxBlocks));
  AFFMAE_LAUNCH("dropout_kernel", stream, dropout_kernel<T>, grid, dim3(kThreads), 0, stream, (const T*)x, (const T*)residual, n, d, (T*)out);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_dropout(const DropoutArgs& a, hipStream_t stream) {
  const Dropout d = make_dropout(a.p, a.rng);
  return a.dtype == 1 ? launch<bf16_t>(a.x, a.residual, a.n, d, a.out, stream) : launch<float>(a.x, a.residual, a.n, d, a.out, stream);
}

}  // namespace affmae
