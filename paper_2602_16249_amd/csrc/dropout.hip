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

template <typename T, int E>
__global__ __launch_bounds__(kThreads) void dropout_kernel(const T* x, const T* residual, long long n, Dropout d, T* out) {
  RngKey key = {};
  if (d.rng) key = rng_key(d.rng);
  for (long long i = ((long long)blockIdx.x * kThreads + threadIdx.x) * E; i < n; i += (long long)gridDim.x * kThreads * E) {
    float v[E];
    load_piece<E>(x + i, v);
    if (d.rng) drop<E>(v, d, key, (uint64_t)i);
    if (residual) {
      float r[E];
      load_piece<E>(residual + i, r);
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] += r[e];
    }
    store_piece<E>(out + i, v);
  }
}

template <typename T>
hipError_t launch(const void* x, const void* residual, long long n, const Dropout& d, void* out, hipStream_t stream) {
  constexpr int E = kPiece<T>;
  const bool whole = n % E == 0 && aligned16(x) && aligned16(residual) && aligned16(out);
  const long long per = (long long)kThreads * (whole ? E : 1);
  const dim3 grid((unsigned)std::min((n + per - 1) / per, kMaxBlocks));
  if (whole)
    AFFMAE_LAUNCH("dropout_kernel", stream, (dropout_kernel<T, E>), grid, dim3(kThreads), 0, stream, (const T*)x, (const T*)residual, n, d, (T*)out);
  else
    AFFMAE_LAUNCH("dropout_kernel", stream, (dropout_kernel<T, 1>), grid, dim3(kThreads), 0, stream, (const T*)x, (const T*)residual, n, d, (T*)out);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_dropout(const DropoutArgs& a, hipStream_t stream) {
  const Dropout d = make_dropout(a.p, a.rng);
  return a.dtype == 1 ? launch<bf16_t>(a.x, a.residual, a.n, d, a.out, stream) : launch<float>(a.x, a.residual, a.n, d, a.out, stream);
}

}  // namespace affmae
