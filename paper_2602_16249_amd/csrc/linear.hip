// Dense layer of the tokens: out = residual + dropout(act(x W^T + bias)), and its gradients.
#include "launch.h"
#include "timing.h"

#include "dense_common.h"

#include <algorithm>

namespace affmae {
namespace {

constexpr int kThreads = 256;
constexpr int kTile = 64, kDepth = 16;

struct Product {  // c[m][n] = sum_k a(m, k) b(n, k), element (m, k) of a at a + m a_m + k a_k, likewise b
  const void *a, *b;
  size_t a_m, a_k, b_n, b_k;
  long long M, N, K;
};
struct Epilogue {
  const void *bias, *residual;
  void *out, *pre;
  int act;
  Dropout d;
};

// 64 x 64 values of c by 256 threads, 4 x 4 each, 16 deep slices of both operands in LDS
template <typename T>
__global__ __launch_bounds__(kThreads) void linear_kernel(Product p, Epilogue e) {
  __shared__ float as[kDepth][kTile + 1], bs[kDepth][kTile + 1];
  const long long tiles_n = (p.N + kTile - 1) / kTile;
  const long long m0 = (long long)blockIdx.x / tiles_n * kTile, n0 = (long long)blockIdx.x % tiles_n * kTile;
  const T *a = (const T*)p.a, *b = (const T*)p.b;
  const int tm = threadIdx.x / 16 * 4, tn = threadIdx.x % 16 * 4;
  float c[4][4] = {};
  for (long long k0 = 0; k0 < p.K; k0 += kDepth) {
    for (int i = threadIdx.x; i < kTile * kDepth; i += kThreads) {
      const int r = i / kDepth, k = i % kDepth;
      as[k][r] = m0 + r < p.M && k0 + k < p.K ? Elem<T>::load(a + (m0 + r) * p.a_m + (k0 + k) * p.a_k) : 0.f;
      bs[k][r] = n0 + r < p.N && k0 + k < p.K ? Elem<T>::load(b + (n0 + r) * p.b_n + (k0 + k) * p.b_k) : 0.f;
    }
    __syncthreads();
    for (int k = 0; k < kDepth; ++k)
      for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j) c[i][j] += as[k][tm + i] * bs[k][tn + j];
    __syncthreads();
  }
  RngKey key = {};
  if (e.d.rng) key = rng_key(e.d.rng);
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < 4; ++j) {
      const long long m = m0 + tm + i, n = n0 + tn + j;
      if (m >= p.M || n >= p.N) continue;
      const size_t at = (size_t)m * p.N + n;
      float v[1] = {c[i][j]};
      if (e.bias) v[0] += Elem<T>::load((const T*)e.bias + n);
      if (e.pre) Elem<T>::store((T*)e.pre + at, v[0]);
      v[0] = act_value(v[0], e.act);
      if (e.d.rng) drop<1>(v, e.d, key, at);
      if (e.residual) v[0] += Elem<T>::load((const T*)e.residual + at);
      Elem<T>::store((T*)e.out + at, v[0]);
    }
}

// dz = dropout(dout) act'(pre)
template <typename T>
__global__ __launch_bounds__(kThreads) void linear_dz_kernel(const T* __restrict__ dout, const T* __restrict__ pre, long long n, int act, Dropout d, T* __restrict__ dz) {
  RngKey key = {};
  if (d.rng) key = rng_key(d.rng);
  for (long long i = (long long)blockIdx.x * kThreads + threadIdx.x; i < n; i += (long long)gridDim.x * kThreads) {
    float v[1] = {Elem<T>::load(dout + i)};
    if (d.rng) drop<1>(v, d, key, (uint64_t)i);
    if (pre) v[0] *= act_slope(Elem<T>::load(pre + i), act);
    Elem<T>::store(dz + i, v[0]);
  }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void linear_dbias_kernel(const T* __restrict__ dz, long long rows, int C, T* __restrict__ dbias) {
  __shared__ float acc[4];
  float s = 0.f;
  for (long long i = threadIdx.x; i < rows; i += kThreads) s += Elem<T>::load(dz + (size_t)i * C + blockIdx.x);
  s = wave_sum(s);
  if ((threadIdx.x & (kWave - 1)) == 0) acc[threadIdx.x / kWave] = s;
  __syncthreads();
  if (threadIdx.x == 0) Elem<T>::store(dbias + blockIdx.x, (acc[0] + acc[1]) + (acc[2] + acc[3]));
}

template <typename T>
hipError_t product(const Product& p, const Epilogue& e, hipStream_t stream) {
  const long long tiles = (p.M + kTile - 1) / kTile * ((p.N + kTile - 1) / kTile);
  AFFMAE_LAUNCH("linear_kernel", stream, linear_kernel<T>, dim3((unsigned)tiles), dim3(kThreads), 0, stream, p, e);
  return hipGetLastError();
}

template <typename T>
hipError_t fwd(const LinearArgs& a, hipStream_t stream) {
  const Product p = {a.x, a.weight, (size_t)a.Cin, 1, (size_t)a.Cin, 1, a.rows, a.Cout, a.Cin};
  const Epilogue e = {a.bias, a.residual, a.out, a.pre_out, a.act, make_dropout(a.p, a.rng)};
  return product<T>(p, e, stream);
}

template <typename T>
hipError_t bwd(const LinearArgs& a, hipStream_t stream) {
  const void* dz = a.dout;
  const Dropout d = make_dropout(a.p, a.rng);
  if (a.act != kActNone || d.rng) {
    const long long n = (long long)a.rows * a.Cout;
    AFFMAE_LAUNCH("linear_dz_kernel", stream, linear_dz_kernel<T>, dim3((unsigned)std::min((n + kThreads - 1) / kThreads, 1ll << 23)), dim3(kThreads), 0, stream,
                  (const T*)a.dout, a.act != kActNone ? (const T*)a.pre : nullptr, n, a.act, d, (T*)a.workspace);
    dz = a.workspace;
  }
  const Epilogue none = {nullptr, nullptr, nullptr, nullptr, kActNone, make_dropout(0.f, nullptr)};
  hipError_t rc = hipSuccess;
  if (a.dx) {
    Epilogue e = none;
    e.out = a.dx;
    rc = product<T>({dz, a.weight, (size_t)a.Cout, 1, 1, (size_t)a.Cin, a.rows, a.Cin, a.Cout}, e, stream);
  }
  if (rc == hipSuccess && a.dweight) {
    Epilogue e = none;
    e.out = a.dweight;
    rc = product<T>({dz, a.x, 1, (size_t)a.Cout, 1, (size_t)a.Cin, a.Cout, a.Cin, a.rows}, e, stream);
  }
  if (rc == hipSuccess && a.dbias) {
    AFFMAE_LAUNCH("linear_dbias_kernel", stream, linear_dbias_kernel<T>, dim3(a.Cout), dim3(kThreads), 0, stream, (const T*)dz, (long long)a.rows, a.Cout, (T*)a.dbias);
    rc = hipGetLastError();
  }
  return rc;
}

}  // namespace

size_t linear_bwd_workspace_bytes(int rows, int, int Cout, int act, bool drops, int dtype, bool, bool) {
  return act != kActNone || drops ? (size_t)rows * Cout * (dtype == 1 ? 2 : 4) : 0;
}
hipError_t launch_linear_fwd(const LinearArgs& a, hipStream_t stream) { return a.dtype == 1 ? fwd<bf16_t>(a, stream) : fwd<float>(a, stream); }
hipError_t launch_linear_bwd(const LinearArgs& a, hipStream_t stream) { return a.dtype == 1 ? bwd<bf16_t>(a, stream) : bwd<float>(a, stream); }

}  // namespace affmae
