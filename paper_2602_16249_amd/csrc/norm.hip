// Group norm with an activation over token tensors [B,N,C], channels last: an image's group g of Cg = C / G channels has
// mean and variance over its N x Cg values, z = gamma (x - mean) rstd + beta, out = act(z).  B tokens of N = 1 and one group are
// the layer norm of every token.
#include "launch.h"
#include "timing.h"

#include "dense_common.h"

namespace affmae {
namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ float block_sum(float v, float* acc) {
  v = wave_sum(v);
  __syncthreads();
  if ((threadIdx.x & (kWave - 1)) == 0) acc[threadIdx.x / kWave] = v;
  __syncthreads();
  return (acc[0] + acc[1]) + (acc[2] + acc[3]);
}

// workgroup per (image, group): mean, then the variance about it, then the values
template <typename T>
__global__ __launch_bounds__(kThreads) void norm_fwd_kernel(const T* __restrict__ x, const T* __restrict__ gamma, const T* __restrict__ beta, int N, int C,
                                                            int G, float eps, int act, T* __restrict__ out, float* __restrict__ mean, float* __restrict__ rstd) {
  __shared__ float acc[4];
  const int b = blockIdx.x / G, g = blockIdx.x % G, Cg = C / G;
  const size_t base = (size_t)b * N * C + (size_t)g * Cg;
  const long long n = (long long)N * Cg;
  float s = 0.f;
  for (long long i = threadIdx.x; i < n; i += kThreads) s += Elem<T>::load(x + base + (size_t)(i / Cg) * C + i % Cg);
  const float m = block_sum(s, acc) / (float)n;
  s = 0.f;
  for (long long i = threadIdx.x; i < n; i += kThreads) {
    const float d = Elem<T>::load(x + base + (size_t)(i / Cg) * C + i % Cg) - m;
    s += d * d;
  }
  const float r = 1.f / sqrtf(block_sum(s, acc) / (float)n + eps);
  if (threadIdx.x == 0) {
    mean[blockIdx.x] = m;
    rstd[blockIdx.x] = r;
  }
  for (long long i = threadIdx.x; i < n; i += kThreads) {
    const int c = (int)(i % Cg);
    const size_t at = base + (size_t)(i / Cg) * C + c;
    float z = (Elem<T>::load(x + at) - m) * r;
    if (gamma) z = z * Elem<T>::load(gamma + g * Cg + c) + Elem<T>::load(beta + g * Cg + c);
    Elem<T>::store(out + at, act_value(z, act));
  }
}

template <typename T>
__device__ __forceinline__ void norm_terms(const T* x, const T* dout, const T* gamma, const T* beta, size_t at, int c, float m, float r, int act,
                                           float& xhat, float& dz, float& gm) {
  xhat = (Elem<T>::load(x + at) - m) * r;
  gm = gamma ? Elem<T>::load(gamma + c) : 1.f;
  const float z = gamma ? xhat * gm + Elem<T>::load(beta + c) : xhat;
  dz = Elem<T>::load(dout + at) * act_slope(z, act);
}

template <typename T>
__global__ __launch_bounds__(kThreads) void norm_bwd_kernel(const T* __restrict__ x, const T* __restrict__ gamma, const T* __restrict__ beta,
                                                            const float* __restrict__ mean, const float* __restrict__ rstd, const T* __restrict__ dout, int N,
                                                            int C, int G, int act, T* __restrict__ dx) {
  __shared__ float acc[4];
  const int b = blockIdx.x / G, g = blockIdx.x % G, Cg = C / G;
  const size_t base = (size_t)b * N * C + (size_t)g * Cg;
  const long long n = (long long)N * Cg;
  const float m = mean[blockIdx.x], r = rstd[blockIdx.x];
  float s1 = 0.f, s2 = 0.f, xhat, dz, gm;
  for (long long i = threadIdx.x; i < n; i += kThreads) {
    norm_terms(x, dout, gamma, beta, base + (size_t)(i / Cg) * C + i % Cg, g * Cg + (int)(i % Cg), m, r, act, xhat, dz, gm);
    s1 += dz * gm;
    s2 += dz * gm * xhat;
  }
  s1 = block_sum(s1, acc) / (float)n;
  s2 = block_sum(s2, acc) / (float)n;
  for (long long i = threadIdx.x; i < n; i += kThreads) {
    const size_t at = base + (size_t)(i / Cg) * C + i % Cg;
    norm_terms(x, dout, gamma, beta, at, g * Cg + (int)(i % Cg), m, r, act, xhat, dz, gm);
    Elem<T>::store(dx + at, r * (dz * gm - s1 - xhat * s2));
  }
}

// workgroup per channel
template <typename T>
__global__ __launch_bounds__(kThreads) void norm_affine_kernel(const T* __restrict__ x, const T* __restrict__ gamma, const T* __restrict__ beta,
                                                               const float* __restrict__ mean, const float* __restrict__ rstd, const T* __restrict__ dout,
                                                               int B, int N, int C, int G, int act, float* __restrict__ dgamma, float* __restrict__ dbeta) {
  __shared__ float acc[4];
  const int c = blockIdx.x, g = c / (C / G);
  float sg = 0.f, sb = 0.f, xhat, dz, gm;
  for (long long i = threadIdx.x; i < (long long)B * N; i += kThreads) {
    const size_t bg = (size_t)(i / N) * G + g;
    norm_terms(x, dout, gamma, beta, (size_t)i * C + c, c, mean[bg], rstd[bg], act, xhat, dz, gm);
    sg += dz * xhat;
    sb += dz;
  }
  sg = block_sum(sg, acc);
  sb = block_sum(sb, acc);
  if (threadIdx.x == 0) {
    dgamma[c] = sg;
    dbeta[c] = sb;
  }
}

template <typename T>
hipError_t fwd(const NormArgs& a, hipStream_t stream) {
  AFFMAE_LAUNCH("norm_fwd_kernel", stream, norm_fwd_kernel<T>, dim3(a.B * a.G), dim3(kThreads), 0, stream, (const T*)a.x, (const T*)a.gamma, (const T*)a.beta, a.N,
                a.C, a.G, a.eps, a.act, (T*)a.out, a.mean, a.rstd);
  return hipGetLastError();
}
template <typename T>
hipError_t bwd(const NormArgs& a, hipStream_t stream) {
  AFFMAE_LAUNCH("norm_bwd_kernel", stream, norm_bwd_kernel<T>, dim3(a.B * a.G), dim3(kThreads), 0, stream, (const T*)a.x, (const T*)a.gamma, (const T*)a.beta,
                a.mean, a.rstd, (const T*)a.dout, a.N, a.C, a.G, a.act, (T*)a.dx);
  if (a.dgamma)
    AFFMAE_LAUNCH("norm_affine_kernel", stream, norm_affine_kernel<T>, dim3(a.C), dim3(kThreads), 0, stream, (const T*)a.x, (const T*)a.gamma,
                  (const T*)a.beta, a.mean, a.rstd, (const T*)a.dout, a.B, a.N, a.C, a.G, a.act, a.dgamma, a.dbeta);
  return hipGetLastError();
}

}  // namespace

size_t norm_fwd_workspace_bytes(int, int, int, int, int) { return 0; }
size_t norm_bwd_workspace_bytes(int, int, int, int, int) { return 0; }
hipError_t launch_norm_fwd(const NormArgs& a, hipStream_t stream) { return a.dtype == 1 ? fwd<bf16_t>(a, stream) : fwd<float>(a, stream); }
hipError_t launch_norm_bwd(const NormArgs& a, hipStream_t stream) { return a.dtype == 1 ? bwd<bf16_t>(a, stream) : bwd<float>(a, stream); }

}  // namespace affmae
