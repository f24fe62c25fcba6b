// C ABI of the dense operators: host-side argument validation and kernel dispatch.
// Declarations and the meaning of every argument are in include/affmae.h.
#include "../../include/affmae.h"

#include "launch.h"

namespace {

constexpr size_t kAlign = 256;
size_t align_up(size_t n) { return (n + kAlign - 1) / kAlign * kAlign; }

bool misaligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) != 0; }
size_t element(int dtype) { return dtype == AFFMAE_BF16 ? 2 : 4; }

int check_type(int dtype) { return dtype == AFFMAE_F32 || dtype == AFFMAE_BF16 ? AFFMAE_OK : AFFMAE_ERR_DTYPE; }
bool bad_act(int act) { return act < AFFMAE_ACT_NONE || act > AFFMAE_ACT_SILU; }

// Probability of dropout, and the generator's state that it needs.
int check_dropout(float p, const int64_t* rng) {
  if (!(p >= 0.f) || !(p < 1.f)) return AFFMAE_ERR_SHAPE;
  if (p > 0.f && !rng) return AFFMAE_ERR_NULL;
  if (misaligned(rng, 8)) return AFFMAE_ERR_SHAPE;
  return AFFMAE_OK;
}

int check_linear_shape(int rows, int Cin, int Cout, int act, int dtype) {
  const int rc = check_type(dtype);
  if (rc != AFFMAE_OK) return rc;
  if (rows < 1 || Cin < 1 || Cout < 1 || bad_act(act)) return AFFMAE_ERR_SHAPE;
  // a tile's rows are addressed from its first one with 32-bit offsets; the runtime counts the threads of a launch in 32 bits
  if (rows > (1 << 29) || Cin > (1 << 20) || Cout > (1 << 20)) return AFFMAE_ERR_UNSUPPORTED;
  if ((long long)rows * Cin > (1ll << 35) || (long long)rows * Cout > (1ll << 35) || (long long)Cin * Cout > (1ll << 35)) return AFFMAE_ERR_UNSUPPORTED;
  return AFFMAE_OK;
}

int check_norm_shape(int B, int N, int C, int groups, int dtype) {
  const int rc = check_type(dtype);
  if (rc != AFFMAE_OK) return rc;
  if (B < 1 || N < 1 || C < 1 || groups < 1 || C % groups) return AFFMAE_ERR_SHAPE;
  // tokens are counted in 31 bits, and those beyond the last that a workgroup's threads look at: up to 64 times 256 where they hold its run
  // in registers, up to 255 where they walk it
  if ((long long)B * N > (1ll << 31) - (1 << 16) || (long long)B * groups > (1ll << 24)) return AFFMAE_ERR_UNSUPPORTED;
  if (C > (1 << 20) || (long long)B * N * C > (1ll << 38)) return AFFMAE_ERR_UNSUPPORTED;
  return AFFMAE_OK;
}

int status(hipError_t e) { return e == hipSuccess ? AFFMAE_OK : AFFMAE_ERR_DEVICE; }

}  // namespace

extern "C" {

int affmae_linear_fwd(const void* x, const void* weight, const void* bias, const void* residual, int rows, int Cin, int Cout,
                      int act, float p, const int64_t* rng, int dtype, void* out, void* pre, void* stream) {
  if (!x || !weight || !out) return AFFMAE_ERR_NULL;
  int rc = check_linear_shape(rows, Cin, Cout, act, dtype);
  if (rc != AFFMAE_OK) return rc;
  rc = check_dropout(p, rng);
  if (rc != AFFMAE_OK) return rc;
  const size_t el = element(dtype);
  if (misaligned(x, el) || misaligned(weight, el) || misaligned(bias, el) || misaligned(residual, el) || misaligned(out, el) || misaligned(pre, el))
    return AFFMAE_ERR_SHAPE;
  affmae::LinearArgs a = {};
  a.x = x; a.weight = weight; a.bias = bias; a.residual = residual;
  a.rows = rows; a.Cin = Cin; a.Cout = Cout; a.act = act; a.dtype = dtype; a.p = p; a.rng = rng;
  a.out = out; a.pre_out = pre;
  return status(affmae::launch_linear_fwd(a, static_cast<hipStream_t>(stream)));
}

size_t affmae_linear_bwd_workspace_bytes(int rows, int Cin, int Cout, int act, float p, int dtype, int want_dx, int want_dweight) {
  if (check_linear_shape(rows, Cin, Cout, act, dtype) != AFFMAE_OK || !(p >= 0.f) || !(p < 1.f)) return 0;
  return align_up(affmae::linear_bwd_workspace_bytes(rows, Cin, Cout, act, p > 0.f, dtype, want_dx != 0, want_dweight != 0));
}

int affmae_linear_bwd(const void* x, const void* weight, const void* pre, const void* dout, int rows, int Cin, int Cout, int act,
                      float p, const int64_t* rng, int dtype, void* dx, void* dweight, void* dbias, void* workspace,
                      size_t workspace_bytes, void* stream) {
  if (!dout || (!dx && !dweight) || (dx && !weight) || (dweight && !x) || (dbias && !dweight)) return AFFMAE_ERR_NULL;
  if (act != AFFMAE_ACT_NONE && !pre) return AFFMAE_ERR_NULL;
  int rc = check_linear_shape(rows, Cin, Cout, act, dtype);
  if (rc != AFFMAE_OK) return rc;
  rc = check_dropout(p, rng);
  if (rc != AFFMAE_OK) return rc;
  const size_t el = element(dtype);
  if (misaligned(x, el) || misaligned(weight, el) || misaligned(pre, el) || misaligned(dout, el) || misaligned(dx, el) || misaligned(dweight, el) ||
      misaligned(dbias, el))
    return AFFMAE_ERR_SHAPE;
  const size_t need = affmae_linear_bwd_workspace_bytes(rows, Cin, Cout, act, p, dtype, dx != nullptr, dweight != nullptr);
  if (need && (!workspace || workspace_bytes < need || misaligned(workspace, kAlign))) return AFFMAE_ERR_WORKSPACE;
  affmae::LinearArgs a = {};
  a.x = x; a.weight = weight; a.pre = pre; a.dout = dout;
  a.rows = rows; a.Cin = Cin; a.Cout = Cout; a.act = act; a.dtype = dtype; a.p = p; a.rng = rng;
  a.dx = dx; a.dweight = dweight; a.dbias = dbias; a.workspace = workspace;
  return status(affmae::launch_linear_bwd(a, static_cast<hipStream_t>(stream)));
}

size_t affmae_norm_fwd_workspace_bytes(int B, int N, int C, int groups, int dtype) {
  if (check_norm_shape(B, N, C, groups, dtype) != AFFMAE_OK) return 0;
  return align_up(affmae::norm_fwd_workspace_bytes(B, N, C, groups, dtype));
}

int affmae_norm_fwd(const void* x, const void* gamma, const void* beta, int B, int N, int C, int groups, float eps, int act,
                    int dtype, void* out, float* mean, float* rstd, void* workspace, size_t workspace_bytes, void* stream) {
  if (!x || !out || !mean || !rstd || (gamma == nullptr) != (beta == nullptr)) return AFFMAE_ERR_NULL;
  const int rc = check_norm_shape(B, N, C, groups, dtype);
  if (rc != AFFMAE_OK) return rc;
  if (bad_act(act) || !(eps > 0.f) || !(eps < 3e38f)) return AFFMAE_ERR_SHAPE;
  const size_t el = element(dtype);
  if (misaligned(x, el) || misaligned(gamma, el) || misaligned(beta, el) || misaligned(out, el) || misaligned(mean, 4) || misaligned(rstd, 4))
    return AFFMAE_ERR_SHAPE;
  const size_t need = affmae_norm_fwd_workspace_bytes(B, N, C, groups, dtype);
  if (need && (!workspace || workspace_bytes < need || misaligned(workspace, kAlign))) return AFFMAE_ERR_WORKSPACE;
  affmae::NormArgs a = {};
  a.x = x; a.gamma = gamma; a.beta = beta;
  a.B = B; a.N = N; a.C = C; a.G = groups; a.act = act; a.dtype = dtype; a.eps = eps;
  a.mean = mean; a.rstd = rstd; a.out = out; a.workspace = workspace;
  return status(affmae::launch_norm_fwd(a, static_cast<hipStream_t>(stream)));
}

size_t affmae_norm_bwd_workspace_bytes(int B, int N, int C, int groups, int dtype) {
  if (check_norm_shape(B, N, C, groups, dtype) != AFFMAE_OK) return 0;
  return align_up(affmae::norm_bwd_workspace_bytes(B, N, C, groups, dtype));
}

int affmae_norm_bwd(const void* x, const void* gamma, const void* beta, const float* mean, const float* rstd, const void* dout,
                    int B, int N, int C, int groups, int act, int dtype, void* dx, float* dgamma, float* dbeta, void* workspace,
                    size_t workspace_bytes, void* stream) {
  if (!x || !mean || !rstd || !dout || !dx || (gamma == nullptr) != (beta == nullptr)) return AFFMAE_ERR_NULL;
  if ((dgamma == nullptr) != (dbeta == nullptr) || (dgamma && !gamma)) return AFFMAE_ERR_NULL;
  const int rc = check_norm_shape(B, N, C, groups, dtype);
  if (rc != AFFMAE_OK) return rc;
  if (bad_act(act)) return AFFMAE_ERR_SHAPE;
  const size_t el = element(dtype);
  if (misaligned(x, el) || misaligned(gamma, el) || misaligned(beta, el) || misaligned(mean, 4) || misaligned(rstd, 4) || misaligned(dout, el) ||
      misaligned(dx, el) || misaligned(dgamma, 4) || misaligned(dbeta, 4))
    return AFFMAE_ERR_SHAPE;
  const size_t need = affmae_norm_bwd_workspace_bytes(B, N, C, groups, dtype);
  if (need && (!workspace || workspace_bytes < need || misaligned(workspace, kAlign))) return AFFMAE_ERR_WORKSPACE;
  affmae::NormArgs a = {};
  a.x = x; a.gamma = gamma; a.beta = beta; a.mean = const_cast<float*>(mean); a.rstd = const_cast<float*>(rstd); a.dout = dout;
  a.B = B; a.N = N; a.C = C; a.G = groups; a.act = act; a.dtype = dtype;
  a.dx = dx; a.dgamma = dgamma; a.dbeta = dbeta; a.workspace = workspace;
  return status(affmae::launch_norm_bwd(a, static_cast<hipStream_t>(stream)));
}

int affmae_dropout_fwd(const void* x, const void* residual, int64_t n, float p, const int64_t* rng, int dtype, void* out,
                       void* stream) {
  if (!x || !out) return AFFMAE_ERR_NULL;
  int rc = check_type(dtype);
  if (rc != AFFMAE_OK) return rc;
  if (n < 1) return AFFMAE_ERR_SHAPE;
  rc = check_dropout(p, rng);
  if (rc != AFFMAE_OK) return rc;
  const size_t el = element(dtype);
  if (misaligned(x, el) || misaligned(residual, el) || misaligned(out, el)) return AFFMAE_ERR_SHAPE;
  affmae::DropoutArgs a = {};
  a.x = x; a.residual = residual; a.n = n; a.p = p; a.rng = rng; a.dtype = dtype; a.out = out;
  return status(affmae::launch_dropout(a, static_cast<hipStream_t>(stream)));
}

int affmae_dropout_bwd(const void* dout, int64_t n, float p, const int64_t* rng, int dtype, void* dx, void* stream) {
  return affmae_dropout_fwd(dout, nullptr, n, p, rng, dtype, dx, stream);
}

}  // extern "C"
