// C ABI of attention between all tokens and of rotary positions: host-side argument validation and kernel dispatch.
// Declarations and the meaning of every argument are in include/affmae.h.
#include "../../include/affmae.h"

#include "launch.h"

namespace {

constexpr size_t kAlign = 256;
size_t align_up(size_t n) { return (n + kAlign - 1) / kAlign * kAlign; }
bool misaligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) != 0; }
int status(hipError_t e) { return e == hipSuccess ? AFFMAE_OK : AFFMAE_ERR_DEVICE; }
bool finite(float x) { return x - x == 0.f; }

int check_rotary(int B, int N, int H, int Hk, int d, int axes, int layout, int dtype) {
  if (dtype != AFFMAE_F32 && dtype != AFFMAE_BF16) return AFFMAE_ERR_DTYPE;
  if (B < 1 || N < 1 || H < 1 || Hk < 0 || d < 2 || d % 2 || axes < 1) return AFFMAE_ERR_SHAPE;
  if (layout != AFFMAE_ROTARY_PAIRS && layout != AFFMAE_ROTARY_HALVES) return AFFMAE_ERR_SHAPE;
  // a token's values are numbered in 31 bits
  if (d > 512 || axes > 3 || H > 4096 || Hk > 4096) return AFFMAE_ERR_UNSUPPORTED;
  if ((long long)B * N > (1ll << 31) - (1 << 16) || (long long)B * N * (H + Hk) > (1ll << 38) / d) return AFFMAE_ERR_UNSUPPORTED;
  return AFFMAE_OK;
}

int check_attn(int B, int Nq, int Nk, int H, int Hk, int d, int dtype) {
  if (dtype != AFFMAE_F32 && dtype != AFFMAE_BF16) return AFFMAE_ERR_DTYPE;
  if (B < 1 || Nq < 1 || Nk < 1 || H < 1 || Hk < 1 || H % Hk || d < 1) return AFFMAE_ERR_SHAPE;
  if (d % 8 || d > 128 || H > 4096 || Nq > (1 << 24) || Nk > (1 << 24)) return AFFMAE_ERR_UNSUPPORTED;
  // (query, head) pairs of a key head are numbered in 31 bits; a launch has at most 2^24 workgroups of 128 of them, or of 128 keys
  const long long rows = (long long)Nq * (H / Hk), most = (1ll << 24) - 8;
  if (rows > (1ll << 28) || (rows + 127) / 128 * B * Hk > most || ((long long)Nk + 127) / 128 * B * Hk > most) return AFFMAE_ERR_UNSUPPORTED;
  return AFFMAE_OK;
}

// The terms of the scores.
int check_terms(float scale, float cap, const float* q_xy, const float* k_xy, const float* slope, const int32_t* q_doc, const int32_t* k_doc) {
  if ((q_xy == nullptr) != (slope == nullptr) || (k_xy == nullptr) != (slope == nullptr) || (q_doc == nullptr) != (k_doc == nullptr)) return AFFMAE_ERR_NULL;
  if (!finite(scale) || !finite(cap) || cap < 0.f || (cap > 0.f && (cap < 1e-30f || !finite(scale / cap)))) return AFFMAE_ERR_SHAPE;
  // (scores are in units of log 2: scale log2 e without a cap, and 2 cap log2 e, are numbers of the kernels)
  if (cap > 0.f ? !finite(cap * 2.88539008f) : !finite(scale * 1.44269504f)) return AFFMAE_ERR_SHAPE;
  if (misaligned(q_xy, 8) || misaligned(k_xy, 8) || misaligned(slope, 4) || misaligned(q_doc, 4) || misaligned(k_doc, 4)) return AFFMAE_ERR_SHAPE;
  return AFFMAE_OK;
}

}  // namespace

extern "C" {

int affmae_rotary_fwd(const void* q, const void* k, const float* coords, const float* freq, int B, int N, int H, int Hk, int d,
                      int axes, int layout, int dtype, void* q_out, void* k_out, void* stream) {
  const int rc = check_rotary(B, N, H, Hk, d, axes, layout, dtype);
  if (!q || !coords || !freq || !q_out || (Hk > 0 && (!k || !k_out)) || (Hk == 0 && (k || k_out))) return AFFMAE_ERR_NULL;
  if (rc != AFFMAE_OK) return rc;
  const size_t el = dtype == AFFMAE_BF16 ? 2 : 4;
  if (misaligned(q, el) || misaligned(k, el) || misaligned(q_out, el) || misaligned(k_out, el) || misaligned(coords, 4) || misaligned(freq, 4)) return AFFMAE_ERR_SHAPE;
  affmae::RotaryArgs a = {};
  a.q = q; a.k = k; a.coords = coords; a.freq = freq;
  a.B = B; a.N = N; a.H = H; a.Hk = Hk; a.d = d; a.axes = axes; a.dtype = dtype; a.halves = layout == AFFMAE_ROTARY_HALVES;
  a.to_q = q_out; a.to_k = k_out;
  return status(affmae::launch_rotary(a, static_cast<hipStream_t>(stream)));
}

int affmae_rotary_bwd(const void* dq_out, const void* dk_out, const void* q_out, const void* k_out, const float* coords,
                      const float* freq, int B, int N, int H, int Hk, int d, int axes, int layout, int dtype, void* dq, void* dk,
                      float* dcoords, void* stream) {
  const int rc = check_rotary(B, N, H, Hk, d, axes, layout, dtype);
  if (!dq_out || !coords || !freq || !dq || (Hk > 0 && (!dk_out || !dk)) || (Hk == 0 && (dk_out || dk))) return AFFMAE_ERR_NULL;
  if (dcoords && (!q_out || (Hk > 0 && !k_out))) return AFFMAE_ERR_NULL;
  if (rc != AFFMAE_OK) return rc;
  const size_t el = dtype == AFFMAE_BF16 ? 2 : 4;
  if (misaligned(dq_out, el) || misaligned(dk_out, el) || misaligned(q_out, el) || misaligned(k_out, el) || misaligned(dq, el) || misaligned(dk, el) ||
      misaligned(coords, 4) || misaligned(freq, 4) || misaligned(dcoords, 4))
    return AFFMAE_ERR_SHAPE;
  affmae::RotaryArgs a = {};
  a.q = dq_out; a.k = dk_out; a.q_out = q_out; a.k_out = k_out; a.coords = coords; a.freq = freq;
  a.B = B; a.N = N; a.H = H; a.Hk = Hk; a.d = d; a.axes = axes; a.dtype = dtype; a.halves = layout == AFFMAE_ROTARY_HALVES; a.backward = true;
  a.to_q = dq; a.to_k = dk; a.dcoords = dcoords;
  return status(affmae::launch_rotary(a, static_cast<hipStream_t>(stream)));
}

size_t affmae_attn_fwd_workspace_bytes(int B, int Nq, int Nk, int H, int Hk, int d, int dtype, int docs) {
  if (check_attn(B, Nq, Nk, H, Hk, d, dtype) != AFFMAE_OK) return 0;
  return align_up(affmae::attn_fwd_workspace_bytes(B, Nq, Nk, H, Hk, d, dtype, docs != 0));
}

int affmae_attn_fwd(const void* q, const void* k, const void* v, const float* q_xy, const float* k_xy, const float* slope,
                    const int32_t* q_doc, const int32_t* k_doc, int B, int Nq, int Nk, int H, int Hk, int d, float scale, float cap,
                    int dtype, void* out, float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  if (!q || !k || !v || !out || !lse) return AFFMAE_ERR_NULL;
  int rc = check_attn(B, Nq, Nk, H, Hk, d, dtype);
  if (rc != AFFMAE_OK) return rc;
  rc = check_terms(scale, cap, q_xy, k_xy, slope, q_doc, k_doc);
  if (rc != AFFMAE_OK) return rc;
  if (misaligned(q, 16) || misaligned(k, 16) || misaligned(v, 16) || misaligned(out, 16) || misaligned(lse, 4)) return AFFMAE_ERR_SHAPE;
  const size_t need = affmae_attn_fwd_workspace_bytes(B, Nq, Nk, H, Hk, d, dtype, q_doc != nullptr);
  if (need && (!workspace || workspace_bytes < need || misaligned(workspace, kAlign))) return AFFMAE_ERR_WORKSPACE;
  affmae::AttnArgs a = {};
  a.q = q; a.k = k; a.v = v; a.q_xy = q_xy; a.k_xy = k_xy; a.slope = slope; a.q_doc = q_doc; a.k_doc = k_doc;
  a.B = B; a.Nq = Nq; a.Nk = Nk; a.H = H; a.Hk = Hk; a.d = d; a.dtype = dtype; a.scale = scale; a.cap = cap;
  a.out = out; a.lse = lse; a.workspace = workspace;
  return status(affmae::launch_attn_fwd(a, static_cast<hipStream_t>(stream)));
}

size_t affmae_attn_bwd_workspace_bytes(int B, int Nq, int Nk, int H, int Hk, int d, int dtype, int docs, int want_dslope) {
  if (check_attn(B, Nq, Nk, H, Hk, d, dtype) != AFFMAE_OK) return 0;
  return align_up(affmae::attn_bwd_workspace_bytes(B, Nq, Nk, H, Hk, d, dtype, docs != 0, want_dslope != 0));
}

int affmae_attn_bwd(const void* q, const void* k, const void* v, const float* q_xy, const float* k_xy, const float* slope,
                    const int32_t* q_doc, const int32_t* k_doc, const void* out, const float* lse, const void* dout, int B, int Nq,
                    int Nk, int H, int Hk, int d, float scale, float cap, int dtype, void* dq, void* dk, void* dv, float* dslope,
                    void* workspace, size_t workspace_bytes, void* stream) {
  if (!q || !k || !v || !out || !lse || !dout || !dq || !dk || !dv || (dslope && !slope)) return AFFMAE_ERR_NULL;
  int rc = check_attn(B, Nq, Nk, H, Hk, d, dtype);
  if (rc != AFFMAE_OK) return rc;
  rc = check_terms(scale, cap, q_xy, k_xy, slope, q_doc, k_doc);
  if (rc != AFFMAE_OK) return rc;
  if (misaligned(q, 16) || misaligned(k, 16) || misaligned(v, 16) || misaligned(out, 16) || misaligned(dout, 16) || misaligned(dq, 16) || misaligned(dk, 16) ||
      misaligned(dv, 16) || misaligned(lse, 4) || misaligned(dslope, 4))
    return AFFMAE_ERR_SHAPE;
  const size_t need = affmae_attn_bwd_workspace_bytes(B, Nq, Nk, H, Hk, d, dtype, q_doc != nullptr, dslope != nullptr);
  if (need && (!workspace || workspace_bytes < need || misaligned(workspace, kAlign))) return AFFMAE_ERR_WORKSPACE;
  affmae::AttnArgs a = {};
  a.q = q; a.k = k; a.v = v; a.q_xy = q_xy; a.k_xy = k_xy; a.slope = slope; a.q_doc = q_doc; a.k_doc = k_doc;
  a.B = B; a.Nq = Nq; a.Nk = Nk; a.H = H; a.Hk = Hk; a.d = d; a.dtype = dtype; a.scale = scale; a.cap = cap;
  a.out = const_cast<void*>(out); a.lse = const_cast<float*>(lse); a.dout = dout;
  a.dq = dq; a.dk = dk; a.dv = dv; a.dslope = dslope; a.workspace = workspace;
  return status(affmae::launch_attn_bwd(a, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
