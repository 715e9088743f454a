// C entry points of the operators around the solver (end layers, loss, clipping): argument checks, workspace layout and
// the order of the launches.  The arithmetic is in mgrit_affine.hip, mgrit_loss.hip and mgrit_clip.hip.
#include <math.h>

#include "../../include/mgrit.h"
#include "mgrit_ops.h"

using namespace mgrit;

namespace {

inline size_t up(size_t x) { return (x + 255) / 256 * 256; }
inline bool aligned_to(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
inline bool good_type(int t) { return t == MGRIT_FP32 || t == MGRIT_BF16; }

int check_affine(const mgrit_affine_t* p) {
  if (!p) return MGRIT_ERR_POINTER;
  if (p->M < 0 || p->K < 1 || p->F < 1) return MGRIT_ERR_PROBLEM;
  if (p->act != MGRIT_ACT_TANH && p->act != MGRIT_ACT_RELU && p->act != MGRIT_ACT_IDENTITY) return MGRIT_ERR_PROBLEM;
  if (!good_type(p->xtype) || !good_type(p->wtype) || !good_type(p->ytype) || !isfinite(p->scale)) return MGRIT_ERR_PROBLEM;
  const long long M = p->M, K = p->K, F = p->F, most = 1LL << 38;
  if (M * K > most || F * K > most || M * F > most) return MGRIT_ERR_UNSUPPORTED;
  return MGRIT_OK;
}

Product forward_product(const mgrit_affine_t* p, const void* X, const void* W, const float* b, const void* R, void* Y, void* D) {
  Product q = {};
  q.A = Operand{X, nullptr, p->K, p->xtype, 0};
  q.B = Operand{W, nullptr, p->K, p->wtype, 0};
  q.e = Epilogue{1, p->act, p->ytype, p->scale, b, R, Y, D};
  q.I = p->M; q.J = p->F; q.Kc = p->K;
  return q;
}
BackwardArgs backward_args(const mgrit_affine_t* p, const void* X, const void* W, const void* D, const void* dY, void* dX, float* dW, float* db) {
  // (the factors hold the layer's scale already)
  return BackwardArgs{p->M, p->K, p->F, p->xtype, p->wtype, p->ytype, D ? 1.0f : p->scale, X, W, D, dY, dX, dW, db};
}
inline size_t larger(size_t a, size_t b) { return a > b ? a : b; }

int check_loss(const mgrit_loss_t* p) {
  if (!p) return MGRIT_ERR_POINTER;
  if (p->B < 0 || p->V < 1 || !good_type(p->dtype) || !isfinite(p->scale)) return MGRIT_ERR_PROBLEM;
  if (p->reduction != MGRIT_LOSS_SUM && p->reduction != MGRIT_LOSS_MEAN) return MGRIT_ERR_PROBLEM;
  if ((long long)p->B * p->V > 1LL << 38) return MGRIT_ERR_UNSUPPORTED;
  return MGRIT_OK;
}
LossArgs loss_args(const mgrit_loss_t* p) {
  LossArgs a = {};
  a.B = p->B; a.V = p->V; a.dtype = p->dtype; a.mean = p->reduction == MGRIT_LOSS_MEAN; a.scale = p->scale;
  return a;
}

// filled: how many of the tensors have entries
int check_tensors(const mgrit_tensor_t* t, int32_t n, int* filled) {
  *filled = 0;
  if (n < 0) return MGRIT_ERR_PROBLEM;
  if (n > 0 && !t) return MGRIT_ERR_POINTER;
  long long total = 0;
  for (int i = 0; i < n; ++i) {
    if (t[i].count < 0 || !good_type(t[i].dtype)) return MGRIT_ERR_PROBLEM;
    if (t[i].count > (1LL << 40) || (total += t[i].count) > (1LL << 40)) return MGRIT_ERR_UNSUPPORTED;
    if (t[i].count == 0) continue;
    const size_t e = t[i].dtype == MGRIT_FP32 ? 4 : 2;
    if (!t[i].src || !aligned_to(t[i].src, e) || !aligned_to(t[i].dst, e)) return MGRIT_ERR_POINTER;
    ++*filled;
  }
  return MGRIT_OK;
}

}  // namespace

extern "C" {

size_t mgrit_affine_workspace_bytes(const mgrit_affine_t* p) {
  if (check_affine(p) != MGRIT_OK || p->M == 0) return 0;
  return product_workspace(forward_product(p, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr));
}

size_t mgrit_affine_backward_workspace_bytes(const mgrit_affine_t* p) {
  if (check_affine(p) != MGRIT_OK || p->M == 0) return 0;
  // whether a call brings factors and what it wants is not known here: room for all of it (the pointers only say what is there)
  void* there = const_cast<mgrit_affine_t*>(p);
  float* also = static_cast<float*>(there);
  const size_t with = backward_workspace(backward_args(p, there, there, there, there, there, also, also));
  return larger(with, backward_workspace(backward_args(p, there, there, nullptr, there, there, also, also)));
}

int32_t mgrit_affine_forward(const mgrit_affine_t* p, const void* X, const void* W, const float* b, const void* R, void* Y,
                             void* D, void* workspace, size_t workspace_bytes, void* hip_stream) {
  const int rc = check_affine(p);
  if (rc != MGRIT_OK) return rc;
  if (p->M == 0) return MGRIT_OK;
  const size_t need = mgrit_affine_workspace_bytes(p);
  if (!X || !W || !Y || (need && !workspace)) return MGRIT_ERR_POINTER;
  for (const void* q : {X, W, static_cast<const void*>(b), R, static_cast<const void*>(Y), static_cast<const void*>(D),
                        static_cast<const void*>(workspace)})
    if (!aligned_to(q, 16)) return MGRIT_ERR_POINTER;
  if (workspace_bytes < need) return MGRIT_ERR_WORKSPACE;
  const Product q = forward_product(p, X, W, b, R, Y, D);
  return launch_product(q, workspace, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? MGRIT_OK : MGRIT_ERR_HIP;
}

int32_t mgrit_affine_backward(const mgrit_affine_t* p, const void* X, const void* W, const void* D, const void* dY, void* dX,
                              float* dW, float* db, void* workspace, size_t workspace_bytes, void* hip_stream) {
  const int rc = check_affine(p);
  if (rc != MGRIT_OK) return rc;
  const hipStream_t s = static_cast<hipStream_t>(hip_stream);
  if (!aligned_to(dW, 16) || !aligned_to(db, 16)) return MGRIT_ERR_POINTER;
  hipError_t e = hipSuccess;
  if (p->M == 0) {
    if (dW) e = launch_zero(dW, (long long)p->F * p->K, s);
    if (e == hipSuccess && db) e = launch_zero(db, p->F, s);
    return e == hipSuccess ? MGRIT_OK : MGRIT_ERR_HIP;
  }
  const size_t need = mgrit_affine_backward_workspace_bytes(p);
  if (!dY || (need && !workspace) || (dX && !W) || (dW && !X)) return MGRIT_ERR_POINTER;
  if (!D && p->act != MGRIT_ACT_IDENTITY) return MGRIT_ERR_POINTER;
  for (const void* q : {X, W, D, dY, static_cast<const void*>(dX), static_cast<const void*>(workspace)})
    if (!aligned_to(q, 16)) return MGRIT_ERR_POINTER;
  if (workspace_bytes < need) return MGRIT_ERR_WORKSPACE;
  if (dX || dW || db) e = launch_backward(backward_args(p, X, W, D, dY, dX, dW, db), workspace, s);
  return e == hipSuccess ? MGRIT_OK : MGRIT_ERR_HIP;
}

size_t mgrit_cross_entropy_workspace_bytes(const mgrit_loss_t* p) {
  return check_loss(p) == MGRIT_OK ? loss_workspace(loss_args(p)) : 0;
}

int32_t mgrit_cross_entropy(const mgrit_loss_t* p, const void* logits, const int64_t* labels, float* loss, float* row_loss,
                            void* grad, void* workspace, size_t workspace_bytes, void* hip_stream) {
  const int rc = check_loss(p);
  if (rc != MGRIT_OK) return rc;
  const size_t need = mgrit_cross_entropy_workspace_bytes(p);
  if ((p->B > 0 && (!logits || !labels)) || (need && !workspace)) return MGRIT_ERR_POINTER;
  for (const void* q : {logits, static_cast<const void*>(labels), static_cast<const void*>(loss), static_cast<const void*>(row_loss),
                        static_cast<const void*>(grad), static_cast<const void*>(workspace)})
    if (!aligned_to(q, 16)) return MGRIT_ERR_POINTER;
  if (workspace_bytes < need) return MGRIT_ERR_WORKSPACE;
  LossArgs a = loss_args(p);
  a.logits = logits; a.labels = labels; a.loss = loss; a.rows = row_loss; a.grad = grad;
  if (!loss && !row_loss && !grad) return MGRIT_OK;
  return launch_loss(a, workspace, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? MGRIT_OK : MGRIT_ERR_HIP;
}

size_t mgrit_clip_workspace_bytes(const mgrit_tensor_t* tensors, int32_t n) {
  int filled = 0;
  return check_tensors(tensors, n, &filled) == MGRIT_OK ? clip_workspace(filled) : 0;
}

int32_t mgrit_clip_gradients(const mgrit_tensor_t* tensors, int32_t n, float max_norm, float* norm, double* norm_host,
                             void* workspace, size_t workspace_bytes, void* hip_stream) {
  int filled = 0;
  const int rc = check_tensors(tensors, n, &filled);
  if (rc != MGRIT_OK) return rc;
  if (!(max_norm >= 0.0f)) return MGRIT_ERR_PROBLEM;
  if (!workspace || !aligned_to(workspace, 16) || !aligned_to(norm, 4)) return MGRIT_ERR_POINTER;
  if (workspace_bytes < clip_workspace(filled)) return MGRIT_ERR_WORKSPACE;
  const hipStream_t s = static_cast<hipStream_t>(hip_stream);
  const double* at = nullptr;
  if (launch_clip(n, tensors, max_norm, norm, workspace, &at, s) != hipSuccess) return MGRIT_ERR_HIP;
  if (norm_host) {
    if (hipMemcpyAsync(norm_host, at, sizeof(double), hipMemcpyDeviceToHost, s) != hipSuccess) return MGRIT_ERR_HIP;
    if (hipStreamSynchronize(s) != hipSuccess) return MGRIT_ERR_HIP;
    if (!isfinite(*norm_host)) return MGRIT_ERR_NONFINITE;
  }
  return MGRIT_OK;
}

}  // extern "C"
