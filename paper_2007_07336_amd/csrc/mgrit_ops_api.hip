// C entry points of the operators around the solver (end layers, loss, clipping, packed values, block norms, sampling): argument checks, workspace layout and
// the order of the launches.  The arithmetic is in mgrit_affine.hip, mgrit_loss.hip, mgrit_clip.hip,
// mgrit_packed.hip, mgrit_norm.hip and mgrit_sample.hip.
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
  return BackwardArgs{p->M, p->K, p->F, p->xtype, p->wtype, p->ytype, p->xtype, D ? 1.0f : p->scale, X, W, D, dY, dX, dW, db};
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

int check_packed(const mgrit_packed_t* p) {
  if (!p) return MGRIT_ERR_POINTER;
  if (p->rows < 0 || p->cols < 1 || (p->format != MGRIT_MX8 && p->format != MGRIT_MX4) || !good_type(p->dtype)) return MGRIT_ERR_PROBLEM;
  if ((long long)p->rows * ((p->cols + 255LL) / 256 * 256) > 1LL << 38) return MGRIT_ERR_UNSUPPORTED;
  return MGRIT_OK;
}
int check_affine_packed(const mgrit_affine_packed_t* p) {
  if (!p) return MGRIT_ERR_POINTER;
  if (p->M < 0 || p->K < 1 || p->F < 1) return MGRIT_ERR_PROBLEM;
  if (p->act != MGRIT_ACT_TANH && p->act != MGRIT_ACT_RELU && p->act != MGRIT_ACT_IDENTITY) return MGRIT_ERR_PROBLEM;
  if (!good_type(p->xtype) || !good_type(p->ytype) || (p->xformat != MGRIT_BF16 && p->xformat != MGRIT_MX4) || !isfinite(p->scale)) return MGRIT_ERR_PROBLEM;
  // (offsets within a tile's rows of codes are 31 bits)
  const long long M = p->M, K = (p->K + 255LL) / 256 * 256, F = p->F, most = 1LL << 38;
  if (K > 1LL << 22 || M * K > most || F * K > most || M * F > most) return MGRIT_ERR_UNSUPPORTED;
  return MGRIT_OK;
}
PackedProduct packed_product(const mgrit_affine_packed_t* p, const void* X, const void* W, const float* b, const void* R, void* Y, void* D) {
  PackedProduct q = {};
  q.M = p->M; q.K = p->K; q.F = p->F;
  q.xtype = p->xtype; q.xformat = p->xformat;
  q.X = X; q.W = W;
  q.e = Epilogue{1, p->act, p->ytype, p->scale, b, R, Y, D};
  return q;
}
// What a backward pass from kept activations has to unpack first: X as bf16 and D as its type, where the products do not read them as they are; the rest of the
// workspace behind them
struct KeptPlaces { bool reads; size_t D, bytes; };
KeptPlaces kept_places(const mgrit_affine_t* p) {
  KeptPlaces k = {};
  k.reads = backward_reads_kept(BackwardArgs{p->M, p->K, p->F, MGRIT_BF16, p->wtype, p->ytype, p->xtype});
  k.D = k.reads ? 0 : up((size_t)p->M * p->K * 2);
  k.bytes = k.reads ? 0 : k.D + up((size_t)p->M * p->F * (p->ytype ? 2 : 4));
  return k;
}
BackwardArgs kept_args(const mgrit_affine_t* p, const void* X, const void* W, const void* D, const void* dY, void* dX, float* dW, float* db) {
  BackwardArgs b = backward_args(p, X, W, D, dY, dX, dW, db);
  b.xtype = MGRIT_BF16;
  if (kept_places(p).reads) {
    if (X) b.X8 = packed_view(p->M, p->K, MGRIT_MX8, const_cast<void*>(X));
    if (D) b.D8 = packed_view(p->M, p->F, MGRIT_MX8, const_cast<void*>(D));
  }
  return b;
}

int check_norm(const mgrit_block_norm_t* p) {
  if (!p) return MGRIT_ERR_POINTER;
  if (p->M < 0 || p->q < 1 || (p->kind != MGRIT_NORM_ROOT && p->kind != MGRIT_NORM_LAYER)) return MGRIT_ERR_PROBLEM;
  if (p->gate != MGRIT_GATE_NONE && p->gate != MGRIT_GATE_FEATURE && p->gate != MGRIT_GATE_ENTRY) return MGRIT_ERR_PROBLEM;
  if (!good_type(p->stype) || !good_type(p->ftype) || !isfinite(p->eps) || !(p->eps >= 0.0f) || !isfinite(p->scale)) return MGRIT_ERR_PROBLEM;
  if ((long long)p->M * p->q > 1LL << 38) return MGRIT_ERR_UNSUPPORTED;
  return MGRIT_OK;
}
BlockNormArgs norm_args(const mgrit_block_norm_t* p, const void* f, const void* r, const void* gate, const float* post, const float* pre) {
  BlockNormArgs a = {};
  a.M = p->M; a.q = p->q;
  a.layer = p->kind == MGRIT_NORM_LAYER; a.gate_kind = p->gate; a.stype = p->stype; a.ftype = p->ftype;
  a.eps = p->eps; a.scale = p->scale;
  a.f = f; a.r = r; a.gate = gate; a.post = post; a.pre = pre;
  return a;
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

size_t mgrit_packed_bytes(const mgrit_packed_t* p) { return check_packed(p) == MGRIT_OK && p->rows ? packed_bytes(p->rows, p->cols, p->format) : 0; }

int32_t mgrit_pack(const mgrit_packed_t* p, const void* X, void* packed, void* hip_stream) {
  const int rc = check_packed(p);
  if (rc != MGRIT_OK) return rc;
  if (p->rows == 0) return MGRIT_OK;
  if (!X || !packed || !aligned_to(X, 16) || !aligned_to(packed, 256)) return MGRIT_ERR_POINTER;
  return launch_pack(packed_view(p->rows, p->cols, p->format, packed), X, p->dtype, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? MGRIT_OK : MGRIT_ERR_HIP;
}
int32_t mgrit_unpack(const mgrit_packed_t* p, const void* packed, void* X, void* hip_stream) {
  const int rc = check_packed(p);
  if (rc != MGRIT_OK) return rc;
  if (p->rows == 0) return MGRIT_OK;
  if (!X || !packed || !aligned_to(X, 16) || !aligned_to(packed, 256)) return MGRIT_ERR_POINTER;
  const Unpack u = {packed_view(p->rows, p->cols, p->format, const_cast<void*>(packed)), X, p->dtype, p->cols};
  return launch_unpack(&u, 1, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? MGRIT_OK : MGRIT_ERR_HIP;
}

size_t mgrit_affine_packed_workspace_bytes(const mgrit_affine_packed_t* p) {
  if (check_affine_packed(p) != MGRIT_OK || p->M == 0) return 0;
  return packed_product_workspace(packed_product(p, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr));
}

int32_t mgrit_affine_packed_forward(const mgrit_affine_packed_t* p, const void* X, const void* W, const float* b, const void* R, void* Y,
                                    void* D, void* workspace, size_t workspace_bytes, void* hip_stream) {
  const int rc = check_affine_packed(p);
  if (rc != MGRIT_OK) return rc;
  if (p->M == 0) return MGRIT_OK;
  const size_t need = mgrit_affine_packed_workspace_bytes(p);
  if (!X || !W || !Y || (need && !workspace) || !aligned_to(W, 256)) return MGRIT_ERR_POINTER;
  for (const void* q : {X, static_cast<const void*>(b), R, static_cast<const void*>(Y), static_cast<const void*>(D), static_cast<const void*>(workspace)})
    if (!aligned_to(q, 16)) return MGRIT_ERR_POINTER;
  if (workspace_bytes < need) return MGRIT_ERR_WORKSPACE;
  const PackedProduct q = packed_product(p, X, W, b, R, Y, D);
  return launch_packed_product(q, workspace, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? MGRIT_OK : MGRIT_ERR_HIP;
}

size_t mgrit_affine_kept_workspace_bytes(const mgrit_affine_t* p) {
  if (check_affine(p) != MGRIT_OK || p->M == 0) return 0;
  // (whether a call brings factors and what it wants is not known here, see mgrit_affine_backward_workspace_bytes)
  void* there = const_cast<mgrit_affine_t*>(p);
  float* also = static_cast<float*>(there);
  const size_t with = backward_workspace(kept_args(p, there, there, there, there, there, also, also));
  return kept_places(p).bytes + larger(with, backward_workspace(kept_args(p, there, there, nullptr, there, there, also, also)));
}

int32_t mgrit_affine_kept_backward(const mgrit_affine_t* p, const void* X, const void* W, const void* D, const void* dY, void* dX,
                                   float* dW, float* db, void* workspace, size_t workspace_bytes, void* hip_stream) {
  const int rc = check_affine(p);
  if (rc != MGRIT_OK) return rc;
  const hipStream_t s = static_cast<hipStream_t>(hip_stream);
  if (p->M == 0) return mgrit_affine_backward(p, nullptr, nullptr, nullptr, nullptr, nullptr, dW, db, nullptr, 0, hip_stream);
  const size_t need = mgrit_affine_kept_workspace_bytes(p);
  if (!dY || (need && !workspace) || (dX && !W) || (dW && !X)) return MGRIT_ERR_POINTER;
  if (!D && p->act != MGRIT_ACT_IDENTITY) return MGRIT_ERR_POINTER;
  for (const void* q : {W, dY, static_cast<const void*>(dX), static_cast<const void*>(dW), static_cast<const void*>(db), static_cast<const void*>(workspace)})
    if (!aligned_to(q, 16)) return MGRIT_ERR_POINTER;
  if (!aligned_to(X, 256) || !aligned_to(D, 256)) return MGRIT_ERR_POINTER;
  if (workspace_bytes < need) return MGRIT_ERR_WORKSPACE;
  if (!dX && !dW && !db) return MGRIT_OK;
  const KeptPlaces at = kept_places(p);
  char* base = static_cast<char*>(workspace);
  if (!at.reads) {
    Unpack u[2];
    int n = 0;
    if (dW) u[n++] = Unpack{packed_view(p->M, p->K, MGRIT_MX8, const_cast<void*>(X)), base, MGRIT_BF16, p->K};
    if (D) u[n++] = Unpack{packed_view(p->M, p->F, MGRIT_MX8, const_cast<void*>(D)), base + at.D, p->ytype, p->F};
    if (n && launch_unpack(u, n, s) != hipSuccess) return MGRIT_ERR_HIP;
    X = base;
    if (D) D = base + at.D;
  }
  return launch_backward(kept_args(p, X, W, D, dY, dX, dW, db), base + at.bytes, s) == hipSuccess ? MGRIT_OK : MGRIT_ERR_HIP;
}

int32_t mgrit_block_norm_forward(const mgrit_block_norm_t* p, const void* f, const void* r, const void* gate, const float* w_post,
                                 const float* w_pre, void* S, void* Y, void* hip_stream) {
  const int rc = check_norm(p);
  if (rc != MGRIT_OK) return rc;
  if (p->M == 0) return MGRIT_OK;
  if (!f || !r || !S || !w_pre != !Y || !gate != (p->gate == MGRIT_GATE_NONE)) return MGRIT_ERR_POINTER;
  for (const void* q : {f, r, gate, static_cast<const void*>(w_post), static_cast<const void*>(w_pre), static_cast<const void*>(S), static_cast<const void*>(Y)})
    if (!aligned_to(q, 16)) return MGRIT_ERR_POINTER;
  BlockNormArgs a = norm_args(p, f, r, gate, w_post, w_pre);
  a.S = S; a.Y = Y;
  return launch_block_norm(a, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? MGRIT_OK : MGRIT_ERR_HIP;
}

size_t mgrit_block_norm_workspace_bytes(const mgrit_block_norm_t* p) {
  return check_norm(p) == MGRIT_OK && p->M ? block_norm_workspace(norm_args(p, nullptr, nullptr, nullptr, nullptr, nullptr)) : 0;
}

int32_t mgrit_block_norm_backward(const mgrit_block_norm_t* p, const void* f, const void* S, const void* gate, const float* w_post,
                                  const float* w_pre, const void* dS, const void* dY, void* df, void* dr, void* dgate, float* dw_post,
                                  float* dw_pre, void* workspace, size_t workspace_bytes, void* hip_stream) {
  const int rc = check_norm(p);
  if (rc != MGRIT_OK) return rc;
  const hipStream_t s = static_cast<hipStream_t>(hip_stream);
  for (const void* q : {f, S, gate, static_cast<const void*>(w_post), static_cast<const void*>(w_pre), dS, dY, static_cast<const void*>(df),
                        static_cast<const void*>(dr), static_cast<const void*>(dgate), static_cast<const void*>(dw_post), static_cast<const void*>(dw_pre),
                        static_cast<const void*>(workspace)})
    if (!aligned_to(q, 16)) return MGRIT_ERR_POINTER;
  if (dgate && p->gate == MGRIT_GATE_NONE) return MGRIT_ERR_POINTER;
  if (p->M == 0) {
    hipError_t e = hipSuccess;
    float* const gates = p->gate == MGRIT_GATE_FEATURE ? static_cast<float*>(dgate) : nullptr;
    for (float* out : {dw_post, dw_pre, gates})
      if (e == hipSuccess && out) e = launch_zero(out, p->q, s);
    return e == hipSuccess ? MGRIT_OK : MGRIT_ERR_HIP;
  }
  const size_t need = mgrit_block_norm_workspace_bytes(p);
  if (!f || !workspace || (w_pre && !S) || !w_pre != !dY || !gate != (p->gate == MGRIT_GATE_NONE)) return MGRIT_ERR_POINTER;
  if ((dw_post && !w_post) || (dw_pre && !w_pre)) return MGRIT_ERR_POINTER;
  if (workspace_bytes < need) return MGRIT_ERR_WORKSPACE;
  if (!df && !dr && !dgate && !dw_post && !dw_pre) return MGRIT_OK;
  BlockNormArgs a = norm_args(p, f, S, gate, w_post, w_pre);
  a.dS = dS; a.dY = dY; a.df = df; a.dr = dr; a.dgate = dgate; a.dpost = dw_post; a.dpre = dw_pre;
  return launch_block_norm_backward(a, workspace, s) == hipSuccess ? MGRIT_OK : MGRIT_ERR_HIP;
}

size_t mgrit_sample_workspace_bytes(const mgrit_sample_t*) { return 0; }

int32_t mgrit_sample(const mgrit_sample_t* p, const void* logits, const float* u, const float* temperature, const int32_t* top_k, const float* top_p,
                     const float* min_p, int64_t* index, float* logprob, void* workspace, size_t, void* hip_stream) {
  if (!p) return MGRIT_ERR_POINTER;
  if (p->B < 0 || p->V < 1 || !good_type(p->dtype)) return MGRIT_ERR_PROBLEM;
  if ((long long)p->B * p->V > 1LL << 38) return MGRIT_ERR_UNSUPPORTED;
  if (p->B == 0) return MGRIT_OK;
  if (!logits || !u || !index) return MGRIT_ERR_POINTER;
  for (const void* q : {logits, static_cast<const void*>(u), static_cast<const void*>(temperature), static_cast<const void*>(top_k), static_cast<const void*>(top_p),
                        static_cast<const void*>(min_p), static_cast<const void*>(index), static_cast<const void*>(logprob), static_cast<const void*>(workspace)})
    if (!aligned_to(q, 16)) return MGRIT_ERR_POINTER;
  const SampleArgs a = {logits, u, temperature, top_k, top_p, min_p, index, logprob, p->B, p->V, p->dtype};
  return launch_sample(a, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? MGRIT_OK : MGRIT_ERR_HIP;
}

}  // extern "C"
