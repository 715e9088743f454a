// Launch descriptors of the operators around the solver: end layers, loss, clipping.  Internal, as mgrit_internal.h.
#pragma once
#include "../../include/mgrit.h"
#include "mgrit_internal.h"

namespace mgrit {

// One operand of a product C[i][j] = sum_k A(i, k) B(j, k): entry (r, k) lies at p[r * ld + k], or with kslow at p[k * ld + r].
// With a factor it is p * f, entry by entry (the gradient at an activation's input; f has p's type and layout).
struct Operand {
  const void* p;
  const void* f;
  long long ld;
  int type;                          // 0 float, 1 bf16
  int kslow;
  // set for planes in the workspace: rows end in zeros up to ld, and the operand is the sum of `parts` planes, `part` entries apart, each on its scale
  int padded, parts;
  long long part;
};
// What becomes of a sum.  Forward (fwd): z = sum + bias, out = R + scale act(z), D = scale act'(z); else out = scale sum.
struct Epilogue {
  int fwd, act, otype;               // otype: of out, R and D
  float scale;
  const float* bias;
  const void* R;
  void* out;
  void* D;
};
struct Product {
  Operand A, B;
  Epilogue e;
  long long I, J, Kc;                // rows, columns (out is [I][J]) and contraction length
};

size_t     product_workspace(const Product& q);
hipError_t launch_product(const Product& q, void* ws, hipStream_t s);

// The backward pass of an end layer: G = dY * D (D null: dY, with `scale` on every result), dX = G W, dW = G^T X, db = column
// sums of G; dX, dW, db null where they are not wanted.
struct BackwardArgs {
  long long M, K, F;
  int xtype, wtype, ytype;
  float scale;
  const void* X;  const void* W;  const void* D;  const void* dY;
  void* dX;  float* dW;  float* db;
};
size_t     backward_workspace(const BackwardArgs& b);
hipError_t launch_backward(const BackwardArgs& b, void* ws, hipStream_t s);
hipError_t launch_zero(float* out, long long n, hipStream_t s);

struct LossArgs {
  const void* logits;
  const int64_t* labels;
  float* loss;  float* rows;  void* grad;
  int B, V, dtype, mean;
  float scale;
};
size_t     loss_workspace(const LossArgs& a);
hipError_t launch_loss(const LossArgs& a, void* ws, hipStream_t s);

size_t     clip_workspace(int filled);                 // tensors that have entries; the others are passed over
// norm_dev <- where the norm lies in the workspace as a double
hipError_t launch_clip(int n, const mgrit_tensor_t* t, float max_norm, float* norm, void* ws, const double** norm_dev, hipStream_t s);

}  // namespace mgrit
