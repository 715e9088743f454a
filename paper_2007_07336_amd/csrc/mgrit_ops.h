// Launch descriptors of the operators around the solver: end layers, loss, clipping.  Internal, as mgrit_internal.h.
#pragma once
#include "../../include/mgrit.h"
#include "mgrit_internal.h"

namespace mgrit {

// A packed array: codes [rows][pitch bytes], scales [slabs][rows][8] (a slab is 256 columns)
struct Packed {
  unsigned char* codes;
  unsigned char* scales;
  long long rows, cols, slabs, pitch;
  int format;
};
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
  // in 8 bits, p and f only saying whether there is one: p itself, and the factor
  const Packed *p8, *f8;
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

// out = what e makes of the sums of `parts` arrays [I][J], one behind the other
hipError_t join_parts(const Epilogue& e, const float* partial, int parts, long long I, long long J, hipStream_t s);

// The backward pass of an end layer: G = dY * D (D null: dY, with `scale` on every result), dX = G W, dW = G^T X, db = column
// sums of G; dX, dW, db null where they are not wanted.
struct BackwardArgs {
  long long M, K, F;
  int xtype, wtype, ytype, dxtype;
  float scale;
  const void* X;  const void* W;  const void* D;  const void* dY;
  void* dX;  float* dW;  float* db;
  Packed X8, D8;                     // X and D in 8 bits (with codes; xtype is bf16 then, X and D only say whether there is one)
};
size_t     backward_workspace(const BackwardArgs& b);
bool       backward_reads_kept(const BackwardArgs& b);                     // whether launch_backward takes X8 and D8, or they have to be unpacked
hipError_t launch_backward(const BackwardArgs& b, void* ws, hipStream_t s);
hipError_t launch_zero(float* out, long long n, hipStream_t s);

Packed     packed_view(long long rows, long long cols, int format, void* p);
size_t     packed_bytes(long long rows, long long cols, int format);
// rows at X, cols entries each
hipError_t launch_pack(const Packed& p, const void* X, int type, hipStream_t s);
// out: rows `ld` entries apart, zeros from cols on; rows without entries (0) are passed over
struct Unpack { Packed from; void* out; int type; long long ld; };
hipError_t launch_unpack(const Unpack* arrays, int n, hipStream_t s);      // one or two in one launch
struct PackedProduct {
  long long M, K, F;
  int xtype, xformat;
  const void* X;
  const void* W;                     // packed
  Epilogue e;
};
size_t     packed_product_workspace(const PackedProduct& q);
hipError_t launch_packed_product(const PackedProduct& q, void* ws, hipStream_t s);

struct BlockNormArgs {
  long long M, q;
  int layer, gate_kind, stype, ftype;
  float eps, scale;
  const void* f;  const void* r;  const void* gate;  const float* post;  const float* pre;     // r: S in the backward pass
  void* S;  void* Y;
  const void* dS;  const void* dY;
  void* df;  void* dr;  void* dgate;  float* dpost;  float* dpre;
};
hipError_t launch_block_norm(const BlockNormArgs& a, hipStream_t s);
size_t     block_norm_workspace(const BlockNormArgs& a);
hipError_t launch_block_norm_backward(const BlockNormArgs& a, void* ws, hipStream_t s);

struct SampleArgs {
  const void* logits;
  const float *u, *temperature;
  const int32_t* top_k;
  const float *top_p, *min_p;
  int64_t* index;  float* logprob;
  int B, V, dtype;
};
hipError_t launch_sample(const SampleArgs& a, hipStream_t s);

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
