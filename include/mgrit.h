/*
 * mgrit.h -- C ABI of the layer-parallel multigrid (MGRIT-FAS) solver for residual networks
 *            u^{n+1} = u^n + h F(u^n; theta^n),  n = 0..N-1          (paper Sec. II, Eq. (1))
 * on one AMD MI355X (gfx950).  Plain C: only pointers and sizes cross this boundary.
 *
 * Index convention.  N layer steps, N+1 states u^0..u^N ("points" 0..N), parameters
 * theta^0..theta^{N-1}.  The coarsening factor (the paper's c, Sec. III-C) is called m here.
 * Level l has N_l = N / m^l steps and step size h_l = m^l h; point j of level l is fine
 * point j m^l and uses theta^{j m^l} (injection of states, residuals and parameters,
 * Sec. III-C, Eq. (23)).
 *
 * Memory.  The caller owns every buffer.  Pointers marked "device" are HIP device pointers
 * aligned to 256 bytes; pointers marked "host" are ordinary host pointers.  The library
 * allocates no device memory and keeps no state of a solve between calls.  What it does keep, per
 * process, is bookkeeping: for every kernel that needs more than 64 KB of LDS, the largest size it
 * has been raised to on each device (the opt-in is a per-device attribute of the kernel, set at
 * the first launch that needs it), and the optional launch trace at the end of this file.  None
 * of this is guarded: call the library from one host thread at a time.  All device work is enqueued
 * on `hip_stream` (a hipStream_t passed as void*; NULL = the default stream).  A call that
 * writes a host output (resnorm_hist, iters_done, norm_out) synchronises that stream before
 * it returns; otherwise it returns with its work in flight on the stream.  Such a call (tol <= 0,
 * no host outputs) consists of kernel launches only, so it may be recorded into a HIP graph by
 * stream capture and replayed.  Run the same call once outside the capture first: the first launch of
 * a kernel that uses more than 64 KB of LDS sets an attribute of that kernel on the current device.
 *
 * Environment (diagnostic switches, read at every call; results agree with the default path to rounding).
 * MGRIT_NO_SWEEP=1 makes the library use one launch per layer step also where it would fuse many steps
 * into one launch: dense layers of width at most 256, in bf16 1024, and convolution layers whose images fit on a compute unit
 * (in float at most 16 channels and 1024 pixels or 32 and 512; in bf16 at most 48 channels or exactly 64 and 1024
 * pixels, 56 and 512; of stacks with fully connected layers the forward solve's levels in which those open intervals).  A level
 * with few samples and intervals takes one launch per step all the same where that is faster (float of width 136 to 256, bf16 wider
 * than 256, 64 channels on more than 512 pixels, the adjoint of 48 channels on more than 900).
 * MGRIT_ACT_VALUES=1 / 0 stores the act' factors of ReLU layers as values / as bits whatever their number.
 * MGRIT_GRAD_NARROW=1 keeps the
 * parameter gradient of dense layers of width 512 and more on the 128x128 tiles of narrower layers.
 * MGRIT_MASKED_STEP=1 sends dense layer steps whose batch, width and contraction length are whole multiples of
 * the tile through the bounds-masked loop that ragged shapes use.
 * MGRIT_STEP_REREAD=1 makes the epilogue of the bf16 128x128 dense tile read the state for the skip connection
 * from memory again instead of keeping it in registers from the contraction loop.
 * MGRIT_CGRAD_WAVES=4 runs the parameter gradient of convolution layers with more than 32 channels with four
 * wavefronts per workgroup, as for narrower layers, instead of eight.
 * MGRIT_CONV_GENERIC=1 keeps bf16 convolution layers of 64 channels on the kernel that takes the channel count at
 * run time instead of the one compiled for 64.
 * MGRIT_ADJ_TRANSPOSED=1 runs the adjoint of dense and fully connected layers on transposed copies of their
 * weights, made in the workspace at every call, instead of reading the caller's arrays along their slow index;
 * the workspace queries then include those copies, so set it before the query as well as before the call.
 *
 * Layouts (all row-major, last index fastest):
 *   dense: state [B][q] float;  W [N][q_out][q_in];  b [N][q] float
 *   conv : state [B][Himg][Wimg][C] float (NHWC);  W [N][C_out][3][3][C_in];  b [N][C] float
 *          3x3, stride 1, one pixel of zero padding, cross-correlation:
 *          z[b,y,x,o] = sum_{dy,dx,i} W[o][dy][dx][i] u[b,y+dy-1,x+dx-1,i] + b[o]
 *   W is float when dtype = MGRIT_FP32 and bf16 (upper 16 bits of a float, 2 bytes) when
 *   dtype = MGRIT_BF16.  With MGRIT_BF16 the matrix-core operands (weights and the state
 *   operand of the affine map; in the parameter gradient G = act' * Lam and U, and for conv
 *   layers also the G that is summed into db) are rounded to bf16 and everything else --
 *   accumulation, bias, activation, the skip add, states, residuals, corrections -- is float.
 *   State arrays over points are [N+1][state].
 *
 * Return value of every int32_t function: MGRIT_OK or one of the negative codes below.
 * Nothing is printed and nothing is thrown.
 */
#ifndef MGRIT_H
#define MGRIT_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

enum {
  MGRIT_OK = 0,
  MGRIT_ERR_POINTER = -1,     /* required pointer NULL or not 256-byte aligned              */
  MGRIT_ERR_PROBLEM = -2,     /* invalid problem: N < 1, m < 2, bad enum, sizes <= 0, ...    */
  MGRIT_ERR_WORKSPACE = -3,   /* workspace smaller than mgrit_*_workspace_bytes()            */
  MGRIT_ERR_UNSUPPORTED = -4, /* valid request that this build does not implement            */
  MGRIT_ERR_NONFINITE = -5,   /* a residual norm came out NaN or Inf                         */
  MGRIT_ERR_HIP = -6          /* a HIP runtime call failed                                   */
};

enum { MGRIT_RELAX_F = 0, MGRIT_RELAX_FCF = 1 };           /* Sec. III-C, Fig. 3, Alg. 1 step 1 */
enum { MGRIT_NORM_L2 = 0, MGRIT_NORM_RMS = 1 };            /* RMS = L2 / sqrt(#entries)         */
enum { MGRIT_LAYER_DENSE = 0, MGRIT_LAYER_CONV3X3 = 1 };
enum { MGRIT_ACT_TANH = 0, MGRIT_ACT_RELU = 1 };
enum { MGRIT_FP32 = 0, MGRIT_BF16 = 1 };
enum { MGRIT_INIT_ZERO = 0, MGRIT_INIT_COPY = 1, MGRIT_INIT_USER = 2, MGRIT_INIT_NESTED = 3 };
enum { MGRIT_MAX_LEVELS = 16 };

typedef struct mgrit_problem {
  int32_t N;           /* layer steps, >= 1 (at most 65535 in this build)     (Sec. II, Eq. (1)) */
  float   h;           /* fine step size                                      (Sec. II, Eq. (1)) */
  int32_t m;           /* coarsening factor, >= 2                             (Sec. III-C)       */
  int32_t max_levels;  /* 1 = serial propagation, 2 = two-level scheme of Alg. 1,
                          > 2 = the scheme applied recursively (V-cycle)      (Sec. III-A)       */
  int32_t min_coarse;  /* a level with N_l <= min_coarse is not coarsened further; values < 1
                          act as 1                                                               */
  int32_t relax;       /* MGRIT_RELAX_F or MGRIT_RELAX_FCF                    (Alg. 1 step 1)    */
  int32_t cycle;       /* 0 = V-cycle (the only one defined)                                     */
  int32_t max_iter;    /* number of cycles; with tol > 0 an upper bound       (Sec. IV-A)        */
  float   tol;         /* > 0: stop after the first cycle whose residual norm is <= tol
                          (Alg. 1 step 6); <= 0: run exactly max_iter cycles                     */
  int32_t norm_kind;   /* MGRIT_NORM_L2 or MGRIT_NORM_RMS                                        */
  int32_t layer;       /* MGRIT_LAYER_DENSE or MGRIT_LAYER_CONV3X3                                */
  int32_t act;         /* MGRIT_ACT_TANH or MGRIT_ACT_RELU                                       */
  int32_t dtype;       /* MGRIT_FP32 or MGRIT_BF16                                               */
  int32_t B, q;        /* dense: batch and width                                                 */
  int32_t C, Himg, Wimg; /* conv: channels, image height and width                               */
  int32_t init;        /* initial guess of the fine C-points: MGRIT_INIT_ZERO, MGRIT_INIT_COPY
                          (every C-point := the known end value u^0, resp. lambda^N),
                          MGRIT_INIT_USER (take them from the in/out array) or MGRIT_INIT_NESTED
                          (nested iteration: the coarsest level's equation L(V) = (u^0, 0, .., 0)
                          with its own step size is solved in sequence; going up, the C-points of
                          each level take the coarser level's values and its F-points follow by
                          F-relaxation, Sec. III-A / III-C; the paper prints no start-up procedure.
                          Costs N_coarsest + sum over the middle levels of N_l (m-1)/m layer steps) */
} mgrit_problem_t;

/* Level hierarchy (Sec. III-C: every m-th layer of a level is also a member of the next
 * coarser level).  Coarsening goes on while fewer than max_levels levels exist and the level
 * has more than min_coarse steps and at least m of them; N_{l+1} = floor(N_l / m), and a level
 * whose size is not a multiple of m ends in N_l mod m trailing F-points, which F-relaxation
 * updates behind the last C-point (a case the paper does not treat).  This is the hierarchy of
 * the forward solve; the adjoint solve uses the mirror image, counted from layer N (its
 * level-l points are the fine points N - j m^l).
 * Host only, integer only.  n_levels <- number of levels L; N_l[l] <- steps
 * on level l (array of MGRIT_MAX_LEVELS entries); fine_index <- concatenation over levels of
 * the fine point index of every point, sum_l (N_l + 1) entries.  N_l and fine_index may be
 * NULL (then only the count is returned).  Errors: MGRIT_ERR_PROBLEM. */
int32_t mgrit_level_map(const mgrit_problem_t* p, int32_t* n_levels, int32_t* N_l, int32_t* fine_index);

/* Bytes of device workspace the forward solve / residual norm, and the adjoint solve, need
 * for this problem; 0 if the problem is invalid.  Host only. */
size_t mgrit_workspace_bytes(const mgrit_problem_t* p);
size_t mgrit_adjoint_workspace_bytes(const mgrit_problem_t* p);

/* Forward solve of L_h(U) = f_h = (u0, 0, .., 0) (Sec. III-C, Eq. (18)) by max_iter FAS cycles
 * of Alg. 1: relaxation, residual at the C-points, injection, coarse FAS equation
 * L_H(V) = L_H(U_H) + R_H (Eq. (24)) solved recursively / serially on the coarsest level,
 * C-point correction, F-relaxation.  With max_levels = 1 this is serial propagation.
 *   W, b      device, read only
 *   u0        device [state], read only
 *   U         device [(N+1)][state]; out; with init = MGRIT_INIT_USER also in (its C-points)
 *   resnorm_hist  host [max_iter] or NULL; entry k <- norm of the C-point residual of the fine
 *             level evaluated in cycle k after relaxation and before the correction
 *   iters_done    host or NULL; <- cycles run
 *   workspace device, workspace_bytes >= mgrit_workspace_bytes(p)
 * Errors: all codes above; on MGRIT_ERR_NONFINITE U holds the diverged iterate. */
int32_t mgrit_fas_forward(const mgrit_problem_t* p, const void* W, const float* b, const float* u0,
                          float* U, double* resnorm_hist, int32_t* iters_done,
                          void* workspace, size_t workspace_bytes, void* hip_stream);

/* The forward solve for callers that cannot allocate device memory -- code under HIP graph capture, tight
 * serving loops, harnesses that forbid hipMalloc: mgrit_fas_forward without the workspace argument.  Its
 * workspace is a fixed array of MGRIT_STATIC_SCRATCH_BYTES in device memory that belongs to the library; every
 * GPU the library runs on holds one copy until the process ends.  The call itself allocates and frees nothing,
 * on the device or through any allocating runtime call; inputs and outputs are the caller's as above, results are
 * those of mgrit_fas_forward (same kernels, same schedule).
 *   - MGRIT_ERR_WORKSPACE if mgrit_workspace_bytes(p) exceeds MGRIT_STATIC_SCRATCH_BYTES (the plain dense
 *     q = 256, N = 256, B = 128 workload needs 32 MB; the two large benchmark workloads do not fit).
 *   - The first call on a device looks up the address of that device's copy of the array; make it outside
 *     a stream capture (the same rule as for the LDS attribute above).  With tol <= 0 and both host outputs
 *     NULL the call is kernel launches only.
 *   - All calls on one GPU share that GPU's array, whatever their streams: calls that overlap in time on one
 *     GPU race on it.  Nothing in it has to be cleared between calls -- every part is written before it is
 *     read -- so a call may follow one with a different problem.
 * Errors otherwise as mgrit_fas_forward; MGRIT_ERR_UNSUPPORTED for a device index above 63. */
enum { MGRIT_STATIC_SCRATCH_BYTES = 64 * 1024 * 1024 };
int32_t mgrit_fas_forward_static(const mgrit_problem_t* p, const void* W, const float* b, const float* u0,
                                 float* U, double* resnorm_hist, int32_t* iters_done, void* hip_stream);

/* Adjoint (backward) solve by the same cycle on the reversed layer axis.  The paper states
 * that the multigrid removes the serial backward propagation as well (Sec. III-C) and prints
 * no equations; the system solved is the exact reverse-mode derivative of Eq. (1):
 *   z^n = A_n U^n + b_n,  G^n = act'(z^n) * Lam^{n+1},  Lam^n = Lam^{n+1} + h A_n^T G^n,
 * with terminal value Lam^N = lamN, linearised about the given states U (converged or not);
 * the level-l step from point j+1 to point j uses U and theta of fine point j m^l and step h_l.
 * Afterwards dW[n] = h G^n (U^n)^T (summed over the batch / batch and pixels) and
 * db[n] = h sum G^n from the final Lam.
 *   U     device [(N+1)][state], read only      lamN  device [state], read only
 *   Lam   device [(N+1)][state]; out (in for init = MGRIT_INIT_USER)
 *   dW    device float, same shape as W (dense [N][q][q], conv [N][C][3][3][C]), overwritten, or NULL;
 *         db like b, or NULL
 *   workspace_bytes >= mgrit_adjoint_workspace_bytes(p)
 * resnorm_hist / iters_done as above (residual of the adjoint system). */
int32_t mgrit_fas_adjoint(const mgrit_problem_t* p, const void* W, const float* b, const float* U,
                          const float* lamN, float* Lam, float* dW, float* db,
                          double* resnorm_hist, int32_t* iters_done,
                          void* workspace, size_t workspace_bytes, void* hip_stream);

/* || f_h - L_h(U) || over all N+1 points of the fine level (Sec. III-C, Eq. (19); Sec. IV-A).
 *   norm_out  host, required.  Always synchronises the stream. */
int32_t mgrit_residual_norm(const mgrit_problem_t* p, const void* W, const float* b, const float* u0,
                            const float* U, double* norm_out,
                            void* workspace, size_t workspace_bytes, void* hip_stream);

/* ---- Stacks that mix convolution layers with periodic fully connected layers (Sec. IV-E: blocks of one
 * fully connected layer with equal input and output size followed by a run of residual convolution layers).
 * The problem is a MGRIT_LAYER_CONV3X3 problem; in addition every fc_period-th layer, n = 0, fc_period,
 * 2 fc_period, ... < N, is a fully connected layer acting on the flattened sample,
 *   u^{n+1}[b] = u^n[b] + h act(Wfc_k vec(u^n[b]) + bfc_k),   k = n / fc_period,
 * vec = the sample's [Himg][Wimg][C] values in storage order, d = Himg*Wimg*C of them.  The paper does not say
 * whether its fully connected layers carry the skip connection; here they do, so that every layer has the form of
 * Eq. (1).  Coarse levels inject layers as before (a coarse step uses the kind and parameters of its first fine
 * layer).  The slots of W, b (and dW, db) at the fully connected layers' indices keep the [N] layout: their
 * input values are ignored, and dW, db are written as zero there.
 *   fc_period  >= 2;  n_fc = ceil(N / fc_period)
 *   Wfc   device [n_fc][d][d] ([out][in], element type as W)   bfc   device [n_fc][d] float
 *   dWfc  device float [n_fc][d][d], dbfc device [n_fc][d]: adjoint only, overwritten; computed when dW / db are
 *         (dWfc with dW, dbfc with db) and then required
 * MGRIT_ERR_UNSUPPORTED if d*d exceeds 2^31 - 1.  Everything else is as in the plain entry points. */
typedef struct mgrit_fc_layers {
  int32_t     fc_period;
  const void* Wfc;
  const float* bfc;
  float*      dWfc;
  float*      dbfc;
} mgrit_fc_layers_t;

size_t  mgrit_workspace_bytes_mixed(const mgrit_problem_t* p, int32_t fc_period);
size_t  mgrit_adjoint_workspace_bytes_mixed(const mgrit_problem_t* p, int32_t fc_period);
int32_t mgrit_fas_forward_mixed(const mgrit_problem_t* p, const mgrit_fc_layers_t* fc, const void* W, const float* b,
                                const float* u0, float* U, double* resnorm_hist, int32_t* iters_done,
                                void* workspace, size_t workspace_bytes, void* hip_stream);
int32_t mgrit_fas_adjoint_mixed(const mgrit_problem_t* p, const mgrit_fc_layers_t* fc, const void* W, const float* b,
                                const float* U, const float* lamN, float* Lam, float* dW, float* db,
                                double* resnorm_hist, int32_t* iters_done,
                                void* workspace, size_t workspace_bytes, void* hip_stream);
int32_t mgrit_residual_norm_mixed(const mgrit_problem_t* p, const mgrit_fc_layers_t* fc, const void* W,
                                  const float* b, const float* u0, const float* U, double* norm_out,
                                  void* workspace, size_t workspace_bytes, void* hip_stream);

/* ---- The rest of a training step: opening and closing layers, loss, gradient clipping.  u^0 comes from an opening layer,
 * a closing layer turns u^N into logits, the loss and its gradient turn those into lambda^N (the closing layer's dX), and
 * all gradients -- the stack's from the adjoint solve and those of the end layers -- are clipped together.  These layers
 * are not square, so they are no part of a stack; every size is allowed.  As above: the caller owns every buffer, device
 * pointers are aligned to 16 bytes unless stated otherwise (so that a state inside U will do), work is enqueued on `hip_stream` of the current device, nothing
 * is allocated, and a call without host outputs is kernel launches only and may be recorded into a graph (the same rule of a
 * first call outside the capture).  Arrays are row-major without gaps; outputs may not overlap inputs or each other except
 * where it is said.  Two calls that may overlap in time need a workspace each.  Results do not depend on the run: no sum is formed in an
 * order that changes from one call to the next. */
enum { MGRIT_ACT_IDENTITY = 2 };                           /* with MGRIT_ACT_TANH and _RELU; end layers only */

/* An affine layer with activation, residual and step:
 *   z = X W^T + b,  Y = R + scale act(z),  D = scale act'(z)      X [M][K], W [F][K], b [F], R, Y, D [M][F]
 * (ReLU'(0) = 0; a NaN stays a NaN in every activation).  Types: X (and dX) xtype, W wtype, and R, Y, D, dY ytype, each MGRIT_FP32 or
 * MGRIT_BF16; b, dW and db are float.  Operands enter the products as they are stored, sums are float: bf16 operands are
 * not rounded again and float ones not rounded at all (unlike the solver's, whose MGRIT_BF16 rounds the state).  Some products
 * take an operand in several parts whose sum it is, every bit of it down to the smallest normal float; where operands hold infinities, an entry that the formula makes infinite
 * may come out as NaN then.  Entries that no infinity or NaN takes part in are not touched by it. */
typedef struct mgrit_affine {
  int32_t M;           /* rows (samples), >= 0; with 0 rows only dW and db are written, as zero                  */
  int32_t K, F;        /* inputs and outputs per row, >= 1                                                       */
  int32_t act;         /* MGRIT_ACT_TANH, _RELU or _IDENTITY                                                     */
  int32_t xtype, wtype, ytype;
  float   scale;       /* finite                                                                                 */
} mgrit_affine_t;

/* Workspace of the forward and of the backward pass; 0 if the layer is invalid or needs none (then the workspace
 * pointer may be NULL; mgrit_affine_forward tells an invalid layer by its code).  Host only. */
size_t  mgrit_affine_workspace_bytes(const mgrit_affine_t* p);
size_t  mgrit_affine_backward_workspace_bytes(const mgrit_affine_t* p);

/*   X, W      device, read only
 *   b         device float or NULL (no bias)         R   device or NULL (no residual); may be Y itself
 *   Y         device, out                            D   device, out, or NULL: the factors that the backward pass takes
 * Errors: MGRIT_ERR_POINTER, _PROBLEM, _WORKSPACE, _HIP; MGRIT_ERR_UNSUPPORTED if an array has more than 2^38 elements. */
int32_t mgrit_affine_forward(const mgrit_affine_t* p, const void* X, const void* W, const float* b, const void* R,
                             void* Y, void* D, void* workspace, size_t workspace_bytes, void* hip_stream);

/* G = dY * D (entry by entry; D NULL: G = scale dY, for the identity only),
 *   dX = G W,  dW = G^T X,  db = sum over the rows of G            (the residual's gradient is dY itself)
 *   dX, dW, db  device, overwritten; each may be NULL if it is not wanted.  X is read for dW only and may be NULL without
 *               it; likewise W for dX.
 * G is not rounded: a product of two bf16 values enters the sums as it is. */
int32_t mgrit_affine_backward(const mgrit_affine_t* p, const void* X, const void* W, const void* D, const void* dY,
                              void* dX, float* dW, float* db, void* workspace, size_t workspace_bytes, void* hip_stream);

/* Softmax cross-entropy of logits x [B][V] (type dtype) against labels [B]:
 *   row r:  l_r = log(sum_v exp(x_rv)) - x_r,label(r),   loss = scale * sum of l_r, or with MGRIT_LOSS_MEAN of the mean over the
 *   counted rows;   grad_rv = d loss / d x_rv
 * A row with a negative label does not count: l_r = 0 and a zero gradient, whatever its logits hold.  If no row counts the loss
 * is 0.  Logits of minus infinity take part as probability zero; a row whose label is such a class has l_r = +infinity and the
 * gradient of the formula, a row that holds a NaN, +infinity or nothing but minus infinity has NaN for both.  A label of V or
 * more gives its row NaN, too, and reads nothing out of range. */
enum { MGRIT_LOSS_SUM = 0, MGRIT_LOSS_MEAN = 1 };
typedef struct mgrit_loss {
  int32_t B, V;        /* rows >= 0, classes >= 1                                                                */
  int32_t dtype;       /* of logits and grad: MGRIT_FP32 or MGRIT_BF16                                           */
  int32_t reduction;   /* MGRIT_LOSS_SUM or MGRIT_LOSS_MEAN                                                      */
  float   scale;       /* finite                                                                                 */
} mgrit_loss_t;

size_t  mgrit_cross_entropy_workspace_bytes(const mgrit_loss_t* p);
/*   logits    device, read only; int64 labels device        loss   device float [1] or NULL
 *   row_loss  device float [B] (l_r, not scaled) or NULL    grad   device [B][V] or NULL; may be the logits themselves */
int32_t mgrit_cross_entropy(const mgrit_loss_t* p, const void* logits, const int64_t* labels, float* loss,
                            float* row_loss, void* grad, void* workspace, size_t workspace_bytes, void* hip_stream);

/* Clipping of many gradients to one global norm:
 *   norm = sqrt(sum over all tensors and entries of src^2),  dst = c src with c = norm > max_norm ? max_norm / norm : 1
 * The squares are summed in double; c is rounded to float once and multiplies in float.  If the norm is not finite, c is 1,
 * so that in-place gradients stay as they were.
 *   tensors   host array of n descriptors, n >= 0; src and dst need the alignment of their element only.  dst may be src
 *             (clipped in place), or NULL: the tensor counts and is not written.  Apart from that no dst may overlap any src.
 *   max_norm  >= 0; infinity for the norm alone
 *   norm      device float [1], or NULL (4-byte aligned)
 *   norm_host host double or NULL: synchronises the stream, and MGRIT_ERR_NONFINITE tells a norm that is not finite */
typedef struct mgrit_tensor {
  const void* src;
  void*       dst;
  int64_t     count;   /* >= 0; with 0 the pointers are not looked at                                            */
  int32_t     dtype;   /* MGRIT_FP32 or MGRIT_BF16                                                               */
} mgrit_tensor_t;

size_t  mgrit_clip_workspace_bytes(const mgrit_tensor_t* tensors, int32_t n);
int32_t mgrit_clip_gradients(const mgrit_tensor_t* tensors, int32_t n, float max_norm, float* norm, double* norm_host,
                             void* workspace, size_t workspace_bytes, void* hip_stream);

/* ---- Values in few bits.  A packed array holds rows in blocks of 32 entries, each block with a power of two as its scale: the smallest
 * 2^s, s >= -127, for which no entry of the block exceeds the format's largest value times 2^s.  Entries are divided by it (exactly) and rounded
 * to nearest, ties to even; nothing is cut off.  A block that holds an infinity or a NaN is NaN throughout.
 *   MGRIT_MX8   sign, 4 exponent and 3 mantissa bits (bias 7), largest value 448, smallest 2^-9; a byte each
 *   MGRIT_MX4   sign, 2 exponent and 1 mantissa bits (bias 1): 0 .5 1 1.5 2 3 4 6; two in a byte, the first in its low half
 * Layout, with C = cols rounded up to a multiple of 256: codes [rows][C] (MX4: C / 2 bytes a row), and from the next multiple of 256 bytes on
 * scales [C / 256][rows][8], a byte s + 127 each (255: NaN), the eight in the order of blocks 0 2 4 6 1 3 5 7.  Entries
 * behind the last column are zero.  Scales lie so that the matrix instructions' lanes find theirs side by side. */
enum { MGRIT_MX8 = 8, MGRIT_MX4 = 4 };
typedef struct mgrit_packed {
  int32_t rows, cols;  /* rows >= 0, cols >= 1                                                                   */
  int32_t format;      /* MGRIT_MX8 or MGRIT_MX4                                                                 */
  int32_t dtype;       /* of the unpacked values: MGRIT_FP32 or MGRIT_BF16                                       */
} mgrit_packed_t;

/* Bytes of the packed array, a multiple of 256; 0 if it is invalid or has no rows. */
size_t  mgrit_packed_bytes(const mgrit_packed_t* p);
/* packed (device, aligned to 256 bytes) <- X [rows][cols], and back (to bf16 a value below 2^-126 in magnitude is rounded, and
 * a largest float that was rounded up to 2^128 is an infinity; everything else is exact).
 * Errors: MGRIT_ERR_POINTER, _PROBLEM, _HIP; MGRIT_ERR_UNSUPPORTED if rows * (cols rounded up to a multiple of 256) exceeds 2^38. */
int32_t mgrit_pack(const mgrit_packed_t* p, const void* X, void* packed, void* hip_stream);
int32_t mgrit_unpack(const mgrit_packed_t* p, const void* packed, void* X, void* hip_stream);

/* The affine layer of mgrit_affine_forward with packed weights:
 *   z = X~ W~^T + b,  Y = R + scale act(z),  D = scale act'(z)
 * W~ the values of W [F][K] packed as MGRIT_MX4.  X [M][K] is of type xtype; X~ are with xformat = MGRIT_BF16 its values rounded to bf16 (of bf16
 * arrays: as they are), with MGRIT_MX4 the values that packing it would give (then the products are those of 4-bit values, and exact).
 * Sums are float.  R, Y, D ytype, b float, as there. */
typedef struct mgrit_affine_packed {
  int32_t M;           /* rows (samples), >= 0                                                                   */
  int32_t K, F;        /* inputs and outputs per row, >= 1                                                       */
  int32_t act;         /* MGRIT_ACT_TANH, _RELU or _IDENTITY                                                     */
  int32_t xtype, xformat, ytype;
  float   scale;       /* finite                                                                                 */
} mgrit_affine_packed_t;

size_t  mgrit_affine_packed_workspace_bytes(const mgrit_affine_packed_t* p);
/*   W   device, packed, read only (256-byte aligned)      X, b, R, Y, D as in mgrit_affine_forward
 * Errors as there, and MGRIT_ERR_UNSUPPORTED if K exceeds 2^22. */
int32_t mgrit_affine_packed_forward(const mgrit_affine_packed_t* p, const void* X, const void* W, const float* b, const void* R,
                                    void* Y, void* D, void* workspace, size_t workspace_bytes, void* hip_stream);

/* The backward pass of an affine layer from activations that were kept in 8 bits: mgrit_affine_backward with X [M][K] and D [M][F]
 * packed as MGRIT_MX8, p->xtype the type of dX alone.  Between the passes a row takes 264 bytes for every 256 columns that it begins: over many columns a
 * quarter of a float state's memory, half of a bf16 one's; up to 66 columns (bf16: 132, and 257 to 264) no less than the state itself.
 *   G = dY * D~ (D NULL: G = scale dY, for the identity only),  dX = G W,  dW = G^T X~,  db = sum over the rows of G
 * X~ and D~ enter as they are packed, but that values of X~ below 2^-126 are rounded to bf16. */
size_t  mgrit_affine_kept_workspace_bytes(const mgrit_affine_t* p);
int32_t mgrit_affine_kept_backward(const mgrit_affine_t* p, const void* X, const void* W, const void* D, const void* dY,
                                   void* dX, float* dW, float* db, void* workspace, size_t workspace_bytes, void* hip_stream);

/* ---- The norms after and before a block, with its gate and residual step: from the stream r and a block's result f
 *   n = norm(f) w_post,   S = r + scale gate n,   Y = norm(S) w_pre                 f, r, S, Y [M][q], w_post, w_pre [q]
 * S is the stream behind the block, Y what the next block takes.  norm(x) = x / sqrt(mean(x^2) + eps), or with MGRIT_NORM_LAYER the same of
 * x less its mean, over the q features of a row.  w_post NULL: n = f; w_pre NULL: no Y.  The gate is absent, one value a feature
 * (float [q]) or one an entry ([M][q], type ftype).  r, S (and dS, dr) are of type stype, f, Y (and df, dY) of type ftype, weights and their
 * gradients float.  Y comes from S before that is rounded to its type.  Entries that are all the same have no deviation from their mean, whatever its
 * rounding; with eps = 0 a row without deviation gives NaN.  A deviation between 2^-126 and 2^126 is a float's, also where its square is none. */
enum { MGRIT_NORM_ROOT = 0, MGRIT_NORM_LAYER = 1 };
enum { MGRIT_GATE_NONE = 0, MGRIT_GATE_FEATURE = 1, MGRIT_GATE_ENTRY = 2 };
typedef struct mgrit_block_norm {
  int32_t M, q;        /* rows >= 0, features >= 1                                                               */
  int32_t kind;        /* MGRIT_NORM_ROOT or MGRIT_NORM_LAYER                                                    */
  int32_t gate;        /* MGRIT_GATE_NONE, _FEATURE or _ENTRY                                                    */
  int32_t stype, ftype;
  float   eps;         /* >= 0, finite                                                                           */
  float   scale;       /* finite                                                                                 */
} mgrit_block_norm_t;

/*   S    device, out; may be r                    Y    device, out; NULL exactly if w_pre is.  May be f
 * Errors: MGRIT_ERR_POINTER, _PROBLEM, _HIP; MGRIT_ERR_UNSUPPORTED if M * q exceeds 2^38. */
int32_t mgrit_block_norm_forward(const mgrit_block_norm_t* p, const void* f, const void* r, const void* gate, const float* w_post,
                                 const float* w_pre, void* S, void* Y, void* hip_stream);
/* Backwards, from f, gate, S and the gradients by S (from what else uses the stream; NULL: none) and by Y (NULL exactly if w_pre is):
 *   dr = dS + the gradient by S through Y,   df, dgate (type and shape of the gate), dw_post, dw_pre float [q]
 * dr is the whole gradient by S, which is that by r.  Each output may be NULL if it is not wanted.  dr may be dS, df may be dY or f.
 * Without rows the gradients of vectors are written as zero. */
size_t  mgrit_block_norm_workspace_bytes(const mgrit_block_norm_t* p);
int32_t mgrit_block_norm_backward(const mgrit_block_norm_t* p, const void* f, const void* S, const void* gate, const float* w_post,
                                  const float* w_pre, const void* dS, const void* dY, void* df, void* dr, void* dgate, float* dw_post,
                                  float* dw_pre, void* workspace, size_t workspace_bytes, void* hip_stream);

/* ---- Answers: one class for each row of logits x [B][V] from a given random number u in [0, 1).  With the row's temperature t the
 * weights are w_v = exp((x_v - max x) / t).  The classes in falling order of their logits, equal ones lowest index first, are narrowed to
 *   top_k   the first k (k <= 0 or k >= V: all)
 *   top_p   of these the first ones up to where their weights reach p times the sum of all of these (p >= 1: all; p <= 0: the first)
 *   min_p   those with w_v >= min_p (<= 0: all; above 1: as 1)
 * all three; index <- the first class v in the order of indices for which the kept weights up to and with v sum to more than u times all
 * kept weights, logprob <- log(w_v / the sum of the kept weights).  t = 0: the largest logit, lowest index first, logprob 0.
 * Logits of minus infinity have weight zero.  A row that holds a NaN, +infinity or nothing but minus infinity, or whose t is negative, infinite or NaN, whose u is
 * not in [0, 1), or whose top_p or min_p is NaN, gives index -1 and logprob NaN.
 * Weights are computed to 1e-13 and summed as integers in units of 2^-min(50, 62 - log2 V): the same class every time, however the sums are formed. */
typedef struct mgrit_sample {
  int32_t B, V;        /* rows >= 0, classes >= 1                                                                */
  int32_t dtype;       /* of the logits: MGRIT_FP32 or MGRIT_BF16                                                */
} mgrit_sample_t;

/* 0: none is needed in this build (then the workspace pointer may be NULL) */
size_t  mgrit_sample_workspace_bytes(const mgrit_sample_t* p);
/*   logits  device, read only                     u          device float [B]
 *   temperature, top_p, min_p  device float [B], top_k  device int32 [B], each NULL if no row asks for it (t = 1)
 *   index   device int64 [B], out                 logprob    device float [B] or NULL
 * Errors: MGRIT_ERR_POINTER, _PROBLEM, _WORKSPACE, _HIP; MGRIT_ERR_UNSUPPORTED if B * V exceeds 2^38. */
int32_t mgrit_sample(const mgrit_sample_t* p, const void* logits, const float* u, const float* temperature, const int32_t* top_k, const float* top_p,
                     const float* min_p, int64_t* index, float* logprob, void* workspace, size_t workspace_bytes, void* hip_stream);

/* Diagnostic launch tracing, off by default and the one piece of state the library keeps: between
 * mgrit_trace_begin() and mgrit_trace_end() every layer-step and gradient launch is bracketed by a
 * pair of HIP events on its stream.  mgrit_trace_end synchronises on the last event and returns,
 * per kernel class (MGRIT_TRACE_*; CONV_SWEEP_F32 counts sweeps of both types), the summed elapsed milliseconds,
 * the number of launches, the number of layer steps (groups) they processed -- a fused launch: the layer steps of the
 * one-launch-per-step schedule that it stands for -- and (bytes, may be NULL) their algorithmic bytes --
 * per layer step the layer's weights and bias, the input state, every fused epilogue operand, the
 * act' factor and the output, each moved once; arrays of n_classes entries, host.  Not thread
 * safe; meant for the benchmark's roofline figures (Sec. IV-B reports such a timeline). */
enum {
  MGRIT_TRACE_DENSE_F32_T64 = 0, MGRIT_TRACE_DENSE_F32_T128, MGRIT_TRACE_DENSE_BF16_T64,
  MGRIT_TRACE_DENSE_BF16_T128, MGRIT_TRACE_CONV_F32, MGRIT_TRACE_CONV_BF16, MGRIT_TRACE_GRAD,
  MGRIT_TRACE_SWEEP_F32, MGRIT_TRACE_SWEEP_BF16, MGRIT_TRACE_DENSE_F32_KSPLIT8,
  MGRIT_TRACE_DENSE_F32_KSPLIT, MGRIT_TRACE_DENSE_BF16_KSPLIT, MGRIT_TRACE_DENSE_BF16_KSPLIT8,
  MGRIT_TRACE_CONV_SWEEP_F32, MGRIT_TRACE_NCLASS
};
void    mgrit_trace_begin(void);
int32_t mgrit_trace_end(double* ms, int64_t* launches, int64_t* units, double* bytes, int32_t n_classes);

#ifdef __cplusplus
}
#endif
#endif /* MGRIT_H */
