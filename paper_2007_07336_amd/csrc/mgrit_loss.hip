// Softmax cross-entropy of rows of logits, and its gradient.
#include "mgrit_device.h"
#include "mgrit_ops.h"

namespace mgrit {

namespace {

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

template <typename T> struct Vec { static constexpr int N = 16 / (int)sizeof(T); T v[N]; };
__device__ __forceinline__ float value(float v) { return v; }
__device__ __forceinline__ float value(__bf16 v) { return static_cast<float>(v); }
// exp(x - m); with x = m = -infinity a NaN, as everything that has no softmax
__device__ __forceinline__ float exp_below(float x, float m) { return __builtin_amdgcn_exp2f((x - m) * LOG2E); }

// Running maximum m and sum s of exp(x - m).  s = 0 means that only minus infinity has come so far; a NaN or plus infinity
// makes s a NaN for good.
struct Running { float m, s; };
__device__ __forceinline__ Running join(Running a, Running b) {
  const float m = fmaxf(a.m, b.m);
  return Running{m, (a.s == 0.0f ? 0.0f : a.s * exp_below(a.m, m)) + (b.s == 0.0f ? 0.0f : b.s * exp_below(b.m, m))};
}
template <int N> __device__ __forceinline__ void take(Running& r, const float (&x)[N]) {
  float m = r.m;
#pragma unroll
  for (int i = 0; i < N; ++i) m = fmaxf(m, x[i]);
  float s = r.s == 0.0f ? 0.0f : r.s * exp_below(r.m, m);
#pragma unroll
  for (int i = 0; i < N; ++i) s += x[i] == -INFINITY ? 0.0f : exp_below(x[i], m);
  r.m = m;
  r.s = s;
}

// TH threads per row; a wavefront (TH = 64) needs no barrier, so four rows share a workgroup then.
template <int TH> __device__ __forceinline__ Running join_threads(Running r, Running* sh) {
#pragma unroll
  for (int d = 32; d; d >>= 1) r = join(r, Running{__shfl_xor(r.m, d), __shfl_xor(r.s, d)});
  if (TH > 64) {
    if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = r;
    __syncthreads();
    r = sh[0];
#pragma unroll
    for (int w = 1; w < TH / 64; ++w) r = join(r, sh[w]);
  }
  return r;
}

// rows <- l_r, grad <- gradient.  weight: scale, divided by the number of counted rows if `counted` is given.
template <typename T, int TH>
__global__ __launch_bounds__(TH == 64 ? 256 : TH) void loss_rows_kernel(const T* logits, const int64_t* labels, float* rows, T* grad, int B, int V,
                                                                      float scale, const int* counted) {
  constexpr int N = Vec<T>::N;
  __shared__ Running sh[TH > 64 ? TH / 64 : 1];
  const int t = threadIdx.x % TH;
  const long long row = TH == 64 ? blockIdx.x * 4LL + (threadIdx.x >> 6) : blockIdx.x;
  if (row >= B) return;
  const int64_t label = labels[row];
  const T* x = logits + row * V;
  T* g = grad ? grad + row * V : nullptr;
  // entries before the first whole vector, whole vectors, entries behind
  const int off = (int)((row * V) % N), head = off ? (N - off < V ? N - off : V) : 0, nv = (V - head) / N, tail = head + nv * N;
  if (label < 0) {
    if (rows && t == 0) rows[row] = 0.0f;
    if (g)
      for (int v = t; v < V; v += TH) g[v] = T(0.0f);
    return;
  }
  Running r = {-INFINITY, 0.0f};
  for (int v = t; v < nv; v += TH) {
    const Vec<T> a = *reinterpret_cast<const Vec<T>*>(__builtin_assume_aligned(x + head + v * N, 16));
    float f[N];
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] = value(a.v[i]);
    take(r, f);
  }
  {
    float f[2] = {t < head ? value(x[t]) : -INFINITY, t < V - tail ? value(x[tail + t]) : -INFINITY};
    take(r, f);
  }
  r = join_threads<TH>(r, sh);
  const bool good = label < V;
  if (r.s == 0.0f || !good) r.s = NAN;
  // (before the gradient is written: it may lie where the logits are)
  if (rows && t == 0) rows[row] = good ? r.m + __builtin_amdgcn_logf(r.s) * LN2 - value(x[label]) : NAN;
  if (!g) return;
  if (TH > 64) __syncthreads();
  const float w = counted ? scale / (float)*counted : scale, f = w / r.s;
  for (int v = t; v < nv; v += TH) {
    Vec<T> a = *reinterpret_cast<const Vec<T>*>(__builtin_assume_aligned(x + head + v * N, 16));
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float p = exp_below(value(a.v[i]), r.m);
      a.v[i] = static_cast<T>(head + v * N + i == label ? (p / r.s - 1.0f) * w : p * f);
    }
    *reinterpret_cast<Vec<T>*>(__builtin_assume_aligned(g + head + v * N, 16)) = a;
  }
  for (int side = 0; side < 2; ++side) {
    const int v = side ? tail + t : t;
    if (side ? v < V : v < head) {
      const float p = exp_below(value(x[v]), r.m);
      g[v] = static_cast<T>(v == label ? (p / r.s - 1.0f) * w : p * f);
    }
  }
}

// Number of rows that count
__global__ __launch_bounds__(1024) void count_rows_kernel(const int64_t* labels, int B, int* counted) {
  __shared__ int part[16];
  int n = 0;
  for (int r = threadIdx.x; r < B; r += 1024) n += labels[r] >= 0;
#pragma unroll
  for (int d = 32; d; d >>= 1) n += __shfl_xor(n, d);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = n;
  __syncthreads();
  if (threadIdx.x == 0) {
    n = 0;
    for (int w = 0; w < 16; ++w) n += part[w];
    *counted = n > 0 ? n : 1;
  }
}
// loss = scale * sum of the rows' losses (/ counted), in double and in a fixed order
__global__ __launch_bounds__(1024) void sum_rows_kernel(const float* rows, int B, float scale, const int* counted, float* loss) {
  __shared__ double part[16];
  double s = 0.0;
  for (int r = threadIdx.x; r < B; r += 1024) s += (double)rows[r];
#pragma unroll
  for (int d = 32; d; d >>= 1) s += __shfl_xor(s, d);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    s = 0.0;
    for (int w = 0; w < 16; ++w) s += part[w];
    *loss = (float)((double)scale * s / (counted ? (double)*counted : 1.0));
  }
}

template <typename T>
hipError_t launch_rows(const LossArgs& a, float* rows, const int* counted, hipStream_t s) {
  const T* x = static_cast<const T*>(a.logits);
  T* g = static_cast<T*>(a.grad);
  if (a.V <= 1024)
    hipLaunchKernelGGL((loss_rows_kernel<T, 64>), dim3((unsigned)((a.B + 3LL) / 4)), dim3(256), 0, s, x, a.labels, rows, g, a.B, a.V, a.scale, counted);
  else if (a.V <= 16384)
    hipLaunchKernelGGL((loss_rows_kernel<T, 256>), dim3((unsigned)a.B), dim3(256), 0, s, x, a.labels, rows, g, a.B, a.V, a.scale, counted);
  else
    hipLaunchKernelGGL((loss_rows_kernel<T, 1024>), dim3((unsigned)a.B), dim3(1024), 0, s, x, a.labels, rows, g, a.B, a.V, a.scale, counted);
  return hipGetLastError();
}

}  // namespace

size_t loss_workspace(const LossArgs& a) { return 256 + (size_t)a.B * sizeof(float); }

hipError_t launch_loss(const LossArgs& a, void* ws, hipStream_t s) {
  int* counted = a.mean ? static_cast<int*>(ws) : nullptr;
  float* rows = a.rows ? a.rows : a.loss ? reinterpret_cast<float*>(static_cast<char*>(ws) + 256) : nullptr;
  if (counted && (a.loss || a.grad)) hipLaunchKernelGGL(count_rows_kernel, dim3(1), dim3(1024), 0, s, a.labels, a.B, counted);
  if (a.B > 0) {
    const hipError_t e = a.dtype ? launch_rows<__bf16>(a, rows, counted, s) : launch_rows<float>(a, rows, counted, s);
    if (e != hipSuccess) return e;
  }
  if (a.loss) hipLaunchKernelGGL(sum_rows_kernel, dim3(1), dim3(1024), 0, s, rows, a.B, a.scale, counted, a.loss);
  return hipGetLastError();
}

}  // namespace mgrit
