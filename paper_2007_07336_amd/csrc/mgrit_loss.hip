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

template <int TH> __device__ __forceinline__ Running join_threads(Running r, Running* sh) {
#pragma unroll
  for (int d = 32; d; d >>= 1) r = join(r, Running{__shfl_xor(r.m, d), __shfl_xor(r.s, d)});
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = r;
  __syncthreads();
  r = sh[0];
#pragma unroll
  for (int w = 1; w < TH / 64; ++w) r = join(r, sh[w]);
  return r;
}
// The vector as it was loaded: without this the compiler keeps its widened values, twice the registers, from one use to the next
template <typename T> __device__ __forceinline__ void keep_packed(Vec<T>& a) {
  typedef unsigned u4 __attribute__((ext_vector_type(4)));
  u4 u = __builtin_bit_cast(u4, a);
  asm volatile("" : "+v"(u));
  a = __builtin_bit_cast(Vec<T>, u);
}
// A row's loss.  The maximum less the label's logit first: the sum's logarithm, at most log V, added to the maximum alone would be rounded to
// that one's size (logits near 1000: 6e-5).
__device__ __forceinline__ float loss_of(Running r, float asked) { return (r.m - asked) + __builtin_amdgcn_logf(r.s) * LN2; }
// What the row's results are made of: f times exp(x - m) is the gradient apart from the label's
struct Row {
  float m, s, w, f;
  __device__ __forceinline__ float gradient(float x, bool label) const {
    const float p = exp_below(x, m);
    return label ? (p / s - 1.0f) * w : p * f;
  }
};

// One row per workgroup of TH threads.  NV > 0: the row's whole 16-byte vectors fit NV registers of each thread, and the row is
// read once.  NV = 0: it is read twice.  rows <- l_r, grad <- gradient; `counted`: the number of rows that scale is divided by.
// Bound by memory: 4096 rows of 50021 bf16, 0.8 GB in and out, 164 us, 5.0 TB/s as a large copy (183 where the same tensors are taken again
// at once, and 197 there with rows that are read twice).
template <typename T, int TH, int NV>
__global__ __launch_bounds__(TH) void loss_rows_kernel(const T* logits, const int64_t* labels, float* rows, T* grad, int V, float scale, const int* counted) {
  constexpr int N = Vec<T>::N;
  __shared__ Running sh[TH / 64];
  const int t = threadIdx.x;
  const long long row = blockIdx.x;
  const int64_t label = labels[row];
  const T* x = logits + row * V;
  T* g = grad ? grad + row * V : nullptr;
  if (label < 0) {
    if (rows && t == 0) rows[row] = 0.0f;
    if (g)
      for (long long v = t; v < V; v += TH) g[v] = T(0.0f);             // (V + TH may pass 31 bits)
    return;
  }
  // entries before the first whole vector, whole vectors, entries behind
  const int off = (int)((row * V) % N), head = off ? (N - off < V ? N - off : V) : 0, nv = (V - head) / N, tail = head + nv * N;
  const bool good = label < V;
  const float asked = good ? value(x[label]) : 0.0f;                     // (before the gradient may take the logits' place)
  const float edge[2] = {t < head ? value(x[t]) : -INFINITY, t < V - tail ? value(x[tail + t]) : -INFINITY};
  Running r = {-INFINITY, 0.0f};
  Vec<T> a[NV ? NV : 1];
  if constexpr (NV > 0) {
    // (loads are not predicated, or each would be waited for: threads behind the last vector read it once more)
#pragma unroll
    for (int i = 0; i < NV; ++i) a[i] = *reinterpret_cast<const Vec<T>*>(__builtin_assume_aligned(x + head + (t + i * TH < nv ? t + i * TH : nv - 1) * N, 16));
    float m = fmaxf(edge[0], edge[1]), s = 0.0f;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < N; ++j) m = fmaxf(m, value(a[i].v[j]));
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      keep_packed(a[i]);
      float q = 0.0f;
#pragma unroll
      for (int j = 0; j < N; ++j) { const float v = value(a[i].v[j]); q += v == -INFINITY ? 0.0f : exp_below(v, m); }
      s += t + i * TH < nv ? q : 0.0f;
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) s += edge[j] == -INFINITY ? 0.0f : exp_below(edge[j], m);
    r = Running{m, s};
  } else {
    for (int v = t; v < nv; v += TH) {
      const Vec<T> b = *reinterpret_cast<const Vec<T>*>(__builtin_assume_aligned(x + head + v * N, 16));
      float f[N];
#pragma unroll
      for (int j = 0; j < N; ++j) f[j] = value(b.v[j]);
      take(r, f);
    }
    take(r, edge);
  }
  r = join_threads<TH>(r, sh);
  if (r.s == 0.0f || !good) r.s = NAN;
  if (rows && t == 0) rows[row] = good ? loss_of(r, asked) : NAN;
  if (!g) return;
  const float w = counted ? scale / (float)*counted : scale;
  const Row o = {r.m, r.s, w, w / r.s};
  auto put = [&](Vec<T> b, int v) {
#pragma unroll
    for (int j = 0; j < N; ++j) b.v[j] = static_cast<T>(o.gradient(value(b.v[j]), head + v * N + j == label));
    *reinterpret_cast<Vec<T>*>(__builtin_assume_aligned(g + head + v * N, 16)) = b;
  };
  if constexpr (NV > 0) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      keep_packed(a[i]);
      if (t + i * TH < nv) put(a[i], t + i * TH);
    }
  } else {
    for (int v = t; v < nv; v += TH) put(*reinterpret_cast<const Vec<T>*>(__builtin_assume_aligned(x + head + v * N, 16)), v);
  }
  if (t < head) g[t] = static_cast<T>(o.gradient(edge[0], t == label));
  if (t < V - tail) g[tail + t] = static_cast<T>(o.gradient(edge[1], tail + t == label));
}

// Short rows, V <= 16 L: L lanes of a wavefront per row, 16 entries each at most.  Alone (one workgroup of 1024 threads, few rows): it
// counts the rows and adds up the losses as well, so that a small loss is a single launch.
template <typename T, int L>
__global__ __launch_bounds__(1024) void loss_short_kernel(const T* logits, const int64_t* labels, float* rows, T* grad, int B, int V, float scale, int mean,
                                                         const int* counted, int alone, float* loss) {
  __shared__ double part[16];
  __shared__ int count[16];
  const int t = threadIdx.x, l = t % L;
  const long long step = (long long)gridDim.x * (blockDim.x / L);
  long long row = blockIdx.x * (long long)(blockDim.x / L) + t / L;
  int64_t label = -1;
  float v[16];
  auto load = [&]() {
    label = labels[row];
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = l + i * L < V ? value(logits[row * V + l + i * L]) : -INFINITY;
  };
  if (row < B) load();                           // (the first row is on its way while rows are counted)
  float w = scale;
  if (mean && alone) {
    int n = 0;
    for (int r = t; r < B; r += blockDim.x) n += labels[r] >= 0;
#pragma unroll
    for (int d = 32; d; d >>= 1) n += __shfl_xor(n, d);
    if ((t & 63) == 0) count[t >> 6] = n;
    __syncthreads();
    n = 0;
    for (int i = 0; i < (int)blockDim.x / 64; ++i) n += count[i];
    w = scale / (float)(n > 0 ? n : 1);
  } else if (mean) {
    w = scale / (float)*counted;
  }
  double total = 0.0;
  for (; row < B; row += step) {
    const T* x = logits + row * V;
    Running r = {-INFINITY, 0.0f};
#pragma unroll
    for (int i = 0; i < 16; ++i) r.m = fmaxf(r.m, v[i]);
    const bool good = label < V;
    const float asked = label >= 0 && good ? value(x[label]) : 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) r.s += v[i] == -INFINITY ? 0.0f : exp_below(v[i], r.m);
#pragma unroll
    for (int d = L / 2; d; d >>= 1) r = join(r, Running{__shfl_xor(r.m, d), __shfl_xor(r.s, d)});
    if (r.s == 0.0f || !good) r.s = NAN;
    const float lr = label < 0 ? 0.0f : good ? loss_of(r, asked) : NAN;
    if (rows && l == 0) rows[row] = lr;
    total += l == 0 ? (double)lr : 0.0;
    if (grad) {
      const Row o = {r.m, r.s, w, w / r.s};
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (l + i * L < V) grad[row * V + l + i * L] = static_cast<T>(label < 0 ? 0.0f : o.gradient(v[i], l + i * L == label));
    }
    if (row + step < B) {
      row += step;
      load();
      row -= step;
    }
  }
  if (!alone || !loss) return;
#pragma unroll
  for (int d = 32; d; d >>= 1) total += __shfl_xor(total, d);
  if ((t & 63) == 0) part[t >> 6] = total;
  __syncthreads();
  if (t) return;
  total = 0.0;
  for (int i = 0; i < (int)blockDim.x / 64; ++i) total += part[i];
  *loss = (float)(total * (double)w);
}

// Number of rows that count
__global__ __launch_bounds__(1024) void count_rows_kernel(const int64_t* labels, int B, int* counted) {
  __shared__ int part[16];
  int n = 0;
  for (long long r = threadIdx.x; r < B; r += 1024) n += labels[r] >= 0;
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
  for (long long r = threadIdx.x; r < B; r += 1024) s += (double)rows[r];
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

// Short rows: V <= 1024 (longer ones are worth a workgroup)
template <typename T>
hipError_t launch_short(const LossArgs& a, float* rows, const int* counted, bool alone, hipStream_t s) {
  const T* x = static_cast<const T*>(a.logits);
  T* g = static_cast<T*>(a.grad);
  const int lanes = a.V <= 16 ? 1 : a.V <= 64 ? 4 : a.V <= 256 ? 16 : 64, threads = alone ? 1024 : 256;
  const long long blocks = (a.B + threads / lanes - 1LL) / (threads / lanes);
  const dim3 grid((unsigned)(alone ? 1 : blocks < 65536 ? blocks : 65536));
#define SHORT_ROWS(L) hipLaunchKernelGGL((loss_short_kernel<T, L>), grid, dim3(threads), 0, s, x, a.labels, rows, g, a.B, a.V, a.scale, a.mean, counted, alone, a.loss)
  if (lanes == 1) SHORT_ROWS(1);
  else if (lanes == 4) SHORT_ROWS(4);
  else if (lanes == 16) SHORT_ROWS(16);
  else SHORT_ROWS(64);
#undef SHORT_ROWS
  return hipGetLastError();
}
template <typename T>
hipError_t launch_rows(const LossArgs& a, float* rows, const int* counted, hipStream_t s) {
  const T* x = static_cast<const T*>(a.logits);
  T* g = static_cast<T*>(a.grad);
  const long long vectors = a.V / Vec<T>::N;
  // a launch has fewer than 2^32 threads; 2^21 rows begin a multiple of 16 bytes further, as the kernel expects of its arrays
  for (long long r0 = 0; r0 < a.B; r0 += 1LL << 21) {
    const unsigned n = (unsigned)(a.B - r0 < 1LL << 21 ? a.B - r0 : 1LL << 21);
    const T* xr = x + r0 * a.V;
    T* gr = g ? g + r0 * a.V : nullptr;
    float* rr = rows ? rows + r0 : nullptr;
#define LONG_ROWS(TH, NV) hipLaunchKernelGGL((loss_rows_kernel<T, TH, NV>), dim3(n), dim3(TH), 0, s, xr, a.labels + r0, rr, gr, a.V, a.scale, counted)
    if (vectors <= 256) LONG_ROWS(256, 1);
    else if (vectors <= 512) LONG_ROWS(256, 2);
    else if (vectors <= 1024) LONG_ROWS(256, 4);
    else if (vectors <= 2048) LONG_ROWS(512, 4);
    else if (vectors <= 4096) LONG_ROWS(1024, 4);
    else if (vectors <= 8192) LONG_ROWS(1024, 8);
    else LONG_ROWS(1024, 0);
#undef LONG_ROWS
  }
  return hipGetLastError();
}

}  // namespace

size_t loss_workspace(const LossArgs& a) { return 256 + (size_t)a.B * sizeof(float); }

hipError_t launch_loss(const LossArgs& a, void* ws, hipStream_t s) {
  // one launch for up to 32 entries of each of its threads
  const bool alone = a.V <= 1024 && (long long)a.B * a.V <= 32768 && a.B <= 4096;
  if (alone) return a.dtype ? launch_short<__bf16>(a, a.rows, nullptr, true, s) : launch_short<float>(a, a.rows, nullptr, true, s);
  int* counted = a.mean ? static_cast<int*>(ws) : nullptr;
  float* rows = a.rows ? a.rows : a.loss ? reinterpret_cast<float*>(static_cast<char*>(ws) + 256) : nullptr;
  if (counted && (a.loss || a.grad)) hipLaunchKernelGGL(count_rows_kernel, dim3(1), dim3(1024), 0, s, a.labels, a.B, counted);
  hipError_t e = hipSuccess;
  if (a.B > 0 && (rows || a.grad)) {            // (a launch of no workgroups is an error)
    if (a.V <= 1024) e = a.dtype ? launch_short<__bf16>(a, rows, counted, false, s) : launch_short<float>(a, rows, counted, false, s);
    else e = a.dtype ? launch_rows<__bf16>(a, rows, counted, s) : launch_rows<float>(a, rows, counted, s);
  }
  if (e == hipSuccess && a.loss) hipLaunchKernelGGL(sum_rows_kernel, dim3(1), dim3(1024), 0, s, rows, a.B, a.scale, counted, a.loss);
  return e != hipSuccess ? e : hipGetLastError();
}

}  // namespace mgrit
