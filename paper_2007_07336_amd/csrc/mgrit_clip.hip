// Global norm of many tensors, and their scaling to at most a given norm.
#include "mgrit_device.h"
#include "mgrit_ops.h"

namespace mgrit {

namespace {

// Two passes, each bound by memory: the sum of squares (4.3 GB in 742 us, 5.8 TB/s) and the scaling (read and written, 1738 us, 5.0 TB/s);
// the second has to wait for the whole of the first.  Squares are summed in double, which costs nothing here and cannot overflow.
constexpr int TH = 256, GRID = 2048;
constexpr long long CHUNK = 4096;               // entries: a workgroup takes consecutive chunks, none across two tensors

struct Entry {
  const void* src;
  void* dst;
  long long count, chunk0;                      // chunk0: chunks of the tensors before
  long long type;
};
// The list of tensors goes to the workspace by kernel arguments, which a captured graph keeps, as many at a time as 4 KB of them
// hold (600 tensors: 4 launches of 2 us).
struct Given { const void* src; void* dst; long long count; };         // count: twice the entries, and 1 for bf16
constexpr int PER = 168;
struct Givens { Given e[PER]; };
static_assert(sizeof(Givens) + 24 <= 4096, "kernel arguments");
struct Space { double norm; double partial[GRID]; Entry table[1]; };

__global__ __launch_bounds__(256) void clip_table_kernel(Givens in, Entry* out, int n, long long before) {
  __shared__ long long of_wave[4];
  const int t = threadIdx.x;
  const long long count = t < n ? in.e[t].count >> 1 : 0, mine = (count + CHUNK - 1) / CHUNK;
  long long sum = mine;                         // running sums
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const long long v = __shfl_up(sum, d);
    if ((t & 63) >= d) sum += v;
  }
  if ((t & 63) == 63) of_wave[t >> 6] = sum;
  __syncthreads();
  for (int w = 0; w < t >> 6; ++w) sum += of_wave[w];
  if (t < n) out[t] = Entry{in.e[t].src, in.e[t].dst, count, before + sum - mine, in.e[t].count & 1};
}

__device__ __forceinline__ float value(float v) { return v; }
__device__ __forceinline__ float value(__bf16 v) { return static_cast<float>(v); }
template <typename T> struct Vec { static constexpr int N = 16 / (int)sizeof(T); T v[N]; };
template <typename T> struct __attribute__((packed)) AnyVec { Vec<T> v; };       // at any address

// Calls run(entry, first, last) for this workgroup's share of every tensor
template <typename R>
__device__ __forceinline__ void for_share(const Entry* table, int n, long long chunks, R run) {
  long long c = chunks * blockIdx.x / gridDim.x;
  const long long c1 = chunks * (blockIdx.x + 1) / gridDim.x;
  if (c >= c1) return;
  int lo = 0, hi = n - 1;                       // the tensor that chunk c belongs to
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (table[mid].chunk0 <= c) lo = mid; else hi = mid - 1;
  }
  for (int t = lo; t < n && c < c1; ++t) {
    const Entry e = table[t];
    const long long of = c - e.chunk0, all = (e.count + CHUNK - 1) / CHUNK, take = all - of < c1 - c ? all - of : c1 - c;
    const long long first = of * CHUNK, last = first + take * CHUNK < e.count ? first + take * CHUNK : e.count;
    run(e, first, last);
    c += take;
  }
}

template <typename T>
__device__ __forceinline__ double square_sum(const T* p, long long first, long long last) {
  constexpr int N = Vec<T>::N;
  const long long nv = (last - first) / N;
  const T* q = p + first;
  double s = 0.0;
  for (long long v = threadIdx.x; v < nv; v += TH) {
    const Vec<T> a = reinterpret_cast<const AnyVec<T>*>(q + v * N)->v;
#pragma unroll
    for (int i = 0; i < N; ++i) { const double d = (double)value(a.v[i]); s += d * d; }
  }
  const long long at = nv * N + threadIdx.x;
  if (at < last - first) { const double d = (double)value(q[at]); s += d * d; }
  return s;
}

// Sum over the workgroup in a fixed order; thread 0 has it.
__device__ __forceinline__ double workgroup_sum(double s) {
  __shared__ double part[TH / 64];
#pragma unroll
  for (int d = 32; d; d >>= 1) s += __shfl_xor(s, d);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
  __syncthreads();
  s = 0.0;
#pragma unroll
  for (int w = 0; w < TH / 64; ++w) s += part[w];
  return s;
}

__global__ __launch_bounds__(TH) void clip_norm_kernel(const Entry* table, int n, long long chunks, double* partial) {
  double s = 0.0;
  for_share(table, n, chunks, [&](const Entry& e, long long first, long long last) {
    s += e.type ? square_sum(static_cast<const __bf16*>(e.src), first, last) : square_sum(static_cast<const float*>(e.src), first, last);
  });
  s = workgroup_sum(s);
  if (threadIdx.x == 0) partial[blockIdx.x] = s;
}

template <typename T>
__device__ __forceinline__ void scale_share(const T* src, T* dst, long long first, long long last, float c) {
  constexpr int N = Vec<T>::N;
  const long long nv = (last - first) / N;
  for (long long v = threadIdx.x; v < nv; v += TH) {
    Vec<T> a = reinterpret_cast<const AnyVec<T>*>(src + first + v * N)->v;
#pragma unroll
    for (int i = 0; i < N; ++i) a.v[i] = static_cast<T>(value(a.v[i]) * c);
    reinterpret_cast<AnyVec<T>*>(dst + first + v * N)->v = a;
  }
  const long long at = first + nv * N + threadIdx.x;
  if (at < last) dst[at] = static_cast<T>(value(src[at]) * c);
}

// Every workgroup adds the partial sums up for itself, in the same order, which costs less than a launch between the two.
__global__ __launch_bounds__(TH) void clip_scale_kernel(const Entry* table, int n, long long chunks, const double* partial, int parts, double* norm_out,
                                                       float* norm, float max_norm) {
  double s = 0.0;
  for (int i = threadIdx.x; i < parts; i += TH) s += partial[i];
  const double nrm = sqrt(workgroup_sum(s));
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    *norm_out = nrm;
    if (norm) *norm = (float)nrm;
  }
  const float c = nrm > (double)max_norm && nrm < INFINITY ? (float)((double)max_norm / nrm) : 1.0f;
  for_share(table, n, chunks, [&](const Entry& e, long long first, long long last) {
    if (!e.dst || (c == 1.0f && e.dst == e.src)) return;
    if (e.type) scale_share(static_cast<const __bf16*>(e.src), static_cast<__bf16*>(e.dst), first, last, c);
    else scale_share(static_cast<const float*>(e.src), static_cast<float*>(e.dst), first, last, c);
  });
}

}  // namespace

size_t clip_workspace(int filled) { return sizeof(Space) + (size_t)filled * sizeof(Entry); }

hipError_t launch_clip(int n, const mgrit_tensor_t* t, float max_norm, float* norm, void* ws, const double** norm_dev, hipStream_t s) {
  Space* sp = static_cast<Space*>(ws);
  long long chunks = 0;
  bool any = false;
  int filled = 0;                               // entries of the table
  for (int i = 0; i < n;) {
    Givens in = {};
    int k = 0;
    const long long before = chunks;
    for (; i < n && k < PER; ++i) {
      if (t[i].count == 0) continue;
      in.e[k++] = Given{t[i].src, t[i].dst, 2 * t[i].count + (t[i].dtype == MGRIT_BF16 ? 1 : 0)};
      chunks += (t[i].count + CHUNK - 1) / CHUNK;
      any = any || t[i].dst;
    }
    if (k > 0) hipLaunchKernelGGL(clip_table_kernel, dim3(1), dim3(256), 0, s, in, sp->table + filled, k, before);
    filled += k;
  }
  const int grid = chunks < GRID ? (int)chunks : GRID;
  if (grid > 0) hipLaunchKernelGGL(clip_norm_kernel, dim3((unsigned)grid), dim3(TH), 0, s, sp->table, filled, chunks, sp->partial);
  hipLaunchKernelGGL(clip_scale_kernel, dim3((unsigned)(any ? grid : 1)), dim3(TH), 0, s, sp->table, any ? filled : 0, any ? chunks : 0, sp->partial, grid, &sp->norm,
                     norm, max_norm);
  *norm_dev = &sp->norm;
  return hipGetLastError();
}

}  // namespace mgrit
