// One class for each row of logits, from a given random number: temperature, top-k, top-p, min-p.
#include "mgrit_device.h"
#include "mgrit_ops.h"

namespace mgrit {

namespace {

typedef unsigned long long u64;
typedef unsigned uint4u __attribute__((ext_vector_type(4), aligned(2)));    // 16-byte accesses of global memory need no alignment

template <typename T> struct Eight { static constexpr int N = 16 / (int)sizeof(T); };
template <typename T> __device__ __forceinline__ float entry(u32x4 v, int j);
template <> __device__ __forceinline__ float entry<float>(u32x4 v, int j) { return __uint_as_float(v[j]); }   // (__builtin_bit_cast of a vector's element takes its first one)
template <> __device__ __forceinline__ float entry<__bf16>(u32x4 v, int j) { return __builtin_bit_cast(float, j & 1 ? v[j / 2] & 0xffff0000u : v[j / 2] << 16); }

// Larger floats have larger keys, equal ones the same (both zeros are one value)
__device__ __forceinline__ unsigned key_of(float x) {
  const unsigned u = __builtin_bit_cast(unsigned, x + 0.0f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ u64 shuffle_up(u64 v, int d) {
  const unsigned lo = __shfl_up((unsigned)v, d), hi = __shfl_up((unsigned)(v >> 32), d);
  return (u64)hi << 32 | lo;
}
__device__ __forceinline__ u64 shuffle_xor(u64 v, int d) {
  const unsigned lo = __shfl_xor((unsigned)v, d), hi = __shfl_xor((unsigned)(v >> 32), d);
  return (u64)hi << 32 | lo;
}
__device__ __forceinline__ u64 shuffle(u64 v, int lane) {
  const unsigned lo = __shfl((unsigned)v, lane), hi = __shfl((unsigned)(v >> 32), lane);
  return (u64)hi << 32 | lo;
}
// Sum over the lanes up to and with this one
__device__ __forceinline__ u64 sum_up(u64 v, int lane) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const u64 o = shuffle_up(v, d);
    if (lane >= d) v += o;
  }
  return v;
}
__device__ __forceinline__ u64 sum_wave(u64 v) {
#pragma unroll
  for (int d = 32; d; d >>= 1) v += shuffle_xor(v, d);
  return v;
}

// 2^y, y <= 0, to 3e-13: y = n + f with |f| <= 1/2, and 2^f = exp(f log 2) as its series up to the tenth power (the next term is
// (log 2 / 2)^11 / 11! = 2e-13)
__device__ __forceinline__ double power2(double y, int shift) {
  const double n = __builtin_rint(y), f = (y - n) * 0.693147180559945309417;
  double p = 1.0 / 3628800.0;
  p = __builtin_fma(p, f, 1.0 / 362880.0);
  p = __builtin_fma(p, f, 1.0 / 40320.0);
  p = __builtin_fma(p, f, 1.0 / 5040.0);
  p = __builtin_fma(p, f, 1.0 / 720.0);
  p = __builtin_fma(p, f, 1.0 / 120.0);
  p = __builtin_fma(p, f, 1.0 / 24.0);
  p = __builtin_fma(p, f, 1.0 / 6.0);
  p = __builtin_fma(p, f, 0.5);
  p = __builtin_fma(p, f, 1.0);
  p = __builtin_fma(p, f, 1.0);
  return __builtin_ldexp(p, (int)n + shift);
}
// Weights exp((x - top) / t) in units of 2^-shift, rounded to whole ones, so that sums are exact and do not depend on their order
struct Weights {
  double top, rate;                  // rate = log2(e) / t
  int shift;
  double floor;                      // y of weights that are zero from there on
  __device__ __forceinline__ u64 of(float x) const {
    const double y = ((double)x - top) * rate;
    if (!(y > floor)) return 0;
    // (below 2^51 + 2^52: the whole units are the last bits)
    return __builtin_bit_cast(u64, power2(y, shift) + 4503599627370496.0) & 0xfffffffffffffull;
  }
};

// What a workgroup knows of its row, and its places in LDS
struct Shared {
  u64 bins[256];
  u64 part[16];
  u64 segment[256];                  // sums of the wavefronts' parts of the row, in order
  u64 base, value;
  unsigned bin, which;
  long long found;
  float top[16];
  unsigned bad[16];
};

// The row's vectors: in registers (NV > 0), or read again
template <typename T, int TH, int NV>
struct Row {
  static constexpr int N = Eight<T>::N, U = NV ? NV : 1;
  const T* x;
  long long V;
  int n;                             // vectors of a thread
  u32x4 held[NV ? NV : 1];
  __device__ __forceinline__ long long at(int i) const { return ((long long)i * TH + threadIdx.x) * N; }
  __device__ __forceinline__ u32x4 read(int i) const {
    const long long k = at(i);
    u32x4 v;
    if (k + N <= V) {
      v = *reinterpret_cast<const uint4u*>(x + k);
    } else {
      // minus infinity behind the last class
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if constexpr (sizeof(T) == 4) {
          v[j] = k + j < V ? reinterpret_cast<const unsigned*>(x)[k + j] : 0xff800000u;
        } else {
          const unsigned short* h = reinterpret_cast<const unsigned short*>(x);
          const unsigned lo = k + 2 * j < V ? h[k + 2 * j] : 0xff80u, hi = k + 2 * j + 1 < V ? h[k + 2 * j + 1] : 0xff80u;
          v[j] = lo | hi << 16;
        }
      }
    }
    return v;
  }
  __device__ __forceinline__ void init(const T* x_, long long V_) {
    x = x_; V = V_;
    n = NV ? NV : (int)((V + (long long)TH * N - 1) / ((long long)TH * N));
    if constexpr (NV > 0) {
#pragma unroll
      for (int i = 0; i < NV; ++i) held[i] = read(i);
    }
  }
  __device__ __forceinline__ u32x4 vec(int i) const { if constexpr (NV > 0) return held[i]; else return read(i); }
  // f(x) for each of this thread's entries
  template <typename F> __device__ __forceinline__ void each(F f) const {
#pragma unroll U
    for (int i = 0; i < n; ++i) {
      const u32x4 v = vec(i);
#pragma unroll
      for (int j = 0; j < N; ++j) f(entry<T>(v, j));
    }
  }
};

template <int TH> __device__ __forceinline__ u64 sum_threads(u64 v, Shared& sh) {
  v = sum_wave(v);
  if constexpr (TH > 64) {
    __syncthreads();                 // (whoever still reads an earlier sum)
    if ((threadIdx.x & 63) == 0) sh.part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0;
#pragma unroll
    for (int w = 0; w < TH / 64; ++w) v += sh.part[w];
  }
  return v;
}

// The first classes in falling order whose measures reach `limit`: those with larger keys than `key`, and of those with that key the first `ties`
struct Prefix { unsigned key; u64 ties; u64 sum; };              // sum: measure of all of it
// measure(x): of one class, the same for equal logits.  A descent over the key's bits, eight at a time from the top: bins of the measures of what agrees
// so far, and the bin in which the limit is reached.  Where rounding puts the limit beyond the sum of all, all are taken.
template <typename T, int TH, int NV, typename M>
__device__ __forceinline__ Prefix first_ones(const Row<T, TH, NV>& row, double limit, Shared& sh, M measure) {
  constexpr int LEVELS = sizeof(T) == 4 ? 4 : 2;
  unsigned key = 0;
  u64 base = 0, value = 0;
  for (int level = 0; level < LEVELS; ++level) {
    const int bits = 24 - 8 * level;
    __syncthreads();
    for (int b = threadIdx.x; b < 256; b += TH) sh.bins[b] = 0;
    __syncthreads();
    row.each([&](float x) {
      const unsigned k = key_of(x);
      if (level && (k >> (bits + 8)) != (key >> (bits + 8))) return;
      const u64 m = measure(x);
      if (m) atomicAdd(&sh.bins[k >> bits & 255u], m);
    });
    __syncthreads();
    if (threadIdx.x < 64) {
      // lane l: bins 255 - 4 l and the three below it
      const int lane = threadIdx.x, b0 = 255 - 4 * lane;
      u64 v[4], s = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) { v[i] = sh.bins[b0 - i]; s += v[i]; }
      const u64 upto = sum_up(s, lane);
      const u64 some = __ballot(s != 0), reached = __ballot(s != 0 && (double)(base + upto) >= limit);
      const int at = reached ? __ffsll(reached) - 1 : some ? 63 - __clzll(some) : 63;     // (some: its last one)
      if (lane == at) {
        u64 before = base + upto - s;
        int i = 0, last = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) last = v[k] ? k : last;
        while (i < last && !(v[i] && (double)(before + v[i]) >= limit)) before += v[i++];
        sh.bin = (unsigned)(b0 - i);
        sh.base = before;
        sh.value = v[i];
      }
    }
    __syncthreads();
    key |= sh.bin << bits;
    base = sh.base;
    value = sh.value;
  }
  if (sizeof(T) == 2 && !(key & 0x80000000u)) key |= 0xffffu;    // (negative bf16 values have all of the lower bits)
  Prefix p;
  p.key = key;
  const u64 w = measure(key & 0x80000000u ? __builtin_bit_cast(float, key & 0x7fffffffu) : __builtin_bit_cast(float, ~key));
  // the fewest of the equal ones that reach the limit
  const u64 all = w ? value / w : 0;
  u64 ties = all;
  if (all > 1) {
    const double want = (limit - (double)base) / (double)w;
    ties = want < 1.0 ? 1 : want > (double)all ? all : (u64)want;
    while (ties > 1 && (double)(base + (ties - 1) * w) >= limit) --ties;
    while (ties < all && !((double)(base + ties * w) >= limit)) ++ties;
  }
  p.ties = ties;
  p.sum = base + ties * w;
  return p;
}

// The first class in index order up to which the measures sum to more than `target` (0 <= target); -1 if none does
template <typename T, int TH, int NV, typename M>
__device__ __forceinline__ long long first_beyond(const Row<T, TH, NV>& row, double target, Shared& sh, M measure) {
  constexpr int N = Row<T, TH, NV>::N, W = TH / 64;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  u64 base = 0;
  __syncthreads();
  if (threadIdx.x == 0) sh.found = -1;
  // segments, 64 N classes each, in groups of 256: 256 / W vectors of every thread
  constexpr int G = 256 / W;
  for (int i0 = 0; i0 < row.n; i0 += G) {
    const int i1 = i0 + G < row.n ? i0 + G : row.n;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < (NV ? NV : G); ++k) {
      const int i = i0 + k;
      if (i >= i1) break;
      const u32x4 v = row.vec(NV ? k : i);
      u64 s = 0;
#pragma unroll
      for (int j = 0; j < N; ++j) s += measure(entry<T>(v, j), row.at(i) + j);
      s = sum_wave(s);
      if (lane == 0) sh.segment[k * W + wave] = s;
    }
    __syncthreads();
    // every wavefront: where in this group (four segments a lane)
    const int many = (i1 - i0) * W;
    u64 v[4], s = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) { v[j] = 4 * lane + j < many ? sh.segment[4 * lane + j] : 0; s += v[j]; }
    const u64 upto = base + sum_up(s, lane);
    const u64 beyond = __ballot((double)upto > target);
    if (!beyond) { base = shuffle(upto, 63); continue; }
    const int at = __ffsll(beyond) - 1;
    u64 before = upto - s;
    int j = 0;
#pragma unroll
    for (int k = 0; k < 3; ++k)
      if (j == k && !((double)(before + v[k]) > target)) { before += v[k]; ++j; }
    const int segment = 4 * at + __shfl(j, at);
    before = shuffle(before, at);
    if (segment % W == wave) {
      const int i = i0 + segment / W;
      const u32x4 x = row.read(i);                               // (registers have no index)
      u64 m[N], t = 0;
#pragma unroll
      for (int k = 0; k < N; ++k) { m[k] = measure(entry<T>(x, k), row.at(i) + k); t += m[k]; }
      const u64 here = before + sum_up(t, lane);
      const u64 who = __ballot((double)here > target);
      if (lane == __ffsll(who) - 1) {
        u64 a = here - t;
        long long found = row.at(i);
#pragma unroll
        for (int k = 0; k < N; ++k) {
          a += m[k];
          found += !((double)a > target);
        }
        sh.found = found;
      }
    }
    break;
  }
  __syncthreads();
  return sh.found;
}

template <typename T, int TH, int NV>
__global__ __launch_bounds__(TH) void sample_kernel(SampleArgs a, long long first) {
  __shared__ Shared sh;
  const long long b = first + blockIdx.x, V = a.V;
  const int lane = threadIdx.x & 63;
  Row<T, TH, NV> row;
  row.init(static_cast<const T*>(a.logits) + b * V, V);
  const float u = a.u[b], t = a.temperature ? a.temperature[b] : 1.0f, p = a.top_p ? a.top_p[b] : 1.0f, least = a.min_p ? a.min_p[b] : 0.0f;
  const int k = a.top_k ? a.top_k[b] : 0;
  // the largest logit, and whether there is anything that has no place in a row
  float top = -INFINITY;
  unsigned bad = 0;
  row.each([&](float x) { top = fmaxf(top, x); bad |= x != x || x == INFINITY; });
#pragma unroll
  for (int d = 32; d; d >>= 1) { top = fmaxf(top, __shfl_xor(top, d)); bad |= __shfl_xor(bad, d); }
  if (lane == 0) { sh.top[threadIdx.x >> 6] = top; sh.bad[threadIdx.x >> 6] = bad; }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < TH / 64; ++w) { top = fmaxf(top, sh.top[w]); bad |= sh.bad[w]; }
  if (bad || top == -INFINITY || !(t >= 0.0f) || t == INFINITY || !(u >= 0.0f && u < 1.0f) || p != p || least != least) {
    if (threadIdx.x == 0) {
      a.index[b] = -1;
      if (a.logprob) a.logprob[b] = NAN;
    }
    return;
  }
  if (t == 0.0f || p <= 0.0f || k == 1) {                        // the first of the order
    const long long at = first_beyond(row, 0.0, sh, [&](float x, long long) { return (u64)(x == top); });
    if (threadIdx.x == 0) {
      a.index[b] = at;
      if (a.logprob) a.logprob[b] = 0.0f;
    }
    return;
  }
  int log2V = 0;
  while ((1LL << log2V) < V) ++log2V;
  Weights w;
  w.top = top;
  w.rate = 1.44269504088896340736 / (double)t;
  w.shift = 62 - log2V < 50 ? 62 - log2V : 50;
  w.floor = -w.shift - 2.0;
  u64 sum = 0;                       // of the weights that are left
  unsigned key = 0;                  // classes with larger keys are left, and those with this one up to index `last`
  u64 ties = ~0ull;
  bool cut = false;
  if (k > 1 && k < V) {
    const Prefix f = first_ones(row, (double)k, sh, [&](float) { return (u64)1; });
    key = f.key;
    ties = f.ties;
    cut = true;
    u64 s = 0;
    row.each([&](float x) { s += key_of(x) > key ? w.of(x) : 0; });
    sum = sum_threads<TH>(s, sh) + ties * w.of(key & 0x80000000u ? __builtin_bit_cast(float, key & 0x7fffffffu) : __builtin_bit_cast(float, ~key));
  } else {
    u64 s = 0;
    row.each([&](float x) { s += w.of(x); });
    sum = sum_threads<TH>(s, sh);
  }
  if (p < 1.0f) {                    // (a prefix of the first k: its limit is at most their sum)
    const Prefix f = first_ones(row, (double)p * (double)sum, sh, [&](float x) { return w.of(x); });
    if (!cut || f.key > key || (f.key == key && f.ties < ties)) {
      key = f.key;
      ties = f.ties;
      sum = f.sum;
      cut = true;
    }
  }
  // the index of the last of the equal ones that is left
  long long last = V;
  if (cut) {
    last = first_beyond(row, (double)(ties - 1), sh, [&](float x, long long at) { return (u64)(at < V && key_of(x) == key); });
    if (last < 0) last = V;
  }
  const double yleast = least > 0.0f ? (double)(least < 1.0f ? least : 1.0f) : 0.0;
  auto kept = [&](float x, long long at) -> u64 {
    const unsigned o = key_of(x);
    if (cut && (o < key || (o == key && at > last))) return 0;
    if (yleast > 0.0 && x != top && !(power2(((double)x - w.top) * w.rate, 0) >= yleast)) return 0;
    return w.of(x);
  };
  if (yleast > 0.0) {
    u64 s = 0;
#pragma unroll row.U
    for (int i = 0; i < row.n; ++i) {
      const u32x4 v = row.vec(i);
#pragma unroll
      for (int j = 0; j < row.N; ++j) s += kept(entry<T>(v, j), row.at(i) + j);
    }
    sum = sum_threads<TH>(s, sh);
  }
  long long at = first_beyond(row, (double)u * (double)sum, sh, kept);
  if (at < 0) at = first_beyond(row, 0.0, sh, kept);             // (u times the sum rounded up to the sum: cannot be, u < 1 - 2^-25)
  if (threadIdx.x == 0) {
    a.index[b] = at;
    if (a.logprob) {
      const float x = static_cast<float>(static_cast<const T*>(a.logits)[b * V + at]);
      a.logprob[b] = (float)(((double)x - w.top) / (double)t - (log((double)sum) - w.shift * 0.693147180559945309417));
    }
  }
}

template <typename T>
hipError_t launch_rows(const SampleArgs& a, hipStream_t s) {
  constexpr int N = Eight<T>::N;
  for (long long r = 0; r < a.B; r += 1LL << 21) {               // (a launch has fewer than 2^32 threads)
    const dim3 grid((unsigned)(a.B - r < 1LL << 21 ? a.B - r : 1LL << 21));
    const long long vectors = ((long long)a.V + N - 1) / N;
#define SAMPLE(TH, NV) hipLaunchKernelGGL((sample_kernel<T, TH, NV>), grid, dim3(TH), 0, s, a, r)
    if (vectors <= 64) SAMPLE(64, 1);
    else if (vectors <= 256) SAMPLE(256, 1);
    else if (vectors <= 512) SAMPLE(256, 2);
    else if (vectors <= 1024) SAMPLE(256, 4);
    else if (vectors <= 2048) SAMPLE(1024, 2);
    else if (vectors <= 4096) SAMPLE(1024, 4);
    else if (vectors <= 8192) SAMPLE(1024, 8);
    else if (vectors <= 16384) SAMPLE(1024, 16);
    else SAMPLE(1024, 0);
#undef SAMPLE
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_sample(const SampleArgs& a, hipStream_t s) { return a.dtype ? launch_rows<__bf16>(a, s) : launch_rows<float>(a, s); }

}  // namespace mgrit
