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

// 2^y 2^shift, y <= 0, to 2e-14: y = n + f with |f| <= 1/2, and 2^f by the polynomial of degree 9 whose largest relative error there is
// least (1.4e-14; found by exchange of the extrema).  Adding 1.5 2^52 rounds to a whole number, whose low bits are those of the sum.
__device__ __forceinline__ double power2(double y, int shift) {
  const double t = y + 6755399441055744.0, f = y - (t - 6755399441055744.0);
  double p = 1.0150336822370344e-07;
  p = __builtin_fma(p, f, 1.325940561258553e-06);
  p = __builtin_fma(p, f, 1.5252984837896388e-05);
  p = __builtin_fma(p, f, 0.00015403434948052159);
  p = __builtin_fma(p, f, 0.001333355761760602);
  p = __builtin_fma(p, f, 0.009618129192067285);
  p = __builtin_fma(p, f, 0.0555041086686856);
  p = __builtin_fma(p, f, 0.24022650695649653);
  p = __builtin_fma(p, f, 0.693147180559871);
  p = __builtin_fma(p, f, 1.0000000000000127);
  return __builtin_ldexp(p, (int)(unsigned)__builtin_bit_cast(u64, t) + shift);
}
// Weights exp((x - top) / t) in units of 2^-shift, rounded to whole ones, so that sums are exact and do not depend on their order
struct Weights {
  double top, rate;                  // rate = log2(e) / t
  int shift;
  double floor;                      // y of weights that are zero from there on
  double least;                      // weights below it do not count but the largest one's
  __device__ __forceinline__ u64 of(float x) const {
    const double d = (double)x - top, y = d * rate;
    if (!(y > floor)) return 0;
    const double w = power2(y, shift);
    // (below 2^51 + 2^52: the whole units are the last bits)
    return w >= least || d == 0.0 ? __builtin_bit_cast(u64, w + 4503599627370496.0) & 0xfffffffffffffull : 0;
  }
};

// What a workgroup knows of its row, and its places in LDS
struct Candidate { unsigned key, at; u64 measure; };
template <int TH> struct Shared {
  union {
    u64 bins[2 * TH];
    Candidate candidates[TH];
    u64 segment[256];                // sums of the wavefronts' parts of the row, in order
  };
  u64 part[16];
  u64 base, value;
  unsigned bin, count, least, most;
  unsigned key, last;
  u64 sum;
  long long found;
  float top[16], low[16];
  unsigned bad[16];
};

// The row's vectors: in LDS (HELD), each at the thread that uses it, or read again.  (In registers, where an index has to be known, every pass is unrolled
// and the compiler keeps keys and doubles of one pass for the next, two thousand registers too many.)
template <typename T, int TH, bool HELD>
struct Row {
  static constexpr int N = Eight<T>::N;
  const T* x;
  u32x4* held;
  long long V;
  int n;                             // vectors of a thread
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
  __device__ __forceinline__ void init(const T* x_, long long V_, u32x4* lds) {
    x = x_; V = V_; held = lds;
    n = (int)((V + (long long)TH * N - 1) / ((long long)TH * N));
    if constexpr (HELD) {
#pragma unroll 4
      for (int i = 0; i < n; ++i) held[i * TH + threadIdx.x] = read(i);
    }
  }
  __device__ __forceinline__ u32x4 vec(int i) const { if constexpr (HELD) return held[i * TH + threadIdx.x]; else return read(i); }
  // f(x, index) for each of this thread's entries
  template <typename F> __device__ __forceinline__ void each(F f) const {
#pragma unroll 1
    for (int i = 0; i < n; ++i) {
      const u32x4 v = vec(i);
#pragma unroll
      for (int j = 0; j < N; ++j) f(entry<T>(v, j), at(i) + j);
    }
  }
};

template <int TH> __device__ __forceinline__ u64 sum_threads(u64 v, Shared<TH>& sh) {
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

// The first class in index order up to which the measures sum to more than `target` (0 <= target); -1 if none does
template <typename T, int TH, bool HELD, typename M>
__device__ __forceinline__ long long first_beyond(const Row<T, TH, HELD>& row, double target, Shared<TH>& sh, M measure) {
  constexpr int N = Row<T, TH, HELD>::N, W = TH / 64;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  u64 base = 0;
  __syncthreads();
  if (threadIdx.x == 0) sh.found = -1;
  // segments, 64 N classes each, in groups of 256: 256 / W vectors of every thread
  constexpr int G = 256 / W;
  for (int i0 = 0; i0 < row.n; i0 += G) {
    const int i1 = i0 + G < row.n ? i0 + G : row.n;
    __syncthreads();
#pragma unroll 1
    for (int i = i0; i < i1; ++i) {
      const u32x4 v = row.vec(i);
      u64 s = 0;
#pragma unroll
      for (int j = 0; j < N; ++j) s += measure(entry<T>(v, j), row.at(i) + j);
      s = sum_wave(s);
      if (lane == 0) sh.segment[(i - i0) * W + wave] = s;
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
      const u32x4 x = row.vec(i);
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

// The first classes in falling order whose measures reach a limit: those with larger keys than `key`, and of those with that key the ones up to
// index `last`; sum: the measure of all of them
struct Prefix { unsigned key; long long last; u64 sum; };
__device__ __forceinline__ float value_of(unsigned key) { return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key); }

// By a descent over the key's bits, eight at a time from the top: bins of the measures of what agrees so far, and the bin in which the limit is
// reached.  Any row, but many classes meet in few bins.
template <typename T, int TH, bool HELD, typename M>
__device__ __forceinline__ Prefix descend(const Row<T, TH, HELD>& row, double limit, Shared<TH>& sh, M measure) {
  constexpr int LEVELS = sizeof(T) == 4 ? 4 : 2;
  static_assert(TH >= 64, "bins");
  u64* const bins = sh.bins;
  constexpr int BITS = TH >= 128 ? 8 : 4, BINS = 1 << BITS, STEPS = LEVELS * 8 / BITS;
  unsigned key = 0;
  u64 base = 0, value = 0;
  for (int level = 0; level < STEPS; ++level) {
    const int bits = 32 - BITS * (level + 1);
    __syncthreads();
    for (int b = threadIdx.x; b < BINS; b += TH) bins[b] = 0;
    __syncthreads();
    row.each([&](float x, long long at) {
      const unsigned k = key_of(x);
      if (level && (k >> (bits + BITS)) != (key >> (bits + BITS))) return;
      const u64 m = measure(x, at);
      if (m) atomicAdd(&bins[k >> bits & (BINS - 1)], m);
    });
    __syncthreads();
    if (threadIdx.x == 0) {
      int b = BINS - 1, last = BINS - 1;
      u64 before = base;
      for (; b >= 0; --b) {
        if (!bins[b]) continue;
        last = b;
        if ((double)(before + bins[b]) >= limit) break;
        before += bins[b];
      }
      if (b < 0) before -= bins[last];                           // (a limit beyond all: the last one)
      sh.bin = (unsigned)last;
      sh.base = before;
      sh.value = bins[last];
    }
    __syncthreads();
    key |= sh.bin << bits;
    base = sh.base;
    value = sh.value;
  }
  if (sizeof(T) == 2 && !(key & 0x80000000u)) key |= 0xffffu;    // (negative bf16 values have all of the lower bits)
  return Prefix{key, -1, base};
}
// Of the classes with this key, whose measure is all the same, the fewest that reach the limit from base on; share > 0: that part of what they sum to
template <typename T, int TH, bool HELD, typename M>
__device__ __forceinline__ Prefix among_equal(const Row<T, TH, HELD>& row, unsigned key, u64 base, double limit, double share, Shared<TH>& sh, M measure) {
  u64 mine = 0, n = 0;
  row.each([&](float x, long long at) {
    if (key_of(x) != key) return;
    const u64 m = measure(x, at);
    if (m) { mine = m; ++n; }
  });
  const u64 all = sum_threads<TH>(n, sh);
#pragma unroll
  for (int d = 32; d; d >>= 1) { const u64 o = shuffle_xor(mine, d); mine = o > mine ? o : mine; }
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sh.part[threadIdx.x >> 6] = mine;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < TH / 64; ++w) mine = sh.part[w] > mine ? sh.part[w] : mine;
  if (share > 0.0) limit = share * (double)(all * mine);
  const double want = mine ? (limit - (double)base) / (double)mine : 1.0;
  u64 ties = want < 1.0 ? 1 : want > (double)all ? all : (u64)want;
  while (ties > 1 && (double)(base + (ties - 1) * mine) >= limit) --ties;
  while (ties < all && !((double)(base + ties * mine) >= limit)) ++ties;
  const long long last = first_beyond(row, (double)(ties - 1), sh, [&](float x, long long at) { return (u64)(key_of(x) == key && measure(x, at)); });
  return Prefix{key, last < 0 ? row.V : last, base + ties * mine};
}
// measure(x, index): 0 of classes that do not take part; top, low: the largest and smallest of the others.  The limit is `share` of the sum of all measures,
// or `most` (or all).  Bins of equal width over the logits between top and low, and the few classes of the bin in which the limit is reached compared with
// each other; a bin of many is divided again.  (Bins by the leading bits of the keys hold most of a row in a handful of them, and LDS atomics on one
// address take turns: 4096 rows of 50021 bf16 took 9.5 ms.)
template <typename T, int TH, bool HELD, typename M>
__device__ __forceinline__ Prefix first_ones(const Row<T, TH, HELD>& row, float top, float low, double share, double most, Shared<TH>& sh, M measure) {
  constexpr int BINS = 2 * TH;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  float hi = top, lo = low;
  u64 base = 0;
  double limit = 0.0;
  for (int level = 0; level < 4; ++level) {
    if (lo == hi) return among_equal(row, key_of(hi), base, level ? limit : most, level ? 0.0 : share, sh, measure);
    const float half = hi * 0.5f, rate = (float)(BINS - 1) / (half - lo * 0.5f);
    auto bin_of = [&](float x) {
      const float b = (half - x * 0.5f) * rate;
      return b < (float)(BINS - 1) ? (int)b : BINS - 1;
    };
    __syncthreads();
    sh.bins[threadIdx.x] = 0;
    sh.bins[threadIdx.x + TH] = 0;
    __syncthreads();
    row.each([&](float x, long long at) {
      if (x > hi || x < lo) return;
      const u64 m = measure(x, at);
      if (m) atomicAdd(&sh.bins[bin_of(x)], m);
    });
    __syncthreads();
    const u64 a = sh.bins[2 * threadIdx.x], b = sh.bins[2 * threadIdx.x + 1];
    const u64 up = sum_up(a + b, lane);
    if (lane == 63) sh.part[wave] = up;
    if (threadIdx.x == 0) { sh.count = 0; sh.least = 0xffffffffu; sh.most = 0; }
    __syncthreads();
    u64 before = base, total = base;
#pragma unroll
    for (int w = 0; w < TH / 64; ++w) { before += w < wave ? sh.part[w] : 0; total += sh.part[w]; }
    if (level == 0) {
      limit = share > 0.0 ? share * (double)total : most;
      limit = limit < (double)total ? limit : (double)total;
    }
    before += up - a - b;
    if ((double)before < limit && (double)(before + a + b) >= limit) {
      const bool second = (double)(before + a) < limit;
      sh.bin = 2 * threadIdx.x + second;
      sh.base = second ? before + a : before;
    }
    __syncthreads();                                             // (the bins have been read)
    const int border = (int)sh.bin;
    base = sh.base;
    row.each([&](float x, long long at) {
      if (x > hi || x < lo || bin_of(x) != border) return;
      const u64 m = measure(x, at);
      if (!m) return;
      const unsigned k = key_of(x), slot = atomicAdd(&sh.count, 1u);
      if (slot < TH) sh.candidates[slot] = Candidate{k, (unsigned)at, m};
      atomicMin(&sh.least, k);
      atomicMax(&sh.most, k);
    });
    __syncthreads();
    const int n = (int)sh.count;
    if (n <= TH) {
      if (threadIdx.x < n) {
        const Candidate c = sh.candidates[threadIdx.x];
        u64 s = base;
        for (int i = 0; i < n; ++i) {
          const Candidate o = sh.candidates[i];
          s += o.key > c.key || (o.key == c.key && o.at < c.at) ? o.measure : 0;
        }
        if ((double)s < limit && (double)(s + c.measure) >= limit) {
          sh.key = c.key;
          sh.last = c.at;
          sh.sum = s + c.measure;
        }
      }
      __syncthreads();
      return Prefix{sh.key, (long long)sh.last, sh.sum};
    }
    lo = value_of(sh.least);
    hi = value_of(sh.most);
    __syncthreads();
  }
  const Prefix p = descend(row, limit, sh, measure);
  return among_equal(row, p.key, p.sum, limit, 0.0, sh, measure);
}

template <typename T, int TH, bool HELD>
__global__ __launch_bounds__(TH) void sample_kernel(SampleArgs a, long long first) {
  __shared__ Shared<TH> sh;
  const long long b = first + blockIdx.x, V = a.V;
  const int lane = threadIdx.x & 63;
  extern __shared__ u32x4 held[];
  Row<T, TH, HELD> row;
  row.init(static_cast<const T*>(a.logits) + b * V, V, held);
  const float u = a.u[b], t = a.temperature ? a.temperature[b] : 1.0f, p = a.top_p ? a.top_p[b] : 1.0f, least = a.min_p ? a.min_p[b] : 0.0f;
  const int k = a.top_k ? a.top_k[b] : 0;
  // the largest logit, the smallest above minus infinity, and whether there is anything that has no place in a row
  float top = -INFINITY, low = INFINITY;
  unsigned bad = 0;
  row.each([&](float x, long long) {
    top = fmaxf(top, x);
    low = x > -INFINITY ? fminf(low, x) : low;
    bad |= x != x || x == INFINITY;
  });
#pragma unroll
  for (int d = 32; d; d >>= 1) { top = fmaxf(top, __shfl_xor(top, d)); low = fminf(low, __shfl_xor(low, d)); bad |= __shfl_xor(bad, d); }
  if (lane == 0) { sh.top[threadIdx.x >> 6] = top; sh.low[threadIdx.x >> 6] = low; sh.bad[threadIdx.x >> 6] = bad; }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < TH / 64; ++w) { top = fmaxf(top, sh.top[w]); low = fminf(low, sh.low[w]); bad |= sh.bad[w]; }
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
  w.least = 0.0;
  // classes with larger keys than this are left, and those with this one up to index `last`
  unsigned key = 0;
  long long last = V;
  u64 sum = 0;                       // of the weights that are left
  bool summed = false;
  if (k > 1 && k < V) {
    const Prefix f = first_ones(row, top, low, 0.0, (double)k, sh, [&](float x, long long) { return (u64)(x > -INFINITY); });
    key = f.key;
    last = f.last;
  }
  auto kept = [&](float x, long long at) -> u64 {
    const unsigned o = key_of(x);
    return o < key || (o == key && at > last) ? 0 : w.of(x);
  };
  if (p < 1.0f) {
    // (weights are zero from 2^floor on)
    const float end = (float)((double)top + 1.01 * w.floor / w.rate);
    const Prefix f = first_ones(row, top, fmaxf(low, key ? fmaxf(end, value_of(key)) : end), (double)p, 0.0, sh, kept);
    key = f.key;
    last = f.last;
    sum = f.sum;
    summed = true;
  }
  if (least > 0.0f) w.least = __builtin_ldexp((double)(least < 1.0f ? least : 1.0f), w.shift);
  if (!summed || least > 0.0f) {
    u64 s = 0;
    row.each([&](float x, long long at) { s += kept(x, at); });
    sum = sum_threads<TH>(s, sh);
  }
  const long long at = first_beyond(row, (double)u * (double)sum, sh, kept);
  if (threadIdx.x == 0) {
    a.index[b] = at;
    if (a.logprob) {
      const float x = static_cast<float>(static_cast<const T*>(a.logits)[b * V + at]);
      a.logprob[b] = (float)(((double)x - w.top) / (double)t - (log((double)sum) - w.shift * 0.693147180559945309417));
    }
  }
}

constexpr size_t HELD_BYTES = 140 * 1024;                        // of a row in LDS beside what the workgroup shares
template <typename T, int TH, bool HELD>
hipError_t launch_held(const SampleArgs& a, size_t smem, hipStream_t s) {
  static LdsOptIn opt;
  // (the attribute is one of dynamic LDS alone, the limit of 64 KB without it one of both kinds)
  const size_t asked = smem + sizeof(Shared<TH>) > 64 * 1024 && smem <= 64 * 1024 ? 64 * 1024 + 16 : smem;
  const hipError_t e = opt.raise(reinterpret_cast<const void*>(&sample_kernel<T, TH, HELD>), asked);
  if (e != hipSuccess) return e;
  for (long long r = 0; r < a.B; r += 1LL << 21)                 // (a launch has fewer than 2^32 threads)
    hipLaunchKernelGGL((sample_kernel<T, TH, HELD>), dim3((unsigned)(a.B - r < 1LL << 21 ? a.B - r : 1LL << 21)), dim3(TH), smem, s, a, r);
  return hipGetLastError();
}
template <typename T, int TH>
hipError_t launch_threads(const SampleArgs& a, hipStream_t s) {
  const size_t whole = TH * 16, smem = ((size_t)a.V * sizeof(T) + whole - 1) / whole * whole;
  return smem <= HELD_BYTES ? launch_held<T, TH, true>(a, smem, s) : launch_held<T, TH, false>(a, 0, s);
}
template <typename T>
hipError_t launch_rows(const SampleArgs& a, hipStream_t s) {
  const long long vectors = ((long long)a.V + Eight<T>::N - 1) / Eight<T>::N;
  return vectors <= 256 ? launch_threads<T, 64>(a, s) : vectors <= 2048 ? launch_threads<T, 256>(a, s) : launch_threads<T, 1024>(a, s);
}

}  // namespace

hipError_t launch_sample(const SampleArgs& a, hipStream_t s) { return a.dtype ? launch_rows<__bf16>(a, s) : launch_rows<float>(a, s); }

}  // namespace mgrit
