// One class for each row of logits, from a given random number: temperature, top-k, top-p, min-p.
#include <float.h>

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
__device__ __forceinline__ double power2(double y, double magic) {        // magic = 1.5 2^52 + shift
  const double t = y + magic, f = y - (t - magic);
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
  return __builtin_ldexp(p, (int)(unsigned)__builtin_bit_cast(u64, t));
}
// Weights exp((x - top) / t) in units of 2^-shift, rounded to whole ones, so that sums are exact and do not depend on their order
struct Weights {
  double top, rate;                  // rate = log2(e) / t
  double magic;                      // 1.5 2^52 + shift
  double floor;                      // y from which on weights are less than half a unit: nothing
  __device__ __forceinline__ double exact(float x) const { return power2(__builtin_fmax(((double)x - top) * rate, floor), magic); }
  // (no branches: the chain of a weight's twenty operations is hidden behind the other seven's.  Below 2^51 + 2^52 the whole units are the last bits)
  __device__ __forceinline__ u64 of(float x) const { return __builtin_bit_cast(u64, exact(x) + 4503599627370496.0) & 0xfffffffffffffull; }
};

// What a workgroup knows of its row, and its places in LDS
struct Candidate { unsigned key, at; u64 measure; };
template <int TH> struct Shared {
  union {
    u64 bins[2 * TH];
    Candidate candidates[TH];
  };
  u64 part[16];
  u64 base;
  unsigned bin, count, least, most;
  unsigned key, last;
  long long found;
  float top[16], low[16];
  unsigned bad[16];
};

// The row's vectors, a contiguous part of the row for each wavefront: in LDS (HELD), each at the thread that uses it, or read again.  (In registers, where an
// index has to be known, every pass is unrolled, and the compiler keeps keys and doubles of one pass for the next, two thousand registers too many.)
template <typename T, int TH, bool HELD>
struct Row {
  static constexpr int N = Eight<T>::N;
  const T* x;
  u32x4* held;
  long long V;
  int n;                             // vectors of a thread
  __device__ __forceinline__ unsigned place(int wave, int i) const { return ((unsigned)wave * n + i) * 64 + (threadIdx.x & 63); }
  // index of the first class in this lane's vector i of a wavefront's (V < 2^31 and less than a round of all threads' vectors behind it)
  __device__ __forceinline__ unsigned at(int wave, int i) const { return place(wave, i) * N; }
  __device__ __forceinline__ u32x4 read(int wave, int i) const {
    const long long k = at(wave, i);
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
  // f(vector) of all of them, as they come in
  template <typename F> __device__ __forceinline__ void init(const T* x_, long long V_, u32x4* lds, F f) {
    x = x_; V = V_; held = lds;
    n = (int)((V + (long long)TH * N - 1) / ((long long)TH * N));
    const int wave = threadIdx.x >> 6;
    int i = 0;
    for (; i + 4 <= n; i += 4) {     // four are on their way
      u32x4 v[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = read(wave, i + j);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (HELD) held[place(wave, i + j)] = v[j];
        f(v[j]);
      }
    }
    for (; i < n; ++i) {
      const u32x4 v = read(wave, i);
      if (HELD) held[place(wave, i)] = v;
      f(v);
    }
  }
  __device__ __forceinline__ u32x4 vec(int wave, int i) const { if constexpr (HELD) return held[place(wave, i)]; else return read(wave, i); }
  // f(x, index) for each of this thread's entries
  template <typename F> __device__ __forceinline__ void each(F f) const {
    const int wave = threadIdx.x >> 6;
#pragma unroll 1
    for (int i = 0; i < n; ++i) {
      const u32x4 v = vec(wave, i);
      const unsigned k = at(wave, i);
#pragma unroll
      for (int j = 0; j < N; ++j) f(entry<T>(v, j), k + j);
    }
  }
  // measure(x) of those of this lane's vector that take part, zero of the others; false, and nothing computed, where no lane has one that does
  template <typename P, typename M> __device__ __forceinline__ bool measures(int wave, int i, u64 (&m)[N], P part, M measure) const {
    const u32x4 v = vec(wave, i);
    const unsigned k = at(wave, i);
    bool in[N], any = false;
#pragma unroll
    for (int j = 0; j < N; ++j) { in[j] = part(entry<T>(v, j), k + j); any |= in[j]; }
    if (!__any(any)) return false;
#pragma unroll
    for (int j = 0; j < N; ++j) m[j] = measure(entry<T>(v, j));
#pragma unroll
    for (int j = 0; j < N; ++j) m[j] = in[j] ? m[j] : 0;
    return true;
  }
};

// A place among sh.candidates for every lane that has one to put there; all lanes of the wavefront call it
template <int TH> __device__ __forceinline__ unsigned slot_for(bool have, Shared<TH>& sh) {
  const u64 who = __ballot(have);
  if (!who) return 0xffffffffu;
  const int lane = threadIdx.x & 63;
  unsigned first = 0;
  if (lane == 0) first = atomicAdd(&sh.count, (unsigned)__popcll(who));
  first = (unsigned)__builtin_amdgcn_readfirstlane((int)first);
  return have ? first + (unsigned)__popcll(who & ((1ull << lane) - 1)) : 0xffffffffu;
}
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

// The first class in index order up to which the measures of those that take part sum to more than `target` (>= 0), or than share >= 0 of all measures;
// -1 if none does.  total: of all of them.  First which wavefront's part of the row, then which of its vectors, one for each wavefront, then which lane.
template <typename T, int TH, bool HELD, typename P, typename M>
__device__ __forceinline__ long long first_beyond(const Row<T, TH, HELD>& row, double target, double share, u64* total, Shared<TH>& sh, P part, M measure) {
  constexpr int N = Row<T, TH, HELD>::N, W = TH / 64;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  u64 m[N], s = 0;
#pragma unroll 1
  for (int i = 0; i < row.n; ++i) {
    if (!row.measures(wave, i, m, part, measure)) continue;
#pragma unroll
    for (int j = 0; j < N; ++j) s += m[j];
  }
  s = sum_wave(s);
  __syncthreads();                   // (whoever still reads an earlier sum)
  if (lane == 0) sh.part[wave] = s;
  if (threadIdx.x == 0) sh.found = -1;
  __syncthreads();
  u64 all = 0;
#pragma unroll
  for (int w = 0; w < W; ++w) all += sh.part[w];
  *total = all;
  if (share >= 0.0) target = share * (double)all;
  u64 before = 0;
  int owner = 0;
  while (owner < W && !((double)(before + sh.part[owner]) > target)) before += sh.part[owner++];
  if (owner == W) return -1;
  // the owner's vectors, W at a time
  for (int i0 = 0; i0 < row.n; i0 += W) {
    const int i = i0 + wave;
    u64 t = 0;
    if (i < row.n && row.measures(owner, i, m, part, measure)) {
#pragma unroll
      for (int j = 0; j < N; ++j) t += m[j];
    } else {
#pragma unroll
      for (int j = 0; j < N; ++j) m[j] = 0;
    }
    const u64 upto = sum_up(t, lane);
    __syncthreads();
    if (lane == 63) sh.part[wave] = upto;
    __syncthreads();
    u64 mine = before;
    int at = 0;
    while (at < W && !((double)(before + sh.part[at]) > target)) before += sh.part[at++];
#pragma unroll
    for (int w = 0; w < W; ++w) mine += w < wave ? sh.part[w] : 0;
    if (at == W) continue;
    if (at == wave) {
      const u64 who = __ballot((double)(mine + upto) > target);
      if (lane == __ffsll(who) - 1) {
        u64 a = mine + upto - t;
        long long found = row.at(owner, i);
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
// index `last`
struct Prefix { unsigned key, last; };
__device__ __forceinline__ float value_of(unsigned key) { return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key); }

struct Above { unsigned key; u64 base; };                        // base: the measure of larger keys
// By a descent over the key's bits, eight at a time from the top: bins of the measures of what agrees so far, and the bin in which the limit is
// reached.  Any row, but many classes meet in few bins.
template <typename T, int TH, bool HELD, typename P, typename M>
__device__ __forceinline__ Above descend(const Row<T, TH, HELD>& row, double limit, Shared<TH>& sh, P part, M measure) {
  constexpr int LEVELS = sizeof(T) == 4 ? 4 : 2;
  static_assert(TH >= 64, "bins");
  u64* const bins = sh.bins;
  constexpr int BITS = TH >= 128 ? 8 : 4, BINS = 1 << BITS, STEPS = LEVELS * 8 / BITS;
  unsigned key = 0;
  u64 base = 0;
  for (int level = 0; level < STEPS; ++level) {
    const int bits = 32 - BITS * (level + 1);
    __syncthreads();
    for (int b = threadIdx.x; b < BINS; b += TH) bins[b] = 0;
    __syncthreads();
    row.each([&](float x, unsigned at) {
      const unsigned k = key_of(x);
      if (level && (k >> (bits + BITS)) != (key >> (bits + BITS))) return;
      const u64 m = part(x, at) ? measure(x) : 0;
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
    }
    __syncthreads();
    key |= sh.bin << bits;
    base = sh.base;
  }
  if (sizeof(T) == 2 && !(key & 0x80000000u)) key |= 0xffffu;    // (negative bf16 values have all of the lower bits)
  return Above{key, base};
}
// Of the classes with this key, whose measure is all the same, the fewest that reach the limit from base on; share > 0: that part of what they sum to
template <typename T, int TH, bool HELD, typename P, typename M>
__device__ __forceinline__ Prefix among_equal(const Row<T, TH, HELD>& row, unsigned key, u64 base, double limit, double share, Shared<TH>& sh, P part, M measure) {
  u64 mine = 0, n = 0;
  row.each([&](float x, unsigned at) {
    if (key_of(x) != key || !part(x, at)) return;
    const u64 m = measure(x);
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
  u64 unused;
  const long long last = first_beyond(row, (double)(ties - 1), -1.0, &unused, sh, [&](float x, unsigned at) { return key_of(x) == key && part(x, at); },
                                      [&](float x) { return (u64)(measure(x) != 0); });
  return Prefix{key, last < 0 ? 0xffffffffu : (unsigned)last};
}
// part(x, index): whether a class takes part, measure(x): of those; top, low: the largest and smallest of them.  The limit is `share` of the sum of all measures,
// or `most` (or all).  Bins of equal width over the logits between top and low, and the few classes of the bin in which the limit is reached compared with
// each other; a bin of many is divided again.  (Bins by the leading bits of the keys hold most of a row in a handful of them, and LDS atomics on one
// address take turns: 4096 rows of 50021 bf16 took 9.5 ms.)
template <typename T, int TH, bool HELD, typename P, typename M>
__device__ __forceinline__ Prefix first_ones(const Row<T, TH, HELD>& row, float top, float low, double share, double most, Shared<TH>& sh, P part, M measure) {
  constexpr int BINS = 2 * TH;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  float hi = top, lo = low;
  u64 base = 0;
  double limit = 0.0;
  for (int level = 0; level < 4; ++level) {
    if (lo == hi) return among_equal(row, key_of(hi), base, level ? limit : most, level ? 0.0 : share, sh, part, measure);
    const float half = hi * 0.5f, rate = (float)(BINS - 1) / (half - lo * 0.5f);
    auto bin_of = [&](float x) {
      const float b = (half - x * 0.5f) * rate;
      return b < (float)(BINS - 1) ? (int)b : BINS - 1;
    };
    __syncthreads();
    sh.bins[threadIdx.x] = 0;
    sh.bins[threadIdx.x + TH] = 0;
    __syncthreads();
#pragma unroll 1
    for (int i = 0; i < row.n; ++i) {
      u64 m[Eight<T>::N];
      if (!row.measures(wave, i, m, [&](float x, unsigned at) { return x <= hi && x >= lo && part(x, at); }, measure)) continue;
      const u32x4 v = row.vec(wave, i);
#pragma unroll
      for (int j = 0; j < Eight<T>::N; ++j)
        if (m[j]) atomicAdd(&sh.bins[bin_of(entry<T>(v, j))], m[j]);
    }
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
    const float first = border, behind = border < BINS - 1 ? (float)(border + 1) : INFINITY;
    row.each([&](float x, unsigned at) {
      const float b = (half - x * 0.5f) * rate;
      bool have = (b >= first && b < behind) || (behind == INFINITY && !(b < first));
      if (!__any(have)) return;
      have = have && x <= hi && x >= lo && part(x, at);
      const u64 m = have ? measure(x) : 0;
      const unsigned slot = slot_for<TH>(m != 0, sh);
      if (slot < TH) sh.candidates[slot] = Candidate{key_of(x), at, m};
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
        }
      }
      __syncthreads();
      return Prefix{sh.key, sh.last};
    }
    // too many: what they lie between
    unsigned least = 0xffffffffu, greatest = 0;
    row.each([&](float x, unsigned at) {
      if (x > hi || x < lo || bin_of(x) != border || !part(x, at) || !measure(x)) return;
      const unsigned k = key_of(x);
      least = k < least ? k : least;
      greatest = k > greatest ? k : greatest;
    });
    if (least <= greatest) {
      atomicMin(&sh.least, least);
      atomicMax(&sh.most, greatest);
    }
    __syncthreads();
    lo = value_of(sh.least);
    hi = value_of(sh.most);
    __syncthreads();
  }
  const Above p = descend(row, limit, sh, part, measure);
  return among_equal(row, p.key, p.base, limit, 0.0, sh, part, measure);
}

// Sum over the threads up to and with this one, and over all
template <int TH> __device__ __forceinline__ u64 sum_before(u64 v, u64* all, Shared<TH>& sh) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  u64 up = sum_up(v, lane);
  __syncthreads();
  if (lane == 63) sh.part[wave] = up;
  __syncthreads();
  *all = 0;
#pragma unroll
  for (int w = 0; w < TH / 64; ++w) { up += w < wave ? sh.part[w] : 0; *all += sh.part[w]; }
  return up;
}
// The whole answer where the first k of the order are few.  The k'th largest of the threads' largest logits is at most the k'th largest of all, so the
// classes from there on hold the first k and little else; they are put in order by comparing each with each.  mine: this thread's largest; returns false if
// they are more than the threads.  least: the least weight asked for, in the weights' units.
struct Answer { bool done; unsigned at; u64 sum; };
template <typename T, int TH, bool HELD>
__device__ __forceinline__ Answer few_ones(const Row<T, TH, HELD>& row, float mine, float top, float low, int k, float p, double least, float u, const Weights& w,
                                           Shared<TH>& sh) {
  constexpr int BINS = 2 * TH;
  const float half = top * 0.5f, rate = (float)(BINS - 1) / (half - low * 0.5f);
  auto bin_of = [&](float x) {
    const float b = (half - x * 0.5f) * rate;
    return b < (float)(BINS - 1) ? (int)b : BINS - 1;
  };
  __syncthreads();
  sh.bins[threadIdx.x] = 0;
  sh.bins[threadIdx.x + TH] = 0;
  if (threadIdx.x == 0) { sh.count = 0; sh.bin = BINS - 1; }
  __syncthreads();
  if (mine > -INFINITY) atomicAdd(&sh.bins[bin_of(mine)], 1ull);
  __syncthreads();
  const u64 a = sh.bins[2 * threadIdx.x], b = sh.bins[2 * threadIdx.x + 1];
  u64 all;
  const u64 up = sum_before<TH>(a + b, &all, sh);
  if (up - a - b < (u64)k && up >= (u64)k) sh.bin = 2 * threadIdx.x + (up - b < (u64)k);
  __syncthreads();                                               // (the bins have been read)
  const float behind = (int)sh.bin < BINS - 1 ? (float)(sh.bin + 1) : INFINITY;
  row.each([&](float x, unsigned at) {
    const bool have = x > -INFINITY && (behind == INFINITY || !((half - x * 0.5f) * rate >= behind));
    const unsigned slot = slot_for<TH>(have, sh);
    if (slot < TH) sh.candidates[slot] = Candidate{key_of(x), at, 0};
  });
  __syncthreads();
  const int n = (int)sh.count;
  if (n > TH) return Answer{false, 0, 0};
  const int t = threadIdx.x;
  Candidate c = {};
  int rank = 0;
  if (t < n) {
    c = sh.candidates[t];
    for (int i = 0; i < n; ++i) {
      const unsigned key = sh.candidates[i].key, at = sh.candidates[i].at;
      rank += key > c.key || (key == c.key && at < c.at);
    }
  }
  __syncthreads();
  if (t < n) sh.candidates[rank] = c;
  __syncthreads();
  // thread t: class t of the order
  u64 v = 0, total;
  bool good = true;
  if (t < n) {
    c = sh.candidates[t];
    if (t < k) {
      const double e = w.exact(value_of(c.key));
      v = w.of(value_of(c.key));
      good = t == 0 || e >= least;
    }
  }
  const u64 upto = sum_before<TH>(v, &total, sh);
  if (p < 1.0f && !((double)(upto - v) < (double)p * (double)total)) good = false;
  v = good ? v : 0;
  if (t < n) sh.candidates[t].measure = v;
  u64 sum;
  sum_before<TH>(v, &sum, sh);
  const double target = (double)u * (double)sum;
  if (v) {
    u64 before = 0;
    const int m = n < k ? n : k;
    for (int i = 0; i < m; ++i) before += sh.candidates[i].at < c.at ? sh.candidates[i].measure : 0;
    if (!((double)before > target) && (double)(before + v) > target) sh.last = c.at;
  }
  __syncthreads();
  return Answer{true, sh.last, sum};
}

template <typename T, int TH, bool HELD>
__global__ __launch_bounds__(TH) void sample_kernel(SampleArgs a, long long first) {
  __shared__ Shared<TH> sh;
  const long long b = first + blockIdx.x, V = a.V;
  const int lane = threadIdx.x & 63;
  extern __shared__ u32x4 held[];
  Row<T, TH, HELD> row;
  // the largest logit, the smallest above minus infinity, and whether there is anything that has no place in a row
  float top = -INFINITY, low = INFINITY;
  unsigned bad = 0;
  row.init(static_cast<const T*>(a.logits) + b * V, V, held, [&](u32x4 v) {
#pragma unroll
    for (int j = 0; j < Eight<T>::N; ++j) {
      const float x = entry<T>(v, j);
      top = fmaxf(top, x);
      low = x > -INFINITY ? fminf(low, x) : low;
      bad |= !(x < INFINITY);
    }
  });
  const float u = a.u[b], t = a.temperature ? a.temperature[b] : 1.0f, p = a.top_p ? a.top_p[b] : 1.0f, least = a.min_p ? a.min_p[b] : 0.0f;
  const int k = a.top_k ? a.top_k[b] : 0;
  const float mine = top;
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
    u64 unused;
    const long long at = first_beyond(row, 0.0, -1.0, &unused, sh, [&](float x, unsigned) { return x == top; }, [](float) { return (u64)1; });
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
  const int shift = 62 - log2V < 50 ? 62 - log2V : 50;
  w.magic = 6755399441055744.0 + shift;
  w.floor = -shift - 2.0;
  // classes above this logit are left, and those with it up to index `last`
  float edge = -INFINITY;
  unsigned last = 0xffffffffu;
  u64 sum = 0;
  long long at = -1;
  const double asked = __builtin_ldexp(least > 0.0f ? (double)(least < 1.0f ? least : 1.0f) : 0.0, shift);
  if (k > 1 && k < V && k <= TH / 2 && low < top) {
    const Answer f = few_ones(row, mine, top, low, k, p, asked, u, w, sh);
    if (f.done) {
      at = f.at;
      sum = f.sum;
    }
  }
  if (at < 0) {
    if (k > 1 && k < V) {
      const Prefix f = first_ones(row, top, low, 0.0, (double)k, sh, [](float x, unsigned) { return x > -INFINITY; }, [](float) { return (u64)1; });
      edge = value_of(f.key);
      last = f.last;
    }
    auto kept = [&](float x, unsigned at) { return x > edge || (x == edge && at <= last); };
    auto weight = [&](float x) { return w.of(x); };
    if (p < 1.0f) {
      // (weights are nothing from 2^floor on)
      const float end = (float)((double)top + 1.01 * w.floor / w.rate);
      const Prefix f = first_ones(row, top, fmaxf(low, fmaxf(end, edge)), (double)p, 0.0, sh, kept, weight);
      edge = value_of(f.key);
      last = f.last;
    }
    if (least > 0.0f) {
      // the smallest float with a weight of at least least: the weights grow with the logits, so by its key, six bits a step
      unsigned lo = key_of(-FLT_MAX), hi = key_of(top);               // in (lo, hi], or lo itself
      if (w.exact(value_of(lo)) >= asked) hi = lo;
      while (lo + 1 < hi) {
        const unsigned span = hi - lo, step = span > 64 ? (span + 63) / 64 : 1;
        const unsigned mine = span - 1 < (lane + 1) * step ? hi : lo + (lane + 1) * step;       // (the last ones: hi)
        const u64 good = __ballot(mine >= hi || w.exact(value_of(mine)) >= asked);
        const int at = __ffsll(good) - 1;
        const unsigned up = (unsigned)__shfl((int)mine, at), down = at ? (unsigned)__shfl((int)mine, at - 1) : lo;
        hi = up;
        lo = down;
      }
      const float from = value_of(hi);
      if (from > edge) { edge = from; last = 0xffffffffu; }
    }
    at = first_beyond(row, 0.0, (double)u, &sum, sh, kept, weight);
  }
  if (threadIdx.x == 0) {
    a.index[b] = at;
    if (a.logprob) {
      const float x = static_cast<float>(static_cast<const T*>(a.logits)[b * V + at]);
      a.logprob[b] = (float)(((double)x - w.top) / (double)t - (log((double)sum) - shift * 0.693147180559945309417));
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
