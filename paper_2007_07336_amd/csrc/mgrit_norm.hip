// The norms after and before a block with its gate and residual step, and their backward pass.
#include "mgrit_epilogue.h"

namespace mgrit {

namespace {

constexpr long long MOST_ROWS = 1LL << 21;                       // of one launch: fewer than 2^32 threads

// Sums over the LANES lanes of a row, or the TH threads of a workgroup (LANES = 64); all of them get them.  sh: two places in turn (one barrier each).
template <int TH, int LANES, int N> __device__ __forceinline__ void sum_threads(float (&v)[N], float (&sh)[2][TH / 64][4], int& place) {
#pragma unroll
  for (int d = LANES / 2; d; d >>= 1)
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += __shfl_xor(v[i], d);
  if constexpr (TH > 64) {
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int i = 0; i < N; ++i) sh[place][threadIdx.x >> 6][i] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = sh[place][0][i];
#pragma unroll
    for (int w = 1; w < TH / 64; ++w)
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] += sh[place][w][i];
    place ^= 1;
  }
}
// Rows that are hard for floats are found by the mean square m of their deviations, and taken once more then.
// Deviations from a mean that is far larger than they are: as a float that is a few ulps off, which may be as much as a deviation (of 10000.1 in each of 500 features
// an ulp or two: 0.89 of a deviation with eps = 1e-6).  The deviations have few bits, so their mean is exact, or nearly, and is taken off them: nothing at all is left
// where the entries are all the same.
// (Means are sums of entries times 1 / q: those of the largest floats do not overflow, those of the smallest lose half of 2^-149 an addition.  And no product that the
// compiler might take into a subtraction, where it would not be rounded, and the deviations of one entry and another would be from two means.)
__device__ __forceinline__ bool far_off(float mean, float m) { return mean * mean > 64.0f * m; }
// Deviations whose squares no float holds, or with few bits: what they are multiplied by before they are squared, 1 for most
__device__ __forceinline__ float squares_scale(float m, float eps) { return !(m < 0x1p100f) ? 0x1p-80f : m + eps < 0x1p-90f ? 0x1p96f : 1.0f; }
// The reciprocal deviation from the mean square of deviations times c, times 1 / c
__device__ __forceinline__ float reciprocal(float m, float eps, float c) { return 1.0f / sqrtf(m + eps * c * c); }
// The reciprocal deviation.  square(c): the mean square of deviations times c; refine(): takes the deviations' mean off them, and returns it
template <typename F, typename G> __device__ __forceinline__ float deviation(float mean, float eps, F square, G refine) {
  float m = square(1.0f), c = 1.0f;
  if (__builtin_expect(far_off(mean, m) || squares_scale(m, eps) != 1.0f, 0)) {
    for (int again = 0; again < 5; ++again) {
      if (far_off(mean * c, m)) {
        mean = refine();
        c = 1.0f;
      } else if (c == 1.0f && squares_scale(m, eps) != 1.0f) {
        c = squares_scale(m, eps);
      } else {
        break;
      }
      m = square(c);
    }
  }
  return c * reciprocal(m, eps, c);
}
// Eight entries of a row from column k on; zeros where there are none
template <typename T> __device__ __forceinline__ void take8(const T* p, long long k, long long q, float (&v)[8]) {
  if (k + 8 <= q) {
    load8(p + k, v);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = k + j < q ? widen(p[k + j]) : 0.0f;
  }
}
template <typename T> __device__ __forceinline__ void give8(T* p, long long k, long long q, const float (&v)[8]) {
  if (k < q) put8(p + k, v, k + 8 <= q, q - k);
}
// The same as they were loaded, to be on their way while something else is computed
template <typename T> __device__ __forceinline__ void take_raw(const T* p, long long k, long long q, Raw8<T>& v) {
  if (k + 8 <= q) {
    v.load(p + k);
  } else {
    T e[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) e[j] = k + j < q ? p[k + j] : T(0.0f);
    __builtin_memcpy(&v, e, sizeof(e));
  }
}
template <int NV> constexpr int ROUNDS = NV > 0 ? NV : 1;       // of a loop over a thread's eights that are unrolled
// d for entries that exist, zero behind them (deviations from a mean are not zero there)
__device__ __forceinline__ float there(float d, long long k, long long q) { return k < q ? d : 0.0f; }

// One row per workgroup of TH threads, or (LANES < 64) 64 / LANES rows, LANES lanes each.  NV > 0: the row's eights fit NV registers sets of each thread and are read once; NV = 0: they are read again
// for every step.  A row's entries are only ever touched by the thread that writes them, so S may take r's place and Y f's.
template <typename ST, typename FT, int TH, int NV, int LANES>
__global__ __launch_bounds__(TH) void norm_forward_kernel(BlockNormArgs a, long long first) {
  __shared__ float sh[2][TH / 64][4];
  int place = 0;
  constexpr int ROWS = LANES < 64 ? 64 / LANES : 1;
  const long long row = first + (long long)blockIdx.x * ROWS + (ROWS > 1 ? threadIdx.x / LANES : 0), q = a.q;
  const unsigned thread = ROWS > 1 ? threadIdx.x % LANES : threadIdx.x;
  if (row >= a.M) return;
  const FT* f = static_cast<const FT*>(a.f) + row * q;
  const ST* r = static_cast<const ST*>(a.r) + row * q;
  const FT* entry = a.gate_kind == MGRIT_GATE_ENTRY ? static_cast<const FT*>(a.gate) + row * q : nullptr;
  const float* feature = a.gate_kind == MGRIT_GATE_FEATURE ? static_cast<const float*>(a.gate) : nullptr;
  const int n = NV > 0 ? NV : (int)((q + 8 * TH - 1) / (8 * TH));
  constexpr int HELD = NV > 0 ? NV : 1, U = HELD;
  const float inv = 1.0f / (float)q;
  float x[HELD][8], y[HELD][8];
  auto at = [&](int i) { return ((long long)i * TH + thread) * 8; };
  if constexpr (NV > 0) {
#pragma unroll
    for (int i = 0; i < NV; ++i) take8(f, at(i), q, x[i]);
#pragma unroll
    for (int i = 0; i < NV; ++i) take8(r, at(i), q, y[i]);
  }
  // the reciprocal deviation of the row that read(i) brings into v; of NV > 0 v becomes the deviations, zeros behind the last entry, of NV = 0 the entries' own
  // are v - mean - less each time that they are read
  auto normalize = [&](auto read, float (&v)[ROUNDS<NV>][8], float& mean, float& less) {
    auto take_off = [&](float m) {
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] = there(v[i][j] - m, at(i) + j, q);
    };
    if (a.layer) {
      float s[1] = {};
#pragma unroll ROUNDS<NV>
      for (int i = 0; i < n; ++i) {
        read(i);
#pragma unroll
        for (int j = 0; j < 8; ++j) s[0] = __builtin_fmaf(NV ? v[NV ? i : 0][j] : there(v[0][j], at(i) + j, q), inv, s[0]);
      }
      sum_threads<TH, LANES>(s, sh, place);
      mean = s[0];
      take_off(mean);
    }
    auto off = [&](int i, int j) { return NV ? v[NV ? i : 0][j] : there(v[0][j] - mean - less, at(i) + j, q); };
    return deviation(mean, a.eps, [&](float c) {
      float s[1] = {};
#pragma unroll ROUNDS<NV>
      for (int i = 0; i < n; ++i) {
        read(i);
#pragma unroll
        for (int j = 0; j < 8; ++j) { const float d = off(i, j) * c; s[0] = __builtin_fmaf(d, d, s[0]); }
      }
      sum_threads<TH, LANES>(s, sh, place);
      return s[0] * inv;
    }, [&]() {
      float s[1] = {};
#pragma unroll ROUNDS<NV>
      for (int i = 0; i < n; ++i) {
        read(i);
#pragma unroll
        for (int j = 0; j < 8; ++j) s[0] += off(i, j);
      }
      sum_threads<TH, LANES>(s, sh, place);
      const float m = s[0] / (float)q;
      less += m;
      take_off(m);
      return m;
    });
  };
  float mean = 0.0f, less = 0.0f, dev = 1.0f;
  if (a.post) dev = normalize([&](int i) { if (NV == 0) take8(f, at(i), q, x[0]); }, x, mean, less);
  // y <- S
  auto stream = [&](int i) {
    const int h = NV ? i : 0;
    float g[8], w[8];
    if (NV == 0) { take8(f, at(i), q, x[0]); take8(r, at(i), q, y[0]); }
    if (a.post) take8(a.post, at(i), q, w);
    if (entry) take8(entry, at(i), q, g);
    if (feature) take8(feature, at(i), q, g);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float m = a.post ? (NV ? x[h][j] : x[0][j] - mean - less) * dev * w[j] : x[h][j];
      y[h][j] += a.scale * (entry || feature ? g[j] * m : m);
    }
  };
  if constexpr (NV > 0) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      stream(i);
#pragma unroll
      for (int j = 0; j < 8; ++j) y[i][j] = there(y[i][j], at(i) + j, q);
      give8(static_cast<ST*>(a.S) + row * q, at(i), q, y[i]);
    }
  }
  float smean = 0.0f, sless = 0.0f, sdev = 1.0f;
  if (a.pre) sdev = normalize([&](int i) { if (NV == 0) stream(i); }, y, smean, sless);
#pragma unroll U
  for (int i = 0; i < n; ++i) {
    const int h = NV ? i : 0;
    if (NV == 0) {
      stream(i);
      give8(static_cast<ST*>(a.S) + row * q, at(i), q, y[0]);
    }
    if (!a.pre) continue;
    float w[8];
    take8(a.pre, at(i), q, w);
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j] *= (NV ? y[h][j] : y[0][j] - smean - sless) * sdev;
    give8(static_cast<FT*>(a.Y) + row * q, at(i), q, w);
  }
}

// The backward pass.  With x^ the normalised rows, h the gradient by x^ and d the reciprocal deviation, the gradient by x is
// d (h - x^ mean(h x^)), with MGRIT_NORM_LAYER less mean(h) inside the brackets too.  A workgroup takes the rows b, b + G, .. and keeps the columns' sums
// of its rows in registers; they go to part[array][b][q] and are added up by a second launch.
struct ColumnSums { float* part[3]; };                           // of dw_pre, dw_post, dgate; null where not wanted
template <typename ST, typename FT, int TH, int NV, int LANES>
__global__ __launch_bounds__(TH) void norm_backward_kernel(BlockNormArgs a, ColumnSums sums) {
  __shared__ float sh[2][TH / 64][4];
  int place = 0;
  const long long q = a.q;
  constexpr int ROWS = LANES < 64 ? 64 / LANES : 1;
  const unsigned thread = ROWS > 1 ? threadIdx.x % LANES : threadIdx.x;
  const long long row0 = (long long)blockIdx.x * ROWS + (ROWS > 1 ? threadIdx.x / LANES : 0), step = (long long)gridDim.x * ROWS;
  const float* feature = a.gate_kind == MGRIT_GATE_FEATURE ? static_cast<const float*>(a.gate) : nullptr;
  const bool entries = a.gate_kind == MGRIT_GATE_ENTRY, gated = entries || feature;
  const int n = NV > 0 ? NV : (int)((q + 8 * TH - 1) / (8 * TH));
  constexpr int HELD = NV > 0 ? NV : 1, U = HELD;
  const float inv = 1.0f / (float)q;
  float x[HELD][8], s[HELD][8], ds[HELD][8], h[HELD][8];         // f, S (or their deviations), the gradient by S, that by S's normalised row
  float cpre[HELD][8] = {}, cpost[HELD][8] = {}, cgate[HELD][8] = {};
  auto at = [&](int i) { return ((long long)i * TH + thread) * 8; };
  // NV = 1: the vectors stay in registers, and the next row is on its way while this one is computed (8192 x 4096 with all of it: one workgroup to a
  // compute unit; of the first form 229 us without, 172 so)
  constexpr bool AHEAD = NV == 1;
  float wpre[8] = {}, wpost[8] = {}, wfeature[8] = {}, wentry[8] = {};
  Raw8<FT> nf = {}, nY = {}, ng = {};
  Raw8<ST> nS = {}, ndS = {};
  auto fetch = [&](long long row) {
    const long long k = at(0);
    take_raw(static_cast<const FT*>(a.f) + row * q, k, q, nf);
    if (a.dS) take_raw(static_cast<const ST*>(a.dS) + row * q, k, q, ndS);
    if (entries) take_raw(static_cast<const FT*>(a.gate) + row * q, k, q, ng);
    if (!a.pre) return;
    take_raw(static_cast<const ST*>(a.r) + row * q, k, q, nS);
    take_raw(static_cast<const FT*>(a.dY) + row * q, k, q, nY);
  };
  if constexpr (AHEAD) {
    if (row0 < a.M) fetch(row0);
    if (a.pre) take8(a.pre, at(0), q, wpre);
    if (a.post) take8(a.post, at(0), q, wpost);
    if (feature) take8(feature, at(0), q, wfeature);
  }
  auto get_pre = [&](int i, float (&w)[8]) { if constexpr (AHEAD) __builtin_memcpy(w, wpre, sizeof(w)); else if (a.pre) take8(a.pre, at(i), q, w); };
  auto get_post = [&](int i, float (&w)[8]) { if constexpr (AHEAD) __builtin_memcpy(w, wpost, sizeof(w)); else if (a.post) take8(a.post, at(i), q, w); };
  for (long long row = row0; row < a.M; row += step) {
    const FT* f = static_cast<const FT*>(a.f) + row * q;
    const ST* S = static_cast<const ST*>(a.r) + row * q;
    const ST* dS = a.dS ? static_cast<const ST*>(a.dS) + row * q : nullptr;
    const FT* dY = a.dY ? static_cast<const FT*>(a.dY) + row * q : nullptr;
    const FT* entry = entries ? static_cast<const FT*>(a.gate) + row * q : nullptr;
    const bool first = row == row0;
    // means of f and S and of the deviations from them (layer); x, s become the deviations, zeros behind the last entry, or with NV = 0 each time that they are read
    float fmean = 0.0f, smean = 0.0f, fless = 0.0f, sless = 0.0f;
    auto take_off = [&](float fm, float sm) {
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          if (a.post) x[k][j] = there(x[k][j] - fm, at(k) + j, q);
          if (a.pre) s[k][j] = there(s[k][j] - sm, at(k) + j, q);
        }
    };
    auto off_f = [&](int i, int j) { return NV ? x[NV ? i : 0][j] : there(x[0][j] - fmean - fless, at(i) + j, q); };
    auto off_s = [&](int i, int j) { return NV ? s[NV ? i : 0][j] : there(s[0][j] - smean - sless, at(i) + j, q); };
    auto load = [&](int i) {
      const int k = NV ? i : 0;
      take8(f, at(i), q, x[k]);
      if (dS) take8(dS, at(i), q, ds[k]);
      if (a.pre) {
        take8(S, at(i), q, s[k]);
        take8(dY, at(i), q, h[k]);
      }
    };
    auto get_gate = [&](int i, float (&g)[8]) {
      if constexpr (AHEAD) {
#pragma unroll
        for (int j = 0; j < 8; ++j) g[j] = entries ? wentry[j] : wfeature[j];
      } else {
        if (entry) take8(entry, at(i), q, g);
        if (feature) take8(feature, at(i), q, g);
      }
    };
    if constexpr (AHEAD) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        x[0][j] = nf.at(j); s[0][j] = nS.at(j); ds[0][j] = ndS.at(j); h[0][j] = nY.at(j); wentry[j] = ng.at(j);
      }
      if (row + step < a.M) fetch(row + step);
    } else if constexpr (NV > 0) {
#pragma unroll
      for (int i = 0; i < NV; ++i) load(i);
    }
    float hmean = 0.0f;
    if (a.layer) {
      float v[3] = {};
#pragma unroll U
      for (int i = 0; i < n; ++i) {
        const int k = NV ? i : 0;
        if (NV == 0) load(i);
        float w[8];
        get_pre(i, w);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          v[0] = __builtin_fmaf(x[k][j], inv, v[0]);
          if (a.pre) { v[1] = __builtin_fmaf(s[k][j], inv, v[1]); v[2] = __builtin_fmaf(h[k][j], w[j], v[2]); }
        }
      }
      sum_threads<TH, LANES>(v, sh, place);
      if (a.post) fmean = v[0];
      if (a.pre) smean = v[1];
      hmean = v[2] * inv;
      take_off(fmean, smean);
    }
    float fdev = 1.0f, sdev = 1.0f, hs = 0.0f;
    {
      float v[3];                                                // means of (x cf)^2, (s cs)^2 and g s cs, with g the gradient by the normalised S
      auto means = [&](float cf, float cs) {
        v[0] = v[1] = v[2] = 0.0f;
#pragma unroll U
        for (int i = 0; i < n; ++i) {
          const int k = NV ? i : 0;
          if (NV == 0) load(i);
          float w[8];
          get_pre(i, w);
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float d = off_f(i, j) * cf;
            v[0] = __builtin_fmaf(d, d, v[0]);                   // (in so many words, so that a second time rounds as the first)
            if (a.pre) {
              const float e = off_s(i, j) * cs;
              v[1] = __builtin_fmaf(e, e, v[1]);
              v[2] = __builtin_fmaf(h[k][j] * w[j], e, v[2]);
            }
          }
        }
        sum_threads<TH, LANES>(v, sh, place);
#pragma unroll
        for (int i = 0; i < 3; ++i) v[i] *= inv;
      };
      means(1.0f, 1.0f);
      float cf = 1.0f, cs = 1.0f;
      auto scale_f = [&]() { return a.post ? squares_scale(v[0], a.eps) : 1.0f; };
      auto scale_s = [&]() { return a.pre ? squares_scale(v[1], a.eps) : 1.0f; };
      auto deviations = [&]() {
        if (a.post) fdev = cf * reciprocal(v[0], a.eps, cf);
        if (a.pre) {
          const float d = reciprocal(v[1], a.eps, cs);
          sdev = cs * d;
          hs = v[2] * d;
        }
      };
      deviations();
      if (__builtin_expect((a.layer && (far_off(fmean, v[0]) || far_off(smean, v[1]))) || scale_f() != 1.0f || scale_s() != 1.0f, 0)) {
        float fm = fmean, sm = smean;
        for (int again = 0; again < 6; ++again) {                // (as in `deviation`)
          if (far_off(fm * cf, v[0]) || far_off(sm * cs, v[1])) {
            float t[2] = {};
#pragma unroll U
            for (int i = 0; i < n; ++i) {
              if (NV == 0) load(i);
#pragma unroll
              for (int j = 0; j < 8; ++j) {
                t[0] += off_f(i, j);
                if (a.pre) t[1] += off_s(i, j);
              }
            }
            sum_threads<TH, LANES>(t, sh, place);
            fm = a.post ? t[0] / (float)q : 0.0f;
            sm = a.pre ? t[1] / (float)q : 0.0f;
            fless += fm;
            sless += sm;
            take_off(fm, sm);
            cf = cs = 1.0f;
          } else {
            const float nf = cf == 1.0f ? scale_f() : cf, ns = cs == 1.0f ? scale_s() : cs;
            if (nf == cf && ns == cs) break;
            cf = nf;
            cs = ns;
          }
          means(cf, cs);
        }
        deviations();
      }
    }
    // ds <- the gradient by S, h <- that by w_pre
    auto by_stream = [&](int i) {
      const int k = NV ? i : 0;
      float w[8];
      get_pre(i, w);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        float d = dS ? ds[k][j] : 0.0f;
        if (a.pre) {
          const float sn = off_s(i, j) * sdev, g = h[k][j] * w[j];
          d += sdev * (g - sn * hs - hmean);
          h[k][j] *= sn;
        }
        ds[k][j] = d;
      }
    };
    // what a block's result gets of it, dn (times w_post): x <- normalised f
    auto by_block = [&](int i, float (&dn)[8], float (&t)[8]) {
      const int k = NV ? i : 0;
      float g[8], w[8];
      get_gate(i, g);
      get_post(i, w);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        t[j] = a.scale * ds[k][j];
        dn[j] = gated ? t[j] * g[j] : t[j];
        if (a.post) {
          x[k][j] = off_f(i, j) * fdev;
          t[j] *= x[k][j] * w[j];                                // dgate
          h[k][j] = dn[j] * x[k][j];                             // dw_post
          dn[j] *= w[j];
        } else {
          t[j] *= x[k][j];
        }
      }
    };
    auto add = [&](int array, float (&c)[8], const float (&v)[8], int i) {       // column sums
      if (NV > 0) {
#pragma unroll
        for (int j = 0; j < 8; ++j) c[j] += v[j];
      } else {
        float* p = sums.part[array] + blockIdx.x * q;
        float old[8] = {};
        if (!first) take8(p, at(i), q, old);
#pragma unroll
        for (int j = 0; j < 8; ++j) old[j] += v[j];
        give8(p, at(i), q, old);
      }
    };
    float kf[2] = {};                                            // sums of dn x^ and of dn
    float dns[HELD][8];
#pragma unroll U
    for (int i = 0; i < n; ++i) {
      const int k = NV ? i : 0;
      if (NV == 0) load(i);
      by_stream(i);
      if (sums.part[0]) add(0, cpre[k], h[k], i);
      float t[8];
      by_block(i, dns[k], t);
      if (sums.part[1]) add(1, cpost[k], h[k], i);
      if (sums.part[2]) add(2, cgate[k], t, i);
      if (entries && a.dgate) give8(static_cast<FT*>(a.dgate) + row * q, at(i), q, t);
      if (NV > 0 && a.dr) give8(static_cast<ST*>(a.dr) + row * q, at(i), q, ds[k]);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        kf[0] += there(dns[k][j] * x[k][j], at(i) + j, q);
        kf[1] += there(dns[k][j], at(i) + j, q);
      }
    }
    if (a.post) sum_threads<TH, LANES>(kf, sh, place);
    const float kx = kf[0] * inv, km = a.layer ? kf[1] * inv : 0.0f;
#pragma unroll U
    for (int i = 0; i < n; ++i) {
      const int k = NV ? i : 0;
      float t[8];
      if (NV == 0) {
        load(i);
        by_stream(i);
        by_block(i, dns[0], t);
        if (a.dr) give8(static_cast<ST*>(a.dr) + row * q, at(i), q, ds[0]);
      }
      if (a.post) {
#pragma unroll
        for (int j = 0; j < 8; ++j) dns[k][j] = fdev * (dns[k][j] - x[k][j] * kx - km);
      }
      if (a.df) give8(static_cast<FT*>(a.df) + row * q, at(i), q, dns[k]);
    }
  }
  if constexpr (ROWS > 1) {          // the rows' lanes, in a fixed order
#pragma unroll
    for (int d = LANES; d < 64; d <<= 1)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        cpre[0][j] += __shfl_xor(cpre[0][j], d);
        cpost[0][j] += __shfl_xor(cpost[0][j], d);
        cgate[0][j] += __shfl_xor(cgate[0][j], d);
      }
    if (threadIdx.x >= LANES) return;
  }
  if constexpr (NV > 0) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      if (sums.part[0]) give8(sums.part[0] + blockIdx.x * q, at(i), q, cpre[i]);
      if (sums.part[1]) give8(sums.part[1] + blockIdx.x * q, at(i), q, cpost[i]);
      if (sums.part[2]) give8(sums.part[2] + blockIdx.x * q, at(i), q, cgate[i]);
    }
  }
}

// out[col] = sum over the workgroups; 32 columns and 32 sets of workgroups each, blockIdx.y: the array
struct ColumnOuts { float* out[3]; };
__global__ __launch_bounds__(1024) void norm_columns_kernel(ColumnSums sums, int groups, long long q, ColumnOuts outs) {
  __shared__ float sh[32][33];
  const float* part = sums.part[blockIdx.y];
  if (!part) return;
  const int lane = threadIdx.x & 31, set = threadIdx.x >> 5;
  for (long long col0 = blockIdx.x * 32LL; col0 < q; col0 += gridDim.x * 32LL) {
    const long long col = col0 + lane;
    float s = 0.0f;
    if (col < q) {
#pragma unroll 8
      for (int g = set; g < groups; g += 32) s += part[g * q + col];
    }
    sh[set][lane] = s;
    __syncthreads();
    if (threadIdx.x < 32 && col < q) {
#pragma unroll
      for (int i = 1; i < 32; ++i) s += sh[i][lane];
      outs.out[blockIdx.y][col] = s;
    }
    __syncthreads();
  }
}

// Threads of a row, and workgroups of the backward pass: about 2048 wavefronts, which is what the compute units hold at once, and two rows each at least.  Their
// columns' sums are written and read once more (whole calls, us with 256 / 512 / 1024 / 2048 workgroups: 8192 x 4096 154 / 159 / 169 / 189, 2000 x 8192
// 133 / 142 / 162 / 208, 4000 x 1024 56 / 41 / 45 / 52, 20000 x 300 345 / 198 / 117 / 79, 21806 x 52 46 / 31 / 22 / 22).
inline int threads_of(long long q) { return q <= 512 ? 64 : q <= 2048 ? 256 : q <= 8192 ? 512 : 1024; }
inline int lanes_of(long long q) { return q <= 64 ? 8 : q <= 128 ? 16 : q <= 256 ? 32 : 64; }
int groups_of(const BlockNormArgs& a) {
  const long long sets = 64 / lanes_of(a.q), rows = (a.M + sets - 1) / sets;
  const long long most = a.q > 8192 ? 256 : 131072 / threads_of(a.q), g = rows < 256 ? rows : rows / 2 > 256 ? rows / 2 : 256;
  return (int)(g < most ? g : most);
}
inline size_t up(size_t x) { return (x + 255) / 256 * 256; }

template <typename ST, typename FT, int TH, int NV, int LANES = 64>
hipError_t forward_rows(const BlockNormArgs& a, hipStream_t s) {
  const long long rows = MOST_ROWS * (64 / LANES);
  for (long long r = 0; r < a.M; r += rows) {
    const long long n = a.M - r < rows ? a.M - r : rows;
    hipLaunchKernelGGL((norm_forward_kernel<ST, FT, TH, NV, LANES>), dim3((unsigned)((n + 64 / LANES - 1) / (64 / LANES))), dim3(TH), 0, s, a, r);
  }
  return hipGetLastError();
}
template <typename ST, typename FT>
hipError_t forward_sizes(const BlockNormArgs& a, hipStream_t s) {
  if (a.q <= 64) return forward_rows<ST, FT, 64, 1, 8>(a, s);
  if (a.q <= 128) return forward_rows<ST, FT, 64, 1, 16>(a, s);
  if (a.q <= 256) return forward_rows<ST, FT, 64, 1, 32>(a, s);
  if (a.q <= 512) return forward_rows<ST, FT, 64, 1>(a, s);
  if (a.q <= 2048) return forward_rows<ST, FT, 256, 1>(a, s);
  if (a.q <= 4096) return forward_rows<ST, FT, 512, 1>(a, s);
  if (a.q <= 8192) return forward_rows<ST, FT, 512, 2>(a, s);
  if (a.q <= 16384) return forward_rows<ST, FT, 1024, 2>(a, s);
  return forward_rows<ST, FT, 1024, 0>(a, s);
}
template <typename ST, typename FT>
hipError_t backward_sizes(const BlockNormArgs& a, const ColumnSums& c, int groups, hipStream_t s) {
#define NORM_BACKWARD(TH, NV, LANES) hipLaunchKernelGGL((norm_backward_kernel<ST, FT, TH, NV, LANES>), dim3((unsigned)groups), dim3(TH), 0, s, a, c)
  if (a.q <= 64) NORM_BACKWARD(64, 1, 8);
  else if (a.q <= 128) NORM_BACKWARD(64, 1, 16);
  else if (a.q <= 256) NORM_BACKWARD(64, 1, 32);
  else if (a.q <= 512) NORM_BACKWARD(64, 1, 64);
  else if (a.q <= 2048) NORM_BACKWARD(256, 1, 64);
  else if (a.q <= 4096) NORM_BACKWARD(512, 1, 64);
  else if (a.q <= 8192) NORM_BACKWARD(512, 2, 64);
  else NORM_BACKWARD(1024, 0, 64);
#undef NORM_BACKWARD
  return hipGetLastError();
}

}  // namespace

hipError_t launch_block_norm(const BlockNormArgs& a, hipStream_t s) {
  if (a.stype) return a.ftype ? forward_sizes<__bf16, __bf16>(a, s) : forward_sizes<__bf16, float>(a, s);
  return a.ftype ? forward_sizes<float, __bf16>(a, s) : forward_sizes<float, float>(a, s);
}
size_t block_norm_workspace(const BlockNormArgs& a) { return 3 * up((size_t)groups_of(a) * a.q * sizeof(float)); }
hipError_t launch_block_norm_backward(const BlockNormArgs& a, void* ws, hipStream_t s) {
  const int groups = groups_of(a);
  const size_t each = up((size_t)groups * a.q * sizeof(float));
  ColumnOuts outs = {{a.dpre, a.dpost, a.gate_kind == MGRIT_GATE_FEATURE ? static_cast<float*>(a.dgate) : nullptr}};
  ColumnSums sums = {};
  bool any = false;
  for (int i = 0; i < 3; ++i)
    if (outs.out[i]) { sums.part[i] = reinterpret_cast<float*>(static_cast<char*>(ws) + i * each); any = true; }
  hipError_t e;
  if (a.stype) e = a.ftype ? backward_sizes<__bf16, __bf16>(a, sums, groups, s) : backward_sizes<__bf16, float>(a, sums, groups, s);
  else e = a.ftype ? backward_sizes<float, __bf16>(a, sums, groups, s) : backward_sizes<float, float>(a, sums, groups, s);
  if (e != hipSuccess || !any) return e;
  const long long blocks = (a.q + 31) / 32;
  hipLaunchKernelGGL(norm_columns_kernel, dim3((unsigned)(blocks < 65536 ? blocks : 65536), 3), dim3(1024), 0, s, sums, groups, a.q, outs);
  return hipGetLastError();
}

}  // namespace mgrit
