// End layers: matrix products with bias, activation and residual in the epilogue, and the products and sums of their
// backward pass.  Every one of them is C[i][j] = sum_k A(i, k) B(j, k) in some order of its operands (mgrit_ops.h).
#include "mgrit_epilogue.h"

namespace mgrit {

namespace {

// Workgroups of one launch along x where there may be more than any launch takes: it has fewer than 2^32 threads, and what is beyond
// is dropped without an error
constexpr long long MOST_BLOCKS = 1LL << 22;

// ------------------------------------------------------------------------------------------ values in parts
// The parts of a value are bf16 values, each kept 2^s times as large (S0, S1, S2).  The second and the third so that they are about as large
// as the value: what is left of small values would be below bf16's range otherwise (floats below 2^-110 lost bits).  The first at one
// half: rounded up it can be past the largest float, or its product with the other operand's, where the whole value or product is not;
// and so that two products of the same scale stay in range together.  Two parts: the product of two bf16 values, which has 16
// significant bits.  Three: a float.
template <int PARTS> struct Scale;
template <> struct Scale<2> { static constexpr int S0 = -1, S1 = 8, S2 = 0; };
template <> struct Scale<3> { static constexpr int S0 = -1, S1 = 7, S2 = 16; };
__device__ __forceinline__ constexpr float two_to(int s) { return __builtin_bit_cast(float, (127 + s) << 23); }

// hi = v 2^s rounded to bf16, and what it leaves of v, 2^t times as large (nothing of an infinity or a NaN)
__device__ __forceinline__ void split2(float v, int s, int t, float* hi, float* lo) {
  const float h = widen(narrow<__bf16>(v * two_to(s)));
  *hi = h;
  *lo = fabsf(h) < INFINITY ? (v - h * two_to(-s)) * two_to(t) : 0.0f;
}

// ------------------------------------------------------------------------------------------ any size, any order
// For operands whose offsets within a tile do not fit 32 bits (rows of over a million entries, see wide_sizes); the kernels further
// down take everything else.  Tile of 64 x 64 outputs, four wavefronts with 32 x 32 of them each; slabs of the contraction go through registers (the
// next one is in flight while this one is multiplied) into LDS, rows along k.  With float operands on the float matrix
// instructions, a bf16 operand widened on the way; two bf16 operands on the bf16 ones.
constexpr int GT = 64;
template <typename CT> struct Slab;
template <> struct Slab<float> { static constexpr int BK = 32, ST = BK + 4; };
template <> struct Slab<__bf16> { static constexpr int BK = 64, ST = BK + 8; };

// Four consecutive entries along the operand's contiguous axis
template <typename T> struct Four { T v[4]; };

// One operand's slab: rows r0.. of `rows`, k0.. of Kc.  NP pieces of four per thread.
template <typename T, typename CT, bool HF, bool KSLOW>
struct Loader {
  static constexpr int BK = Slab<CT>::BK, NP = GT * BK / 4 / 256;
  const T* p;
  const T* f;
  long long ld, rows, Kc;
  bool vec;                                      // pieces lie on multiples of their size
  Four<T> a[NP], b[HF ? NP : 1];

  __device__ __forceinline__ void init(const Operand& o, long long rows_, long long Kc_) {
    p = static_cast<const T*>(o.p); f = static_cast<const T*>(o.f); ld = o.ld; rows = rows_; Kc = Kc_;
    vec = ld % 4 == 0;
  }
  // piece i of this thread: row and k of its first entry within the slab
  static __device__ __forceinline__ void where(int i, int* r, int* k) {
    const int n = threadIdx.x + i * 256;
    if (KSLOW) { *r = n % (GT / 4) * 4; *k = n / (GT / 4); }
    else       { *k = n % (BK / 4) * 4; *r = n / (BK / 4); }
  }
  __device__ __forceinline__ void load(long long r0, long long k0, long long kend) {
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      int r, k;
      where(i, &r, &k);
      const long long row = r0 + r, kk = k0 + k;
      const long long at = KSLOW ? kk * ld + row : row * ld + kk;
      const long long left = KSLOW ? (kk < kend ? rows - row : 0) : (row < rows ? kend - kk : 0);
      if (vec && left >= 4) {
        a[i] = *reinterpret_cast<const Four<T>*>(__builtin_assume_aligned(p + at, 4 * sizeof(T)));
        if (HF) b[HF ? i : 0] = *reinterpret_cast<const Four<T>*>(__builtin_assume_aligned(f + at, 4 * sizeof(T)));
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const bool in = j < left;
          a[i].v[j] = in ? p[at + j] : T(0.0f);
          if (HF) b[HF ? i : 0].v[j] = in ? f[at + j] : T(0.0f);
        }
      }
    }
  }
  __device__ __forceinline__ void store(CT* lds) const {
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      int r, k;
      where(i, &r, &k);
      CT v[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if constexpr (sizeof(CT) == 2) v[j] = a[i].v[j];                     // bf16 as it is
        else v[j] = HF ? widen(a[i].v[j]) * widen(b[HF ? i : 0].v[j]) : widen(a[i].v[j]);
      }
      if (KSLOW) {
#pragma unroll
        for (int j = 0; j < 4; ++j) lds[(r + j) * Slab<CT>::ST + k] = v[j];
      } else {
        Four<CT> o;
#pragma unroll
        for (int j = 0; j < 4; ++j) o.v[j] = v[j];
        *reinterpret_cast<Four<CT>*>(__builtin_assume_aligned(lds + r * Slab<CT>::ST + k, 4 * sizeof(CT))) = o;
      }
    }
  }
};

// acc += rows of As times rows of Bs over a slab
__device__ __forceinline__ void multiply_slab(const float* As, const float* Bs, int lane, floatx16& acc) {
  const int c = lane & 31, g = lane >> 5;
#pragma unroll
  for (int k = 0; k < Slab<float>::BK; k += 8) {
    // (lanes 0-31 take k .. k + 3 over four instructions, lanes 32-63 k + 4 .. k + 7: the order of a sum is free)
    const floatx4 a = *reinterpret_cast<const floatx4*>(As + c * Slab<float>::ST + k + 4 * g);
    const floatx4 b = *reinterpret_cast<const floatx4*>(Bs + c * Slab<float>::ST + k + 4 * g);
#pragma unroll
    for (int j = 0; j < 4; ++j) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(a[j], b[j], acc, 0, 0, 0);
  }
}
__device__ __forceinline__ void multiply_slab(const __bf16* As, const __bf16* Bs, int lane, floatx16& acc) {
  const int c = lane & 31, g = lane >> 5;
#pragma unroll
  for (int k = 0; k < Slab<__bf16>::BK; k += 16) {
    const bf16x8 a = *reinterpret_cast<const bf16x8*>(As + c * Slab<__bf16>::ST + k + 8 * g);
    const bf16x8 b = *reinterpret_cast<const bf16x8*>(Bs + c * Slab<__bf16>::ST + k + 8 * g);
    acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, acc, 0, 0, 0);
  }
}

// blockIdx.x: tile, behind `first` of the launches before; blockIdx.y: part of the contraction (kpart long).  One part: the epilogue here; more: sums to
// partial[part][i][j].
template <typename TA, typename TB, typename CT, bool HF, bool AS, bool BS>
__global__ __launch_bounds__(256) void product_tile_kernel(Product q, long long kpart, float* partial, int first) {
  __shared__ __attribute__((aligned(16))) CT As[GT * Slab<CT>::ST], Bs[GT * Slab<CT>::ST];
  const long long tj = (q.J + GT - 1) / GT;
  const long long L = (long long)first + logical_block(), i0 = L / tj * GT, j0 = L % tj * GT;
  const long long k0 = blockIdx.y * kpart, kend = k0 + kpart < q.Kc ? k0 + kpart : q.Kc;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), wi = wave >> 1, wj = wave & 1;
  Loader<TA, CT, HF, AS> la;
  Loader<TB, CT, false, BS> lb;
  la.init(q.A, q.I, q.Kc);
  lb.init(q.B, q.J, q.Kc);
  floatx16 acc = zero16();
  la.load(i0, k0, kend);
  lb.load(j0, k0, kend);
  for (long long k = k0; k < kend; k += Slab<CT>::BK) {
    la.store(As);
    lb.store(Bs);
    __syncthreads();
    if (k + Slab<CT>::BK < kend) {
      la.load(i0, k + Slab<CT>::BK, kend);
      lb.load(j0, k + Slab<CT>::BK, kend);
    }
    multiply_slab(As + wi * 32 * Slab<CT>::ST, Bs + wj * 32 * Slab<CT>::ST, lane, acc);
    __syncthreads();
  }
  const long long col = j0 + wj * 32 + (lane & 31);
  if (col >= q.J) return;
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    const long long row = i0 + wi * 32 + (r & 3) + 8 * (r >> 2) + 4 * (lane >> 5);
    if (row >= q.I) continue;
    const long long at = row * q.J + col;
    if (partial) partial[(long long)blockIdx.y * q.I * q.J + at] = acc[r];
    else if (q.e.otype) finish<__bf16>(q.e, at, col, acc[r]);
    else finish<float>(q.e, at, col, acc[r]);
  }
}

// The sums of the parts, and the epilogue.  SETS = 16: 64 entries per workgroup and sixteen sets of parts, where there are many
// (204 parts of 2176 entries: 82 us with one thread for an entry, which waits for one load after the other).
template <int SETS>
__global__ __launch_bounds__(SETS == 1 ? 256 : 64 * SETS) void join_parts_kernel(Epilogue e, const float* partial, int parts, long long n, long long J) {
  __shared__ float sh[SETS][64];
  constexpr int PER = SETS == 1 ? 256 : 64;
  const int set = SETS == 1 ? 0 : threadIdx.x >> 6, lane = threadIdx.x & 63;
  for (long long at0 = blockIdx.x * (long long)PER; at0 < n; at0 += gridDim.x * (long long)PER) {
    const long long at = at0 + (SETS == 1 ? (int)threadIdx.x : lane);
    float s = 0.0f;
    if (at < n) {
#pragma unroll 4
      for (int k = set; k < parts; k += SETS) s += partial[k * n + at];
    }
    if (SETS > 1) {
      sh[set][lane] = s;
      __syncthreads();
      if (set == 0)
#pragma unroll
        for (int i = 1; i < SETS; ++i) s += sh[i][lane];
      __syncthreads();
    }
    if (set == 0 && at < n) {
      if (e.otype) finish<__bf16>(e, at, at % J, s);
      else finish<float>(e, at, at % J, s);
    }
  }
}

inline long long tiles_of(const Product& q) { return (q.I + GT - 1) / GT * ((q.J + GT - 1) / GT); }
// Parts of the contraction: where the tiles do not fill the chip's 256 compute units, the sums are split so that
// about two workgroups come to each, down to 256 products a part.
int parts_of(const Product& q) {
  const long long t = tiles_of(q);
  if (t >= 256 || q.Kc < 512) return 1;
  const long long by_tiles = (512 + t - 1) / t, by_k = q.Kc / 256;
  return (int)(by_tiles < by_k ? by_tiles : by_k);
}

template <typename TA, typename TB, typename CT, bool HF, bool AS, bool BS>
hipError_t launch_tiles(const Product& q, float* partial, int parts, hipStream_t s) {
  constexpr int BK = Slab<CT>::BK;
  const long long kpart = ((q.Kc + parts - 1) / parts + BK - 1) / BK * BK;
  const long long tiles = tiles_of(q);
  for (long long b = 0; b < tiles; b += MOST_BLOCKS)
    hipLaunchKernelGGL((product_tile_kernel<TA, TB, CT, HF, AS, BS>), dim3((unsigned)(tiles - b < MOST_BLOCKS ? tiles - b : MOST_BLOCKS), (unsigned)parts), dim3(256),
                       0, s, q, kpart, parts > 1 ? partial : nullptr, (int)b);
  return hipGetLastError();
}
template <bool HF, bool AS, bool BS>
hipError_t launch_types(const Product& q, float* partial, int parts, hipStream_t s) {
  if (q.A.type && q.B.type) {
    if constexpr (!HF) return launch_tiles<__bf16, __bf16, __bf16, false, AS, BS>(q, partial, parts, s);
    else return launch_tiles<__bf16, __bf16, float, true, AS, BS>(q, partial, parts, s);
  }
  if (q.A.type) return launch_tiles<__bf16, float, float, HF, AS, BS>(q, partial, parts, s);
  if (q.B.type) return launch_tiles<float, __bf16, float, HF, AS, BS>(q, partial, parts, s);
  return launch_tiles<float, float, float, HF, AS, BS>(q, partial, parts, s);
}

hipError_t join_parts(const Product& q, const float* partial, int parts, hipStream_t s) { return mgrit::join_parts(q.e, partial, parts, q.I, q.J, s); }
// (for operands beyond the 32-bit offsets of the tiles below)
hipError_t launch_any_product(const Product& q, void* ws, hipStream_t s) {
  const int parts = parts_of(q);
  float* partial = static_cast<float*>(ws);
  hipError_t e;
  if (!q.A.kslow && !q.B.kslow) e = launch_types<false, false, false>(q, partial, parts, s);
  else if (!q.A.kslow) e = q.A.f ? launch_types<true, false, true>(q, partial, parts, s) : launch_types<false, false, true>(q, partial, parts, s);
  else e = q.A.f ? launch_types<true, true, true>(q, partial, parts, s) : launch_types<false, true, true>(q, partial, parts, s);
  return e != hipSuccess || parts == 1 ? e : join_parts(q, partial, parts, s);
}

// ------------------------------------------------------------------------------------------ few rows on one side
// At most 64 rows of one operand (the few) against many of the other (the stream), both with k contiguous: a head's classes, or a
// serving batch on wide weights.  Bound by reading the stream once: a workgroup has SB blocks of 16 stream rows and all of the
// few's, its wavefronts share the contraction, each with slabs of its own in LDS, D of them in flight, and no barrier but the one
// before the sums.  Through LDS because the 16 x 16 matrix instructions want 16 rows in 16 consecutive lanes, and loads are only
// fast if consecutive lanes read one row (64 rows x 4096 x 4096 bf16: 62 cache accesses a load straight into registers, 22 us; so 11.4).
// One row on 32768 x 4096 bf16 weights: 268 MB in 40 us.
// Rows that are no multiples of 16 bytes, and what is left of the contraction, go straight into registers all the same.
template <typename T, typename CT> struct Row8;                  // eight k of a row
template <> struct Row8<__bf16, __bf16> {
  bf16x8 v;
  __device__ __forceinline__ void load(const __bf16* p) { v = *reinterpret_cast<const bf16x8u*>(p); }
  __device__ __forceinline__ void load(const __bf16* p, long long n) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = j < n ? p[j] : __bf16(0.0f);
  }
  __device__ __forceinline__ bf16x8 all() const { return v; }
};
template <> struct Row8<__bf16, float> : Row8<__bf16, __bf16> {
  __device__ __forceinline__ float at(int j) const { return widen(v[j]); }
};
template <> struct Row8<float, float> {
  floatx4 v[2];
  __device__ __forceinline__ void load(const float* p) {
    v[0] = *reinterpret_cast<const floatx4u*>(p);
    v[1] = *reinterpret_cast<const floatx4u*>(p + 4);
  }
  __device__ __forceinline__ void load(const float* p, long long n) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j / 4][j % 4] = j < n ? p[j] : 0.0f;
  }
  __device__ __forceinline__ float at(int j) const { return v[j / 4][j % 4]; }
};
__device__ __forceinline__ void multiply16(const Row8<__bf16, __bf16>& a, const Row8<__bf16, __bf16>& b, floatx4& c) {
  c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.all(), b.all(), c, 0, 0, 0);
}
template <typename A, typename B> __device__ __forceinline__ void multiply16(const A& a, const B& b, floatx4& c) {
#pragma unroll
  for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.at(j), b.at(j), c, 0, 0, 0);
}

// A slab of 16 rows in LDS: panels of 128 bytes a row, 16-byte pieces in the order piece ^ (row / 2 & 7).  Eight k of a row:
// step `st` of 32 k, quarter g.
template <typename T, typename CT> __device__ __forceinline__ void from_slab(Row8<T, CT>& r, const unsigned char* block, int st, int r16, int g) {
  const int turn = (r16 >> 1) & 7;
  if constexpr (sizeof(T) == 2) {
    r.v = *reinterpret_cast<const bf16x8*>(block + r16 * 128 + (((st * 4 + g) ^ turn) << 4));
  } else {
    block += st * 2048 + r16 * 128;
    r.v[0] = *reinterpret_cast<const floatx4*>(block + (((2 * g) ^ turn) << 4));
    r.v[1] = *reinterpret_cast<const floatx4*>(block + (((2 * g + 1) ^ turn) << 4));
  }
}
template <typename TS, typename TF, int SB, int FB> struct FewShape {
  static constexpr int K = sizeof(TS) == 2 || sizeof(TF) == 2 ? 64 : 32;       // of a slab
  static constexpr int PS = K * (int)sizeof(TS) / 128, PF = K * (int)sizeof(TF) / 128, SLAB = (SB * PS + FB * PF) * 2048;   // panels; bytes
  // two blocks of stream rows are taken where there are many workgroups: two of them share a compute unit then, if they fit
  static constexpr int ROOM = (SB == 2 && 4 * 2 * SLAB <= 76 * 1024 ? 76 : 160) * 1024, W = 8 * 2 * SLAB <= ROOM ? 8 : 4 * 2 * SLAB <= ROOM ? 4 : 2;     // wavefronts
  static constexpr int FIT = ROOM / (W * SLAB), D = FIT > 4 ? 4 : FIT;         // slabs
  static_assert(D >= 2, "two slabs in turn");
};

// first: workgroups of the launches before.  SWAP: the stream is A (out's rows), the few are B (out's columns); otherwise the other way round.
template <typename TS, typename TF, typename CT, int SB, int FB, bool SWAP>
__global__ __launch_bounds__((64 * FewShape<TS, TF, SB, FB>::W)) void product_few_kernel(Product q, long long kpart, float* partial, int slabs_in_lds, int first) {
  typedef FewShape<TS, TF, SB, FB> Sh;
  constexpr int NS = SB * 16, NF = FB * 16, PITCH = SWAP ? NF + 1 : NS + 4, U = FB >= 4 ? 1 : 2, FEW_WAVES = Sh::W;
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  float* sums = reinterpret_cast<float*>(lds);
  constexpr int SUMS = (SWAP ? NS : NF) * PITCH;                               // of one wavefront
  static_assert(FEW_WAVES * SUMS * 4 <= Sh::W * Sh::SLAB * Sh::D, "the sums take the slabs' place");
  const Operand &so = SWAP ? q.A : q.B, &fo = SWAP ? q.B : q.A;
  const long long ns = SWAP ? q.I : q.J, nf = SWAP ? q.J : q.I, s0 = ((long long)first + logical_block()) * NS;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), r16 = lane & 15, k8 = (lane >> 4) * 8;
  const long long p0 = blockIdx.y * kpart, p1 = p0 + kpart < q.Kc ? p0 + kpart : q.Kc;
  const long long kw = ((p1 - p0 + FEW_WAVES - 1) / FEW_WAVES + 31) / 32 * 32;
  long long k = p0 + wave * kw;
  const long long kend = k + kw < p1 ? k + kw : p1;
  const TS* ps[SB];
  const TF* pf[FB];
#pragma unroll
  for (int i = 0; i < SB; ++i) { const long long r = s0 + i * 16 + r16; ps[i] = static_cast<const TS*>(so.p) + (r < ns ? r : ns - 1) * so.ld + k8; }
#pragma unroll
  for (int i = 0; i < FB; ++i) { const long long r = i * 16 + r16; pf[i] = static_cast<const TF*>(fo.p) + (r < nf ? r : nf - 1) * fo.ld + k8; }
  floatx4 acc[SB][FB];
#pragma unroll
  for (int i = 0; i < SB; ++i)
#pragma unroll
    for (int j = 0; j < FB; ++j) acc[i][j] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
  if (slabs_in_lds) {
    // (offsets from the first row of the workgroup and of the few; instruction h of a block takes its rows 8 h .. 8 h + 7)
    int offS[SB][2], offF[FB][2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int r = 8 * h + (lane >> 3), piece = ((lane & 7) ^ ((r >> 1) & 7)) * 16;
#pragma unroll
      for (int i = 0; i < SB; ++i) offS[i][h] = (int)((s0 + i * 16 + r < ns ? i * 16 + r : ns - 1 - s0) * so.ld * (int)sizeof(TS)) + piece;
#pragma unroll
      for (int j = 0; j < FB; ++j) offF[j][h] = (int)((j * 16 + r < nf ? j * 16 + r : nf - 1) * fo.ld * (int)sizeof(TF)) + piece;
    }
    const char* baseS = static_cast<const char*>(so.p) + s0 * so.ld * (int)sizeof(TS);
    const char* baseF = static_cast<const char*>(fo.p);
    const int n = kend > k ? (int)((kend - k) / Sh::K) : 0;
    const unsigned mine = (unsigned)(unsigned long long)(LdsPtr*)lds + wave * Sh::D * Sh::SLAB;
    const unsigned char* my = lds + wave * Sh::D * Sh::SLAB;
    constexpr int LOADS = 2 * (SB * Sh::PS + FB * Sh::PF);
    auto issue = [&](int t) {                       // slab t to its place
      const long long at = k + (long long)t * Sh::K;
      const unsigned to = mine + t % Sh::D * Sh::SLAB;
#pragma unroll
      for (int i = 0; i < SB; ++i)
#pragma unroll
        for (int x = 0; x < Sh::PS; ++x)
#pragma unroll
          for (int h = 0; h < 2; ++h) to_lds(baseS, offS[i][h], (int)(at * (int)sizeof(TS)) + x * 128, 0xffffffffu, to + (i * Sh::PS + x) * 2048 + h * 1024);
#pragma unroll
      for (int j = 0; j < FB; ++j)
#pragma unroll
        for (int x = 0; x < Sh::PF; ++x)
#pragma unroll
          for (int h = 0; h < 2; ++h)
            to_lds(baseF, offF[j][h], (int)(at * (int)sizeof(TF)) + x * 128, 0xffffffffu, to + ((SB * Sh::PS) + j * Sh::PF + x) * 2048 + h * 1024);
    };
    if (n > 0) {
#pragma unroll
      for (int t = 0; t < Sh::D - 1; ++t)
        if (t < n) issue(t);
      for (int t = 0; t < n; ++t) {
        // what was read from the place that is filled next has arrived; then all but the last D - 1 slabs' loads (near the end: all)
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (t + Sh::D - 1 < n) {
          issue(t + Sh::D - 1);
          asm volatile("s_waitcnt vmcnt(%0)" :: "n"(LOADS * (Sh::D - 1)) : "memory");
        } else {
          asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        }
        const unsigned char* slab = my + t % Sh::D * Sh::SLAB;
#pragma unroll
        for (int st = 0; st < Sh::K / 32; ++st) {
          Row8<TS, CT> a[SB];
          Row8<TF, CT> b[FB];
#pragma unroll
          for (int i = 0; i < SB; ++i) from_slab(a[i], slab + i * Sh::PS * 2048, st, r16, lane >> 4);
#pragma unroll
          for (int j = 0; j < FB; ++j) from_slab(b[j], slab + (SB * Sh::PS + j * Sh::PF) * 2048, st, r16, lane >> 4);
#pragma unroll
          for (int i = 0; i < SB; ++i)
#pragma unroll
            for (int j = 0; j < FB; ++j) multiply16(a[i], b[j], acc[i][j]);
        }
      }
      k += (long long)n * Sh::K;
    }
  }
  // two sets of registers: one is on its way while the other is multiplied
  Row8<TS, CT> a[2][U][SB];
  Row8<TF, CT> b[2][U][FB];
  auto load = [&](int set, long long at) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
      for (int i = 0; i < SB; ++i) a[set][u][i].load(ps[i] + at + 32 * u);
#pragma unroll
      for (int j = 0; j < FB; ++j) b[set][u][j].load(pf[j] + at + 32 * u);
    }
  };
  auto multiply = [&](int set) {
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < SB; ++i)
#pragma unroll
        for (int j = 0; j < FB; ++j) multiply16(a[set][u][i], b[set][u][j], acc[i][j]);
  };
  const int whole = kend > k ? (int)((kend - k) / (32 * U)) : 0;
  if (whole) load(0, k);
  int n = 0;
  for (; n + 2 <= whole; n += 2, k += 64 * U) {
    load(1, k + 32 * U);
    multiply(0);
    if (n + 2 < whole) load(0, k + 64 * U);
    multiply(1);
  }
  if (n < whole) { multiply(0); k += 32 * U; }
  for (; k < kend; k += 32) {
    const long long left = kend - k - k8;
#pragma unroll
    for (int i = 0; i < SB; ++i) a[0][0][i].load(ps[i] + k, left);
#pragma unroll
    for (int j = 0; j < FB; ++j) b[0][0][j].load(pf[j] + k, left);
#pragma unroll
    for (int i = 0; i < SB; ++i)
#pragma unroll
      for (int j = 0; j < FB; ++j) multiply16(a[0][0][i], b[0][0][j], acc[i][j]);
  }
  __syncthreads();
  // lane: row r16 of the few, four rows of the stream
#pragma unroll
  for (int i = 0; i < SB; ++i)
#pragma unroll
    for (int j = 0; j < FB; ++j)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int s = i * 16 + (lane >> 4) * 4 + r, f = j * 16 + r16;
        sums[wave * SUMS + (SWAP ? s * PITCH + f : f * PITCH + s)] = acc[i][j][r];
      }
  __syncthreads();
  for (int n = threadIdx.x; n < NS * NF; n += 64 * FEW_WAVES) {
    const int s = SWAP ? n / NF : n % NS, f = SWAP ? n % NF : n / NS;
    if (s0 + s >= ns || f >= nf) continue;
    float v = 0.0f;
#pragma unroll
    for (int w = 0; w < FEW_WAVES; ++w) v += sums[w * SUMS + (SWAP ? s * PITCH + f : f * PITCH + s)];
    const long long col = SWAP ? f : s0 + s, at = (SWAP ? s0 + s : f) * q.J + col;
    if (partial) partial[blockIdx.y * q.I * q.J + at] = v;
    else if (q.e.otype) finish<__bf16>(q.e, at, col, v);
    else finish<float>(q.e, at, col, v);
  }
}

constexpr long long FEW_MANY = 8192;
struct FewPlan {
  bool few, swap;
  int sb, fb, parts;
  long long kpart;
};
// Where one side has at most 64 rows.  Workgroups: one for 16 stream rows, from FEW_MANY of them on one for 32 (us with 16 / 32, contraction of
// 4096: 64 rows on 4096 bf16 11.4 / 16.3, on 8192 20 / 16, on 32768 76 / 58; one row on 4096 8.7 / 11.6, on 8192 13.7 / 12.4, on 32768 45 / 39).
// The contraction is shared between workgroups where there are fewer than one for each of the 256 compute units, to about two for each, down
// to 1024 a part (128 for each wavefront where there are eight).
FewPlan few_plan(const Product& q) {
  FewPlan p = {};
  const long long few = q.I < q.J ? q.I : q.J, many = q.I < q.J ? q.J : q.I;
  p.few = !q.A.kslow && !q.B.kslow && !q.A.f && few <= 64 && many <= (1LL << 31);
  if (!p.few) return p;
  p.swap = q.I >= q.J;
  p.fb = few <= 16 ? 1 : few <= 32 ? 2 : 4;
  p.sb = many >= FEW_MANY ? 2 : 1;
  const long long wgs = (many + 16 * p.sb - 1) / (16 * p.sb);
  long long parts = wgs >= 256 ? 1 : (512 + wgs - 1) / wgs;
  if (parts > q.Kc / 1024) parts = q.Kc / 1024 > 1 ? q.Kc / 1024 : 1;
  p.kpart = ((q.Kc + parts - 1) / parts + 31) / 32 * 32;
  p.parts = (int)((q.Kc + p.kpart - 1) / p.kpart);
  return p;
}
template <typename TS, typename TF, typename CT, int SB, int FB, bool SWAP>
hipError_t launch_few_kernel(const Product& q, const FewPlan& p, float* partial, hipStream_t s) {
  typedef FewShape<TS, TF, SB, FB> Sh;
  static LdsOptIn opt;
  const long long many = SWAP ? q.I : q.J;
  const size_t smem = Sh::W * Sh::D * Sh::SLAB;
  const hipError_t e = opt.raise(reinterpret_cast<const void*>(&product_few_kernel<TS, TF, CT, SB, FB, SWAP>), smem);
  if (e != hipSuccess) return e;
  // (16-byte pieces of rows; offsets within the few's 64 rows and along a row are 31 bits)
  const Operand &so = SWAP ? q.A : q.B, &fo = SWAP ? q.B : q.A;
  const int in_lds = so.ld * sizeof(TS) % 16 == 0 && fo.ld * sizeof(TF) % 16 == 0 && q.Kc <= (1LL << 22);
  const long long blocks = (many + 16 * SB - 1) / (16 * SB);
  for (long long b = 0; b < blocks; b += MOST_BLOCKS)
    hipLaunchKernelGGL((product_few_kernel<TS, TF, CT, SB, FB, SWAP>), dim3((unsigned)(blocks - b < MOST_BLOCKS ? blocks - b : MOST_BLOCKS), (unsigned)p.parts),
                       dim3(64 * Sh::W), smem, s, q, p.kpart, p.parts > 1 ? partial : nullptr, in_lds, (int)b);
  return hipGetLastError();
}
template <typename TS, typename TF, typename CT, int SB, int FB>
hipError_t launch_few_swap(const Product& q, const FewPlan& p, float* partial, hipStream_t s) {
  return p.swap ? launch_few_kernel<TS, TF, CT, SB, FB, true>(q, p, partial, s) : launch_few_kernel<TS, TF, CT, SB, FB, false>(q, p, partial, s);
}
template <typename TS, typename TF, typename CT>
hipError_t launch_few_sizes(const Product& q, const FewPlan& p, float* partial, hipStream_t s) {
  if (p.sb == 2) return p.fb == 1 ? launch_few_swap<TS, TF, CT, 2, 1>(q, p, partial, s)
                      : p.fb == 2 ? launch_few_swap<TS, TF, CT, 2, 2>(q, p, partial, s) : launch_few_swap<TS, TF, CT, 2, 4>(q, p, partial, s);
  return p.fb == 1 ? launch_few_swap<TS, TF, CT, 1, 1>(q, p, partial, s)
       : p.fb == 2 ? launch_few_swap<TS, TF, CT, 1, 2>(q, p, partial, s) : launch_few_swap<TS, TF, CT, 1, 4>(q, p, partial, s);
}
hipError_t launch_few(const Product& q, const FewPlan& p, float* partial, hipStream_t s) {
  const int ts = p.swap ? q.A.type : q.B.type, tf = p.swap ? q.B.type : q.A.type;
  if (ts && tf) return launch_few_sizes<__bf16, __bf16, __bf16>(q, p, partial, s);
  if (ts) return launch_few_sizes<__bf16, float, float>(q, p, partial, s);
  if (tf) return launch_few_sizes<float, __bf16, float>(q, p, partial, s);
  return launch_few_sizes<float, float, float>(q, p, partial, s);
}

// ------------------------------------------------------------------------------------------ thin gradients
// The backward pass where G has at most 16 columns (a head's classes) or rows (samples): both of its products in one pass over
// the large operand S, whose rows go with G's long side:
//   outS[r][k] = sum_t G(r, t) T[t][k],   outT[t][k] = sum_r G(r, t) S[r][k]
// (few classes: S = X, T = W, outS = dX, outT = dW; few samples: S = W, T = X, outS = dW, outT = dX).  With few of them bound by reading S and
// writing outS (2 samples on 39889 x 1088 float: 348 MB in 82 us, 4.2 TB/s).  With many by the wavefronts' own work and waits, 2 NT
// multiplications for each entry of S: 8192 samples x 4096, 16 classes, float is 268 MB in 94 us, 2.9 TB/s, the vector units busy 40 % of the time and
// the wavefronts waiting half of theirs, with 1024 workgroups where 768 fit at once.  32 x 65536, 10 classes: latency, 13.  Workgroup: 256 k by a chunk of
// rows, a wavefront every fourth row; a lane has four k of all of T and of outT in registers, G lies in LDS.
template <typename T> struct __attribute__((packed, aligned(sizeof(T)))) Any4 { T v[4]; };
template <typename T> __device__ __forceinline__ floatx4 load4(const T* p, long long n) {       // n of them exist
  floatx4 r = {0.0f, 0.0f, 0.0f, 0.0f};
  if (n >= 4) {
    const Any4<T> a = *reinterpret_cast<const Any4<T>*>(p);
#pragma unroll
    for (int j = 0; j < 4; ++j) r[j] = widen(a.v[j]);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (j < n) r[j] = widen(p[j]);
  }
  return r;
}
template <typename T> __device__ __forceinline__ void store4(T* p, floatx4 v, long long n) {
  if (n >= 4) {
    Any4<T> a;
#pragma unroll
    for (int j = 0; j < 4; ++j) a.v[j] = narrow<T>(v[j]);
    *reinterpret_cast<Any4<T>*>(p) = a;
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (j < n) p[j] = narrow<T>(v[j]);
  }
}
// X in 8 bits: four entries from a multiple of 4 on are within a block, whose scale lies with its slab's
struct Mx8 {};
typedef float floatx2p __attribute__((ext_vector_type(2)));
__device__ __forceinline__ float scale8(const Packed& p, long long row, long long k) {
  const int block = (int)(k >> 5) & 7;
  const unsigned byte = p.scales[((k >> 8) * p.rows + row) * 8 + (block & 1) * 4 + (block >> 1)];
  return byte == 255u ? NAN : __builtin_bit_cast(float, byte ? byte << 23 : 0x00400000u);
}
__device__ __forceinline__ floatx4 load4(const Packed& p, long long row, long long k, long long n) {
  floatx4 r = {0.0f, 0.0f, 0.0f, 0.0f};
  if (n <= 0) return r;              // (codes behind the last column are zero)
  const unsigned c = *reinterpret_cast<const unsigned*>(p.codes + row * p.pitch + k);
  const float scale = scale8(p, row, k);
  const floatx2p a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c, 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c, 1.0f, true);
  return floatx4{a[0] * scale, a[1] * scale, b[0] * scale, b[1] * scale};
}
// Eight from a multiple of 8 on, of which `left` exist (zeros behind them, whatever the block's scale); one
__device__ __forceinline__ void load8(const Packed& p, long long row, long long k, long long left, float (&v)[8]) {
  const uint2 c = *reinterpret_cast<const uint2*>(p.codes + row * p.pitch + k);
  const float scale = scale8(p, row, k);
  const floatx2p a[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c.x, 1.0f, false), __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c.x, 1.0f, true),
                         __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c.y, 1.0f, false), __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c.y, 1.0f, true)};
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = j < left ? a[j / 2][j % 2] * scale : 0.0f;
}
__device__ __forceinline__ float load1(const Packed& p, long long row, long long k) {
  return __builtin_amdgcn_cvt_scalef32_pk_f32_fp8((unsigned)p.codes[row * p.pitch + k], 1.0f, false)[0] * scale8(p, row, k);
}
template <typename T> __device__ __forceinline__ floatx4 load4_of(const void* p, const Packed& kept, long long row, long long K, long long k, long long n) {
  if constexpr (std::is_same<T, Mx8>::value) return load4(kept, row, k, n);
  else return load4(static_cast<const T*>(p) + row * K + k, n);
}
struct ThinArgs {
  const void* S;  const void* T;  const void* g;  const void* f;
  void* outS;  void* outT;            // outT: float sums of every chunk if there are several
  float* sum;                         // db: of every chunk if there are several (few classes), or of the chunk's rows (few samples)
  long long rows, K, F;
  int nt, by_column;                  // by_column: G(r, t) = g[r F + t] (few classes), else g[t F + r] (few samples)
  int chunk, chunks;                  // rows of a workgroup, at most THIN_ROWS
  int outS_type, outT_type;
  float scale;
  Packed kept, f8;                    // S or T, whichever is Mx8; the factors, if f says that there are some and they have codes
};
constexpr int THIN_ROWS = 256;

template <typename TS, typename TT, typename TY, int NT>
__global__ __launch_bounds__(256) void thin_backward_kernel(ThinArgs a) {
  __shared__ float G[THIN_ROWS + 1][NT];         // the last row: zeros for rows behind the chunk's (x is zero there, another row's G may be infinite)
  __shared__ floatx4 half[2][NT][64];
  const long long blocks = (a.K + 255) / 256;
  const long long L = logical_block(), c = L / blocks, r0 = c * a.chunk;
  const int n = (int)(a.rows - r0 < a.chunk ? a.rows - r0 : a.chunk);
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
  const long long k = L % blocks * 256 + lane * 4, left = a.K - k;
  const TY *g = static_cast<const TY*>(a.g), *f = static_cast<const TY*>(a.f);
  // U rows are on their way while U others are multiplied
  constexpr int U = 4;
  floatx4 x[2][U];
  auto load = [&](int set, int r) {
#pragma unroll
    for (int u = 0; u < U; ++u) x[set][u] = load4_of<TS>(a.S, a.kept, r0 + r + 4 * u, a.K, k, r + 4 * u < n ? left : 0);
  };
  if (a.outT && wave < n) load(0, wave);         // (before anything is waited for)
  for (int i = t; i < n * NT; i += 256) {
    const int r = a.by_column ? i / NT : i % n, e = a.by_column ? i % NT : i / n;
    float v = 0.0f;
    if (e < a.nt) {
      const long long at = a.by_column ? (r0 + r) * a.F + e : e * a.F + r0 + r;
      if (f && a.f8.codes) v = widen(g[at]) * (a.by_column ? load1(a.f8, r0 + r, e) : load1(a.f8, e, r0 + r));
      else v = f ? widen(g[at]) * widen(f[at]) : a.scale * widen(g[at]);
    }
    G[r][e] = v;
  }
  if (t < NT) G[THIN_ROWS][t] = 0.0f;
  floatx4 w[NT], s[NT];
#pragma unroll
  for (int e = 0; e < NT; ++e) {
    w[e] = s[e] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
    if (a.outS && e < a.nt) w[e] = load4_of<TT>(a.T, a.kept, e, a.K, k, left);
  }
  __syncthreads();
  auto multiply = [&](int set, int r) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const bool in = r + 4 * u < n;
      const float* q = G[in ? r + 4 * u : THIN_ROWS];
      if (a.outS && in) {
        floatx4 o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int e = 0; e < NT; ++e) o += q[e] * w[e];
        const long long at = (r0 + r + 4 * u) * a.K + k;
        if (a.outS_type) store4(static_cast<__bf16*>(a.outS) + at, o, left);
        else store4(static_cast<float*>(a.outS) + at, o, left);
      }
      if (a.outT) {
#pragma unroll
        for (int e = 0; e < NT; ++e) s[e] += q[e] * x[set][u];
      }
    }
  };
  for (int r = wave; r < n; r += 8 * U) {
    if (a.outT && r + 4 * U < n) load(1, r + 4 * U);
    multiply(0, r);
    if (r + 4 * U >= n) break;
    if (a.outT && r + 8 * U < n) load(0, r + 8 * U);
    multiply(1, r + 4 * U);
  }
  if (a.sum && L % blocks == 0) {
    if (a.by_column) {                 // sums of the chunk's columns
      if (t < a.nt) {
        float v = 0.0f;
        for (int r = 0; r < n; ++r) v += G[r][t];
        a.sum[c * a.F + t] = v;
      }
    } else {
      for (int r = t; r < n; r += 256) {
        float v = 0.0f;
        for (int e = 0; e < a.nt; ++e) v += G[r][e];
        a.sum[r0 + r] = v;
      }
    }
  }
  if (!a.outT) return;
  // the four wavefronts' sums, two by two
#pragma unroll
  for (int from = 2; from; from >>= 1) {
    if (wave >= from && wave < 2 * from) {
#pragma unroll
      for (int e = 0; e < NT; ++e) half[wave - from][e][lane] = s[e];
    }
    __syncthreads();
    if (wave < from) {
#pragma unroll
      for (int e = 0; e < NT; ++e) s[e] += half[wave][e][lane];
    }
    __syncthreads();
  }
  if (wave) return;
#pragma unroll
  for (int e = 0; e < NT; ++e) {
    const long long at = e * a.K + k;
    if (e >= a.nt) continue;
    if (a.chunks > 1) store4(static_cast<float*>(a.outT) + c * a.nt * a.K + at, s[e], left);
    else if (a.outT_type) store4(static_cast<__bf16*>(a.outT) + at, s[e], left);
    else store4(static_cast<float*>(a.outT) + at, s[e], left);
  }
}

// ------------------------------------------------------------------------------------------ large products
// Operands as planes of CT in memory, with rows of any multiple of 16 bytes, along k or with k slow, as the backward pass meets its
// operands.  What the caller has in this form is read
// in place; anything else -- ragged, with a factor, of another type -- is laid out in the workspace first, which costs a pass
// over the operand and keeps the multiplying loop free of everything but multiplications.
template <typename CT> struct Mma;
template <> struct Mma<__bf16> {
  typedef bf16x8 Frag;
  static __device__ __forceinline__ void go(Frag a, Frag b, floatx16& c) { c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};
template <> struct Mma<float> {
  typedef floatx4 Frag;       // (lanes 0-31 take four k, lanes 32-63 the next four, one each per instruction)
  static __device__ __forceinline__ void go(Frag a, Frag b, floatx16& c) {
#pragma unroll
    for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[j], b[j], c, 0, 0, 0);
  }
};

struct Plane {
  const char* p;
  long long ld;                // bytes from row to row (k slow: from k to k)
  long long part;              // bytes from part to part
  int row;                     // bytes of a row that count: zeros from there on (not with k slow)
};
struct WideArgs {
  Plane A, B;
  Epilogue e;
  long long I, J, Kc;
  int slabs;                   // of the contraction
  int passes;                  // pairs of parts that are multiplied
  unsigned partA, partB;       // of pass s: bits 4 s .. 4 s + 3
  unsigned scales;             // of pass s: its products are 2^(n - 2) times as large, n in bits 5 s .. 5 s + 4
  int per;                     // slabs that one workgroup takes, in all passes
  float* partial;              // several workgroups: their sums
};

// One operand's way into LDS and registers.  A slab is SLAB bytes of LDS, either BT rows of 128 bytes along k or 128 / sizeof(CT) rows
// of BT entries.  The hardware writes LDS in lane order, so the lanes pick their 16-byte pieces from memory in the order that
// spreads the later reads over the banks: along k, piece ^ (row / 2 & 7), so that sixteen rows' pieces of one k meet different banks;
// with k slow, the four rows that a transposing read takes from (bf16), or the two that the wavefront's halves take (float), lie
// 64 or 128 bytes apart.
template <typename CT, int BT, bool KS>
struct Stream {
  typedef typename Mma<CT>::Frag Frag;
  static constexpr int ES = sizeof(CT), T = BT / 64, NL = BT / 32, KSLAB = 128 / ES, ROW = BT * ES;   // ROW: bytes of a row with k slow
  static constexpr int SLAB = BT * 128;
  const char* base;            // of the next slab to load
  long long room;              // bytes from there to the end (k slow)
  int along, offset[NL], piece[2], row;          // piece: byte of the row's slab that this lane asks for in even and odd loads
  int at[KS ? T : 4];          // where this lane reads: per tile (k slow) or per step

  // which pieces of row k change places (k slow)
  static __device__ __forceinline__ int turn(int k) { return ES == 4 ? (k >> 2 & 1) << 3 : BT == 64 ? (k >> 1 & 1) << 2 : (k & 3) << 2; }
  // rows r0.. of `rows`; skip: slabs before the first one; side: which half of the tile this wavefront reads
  __device__ __forceinline__ void init(const Plane& p, long long r0, long long rows, long long Kc, int part, int skip, int wave, int lane, int side) {
    const int c = lane & 31, g = lane >> 5;
    if constexpr (KS) {
      base = p.p + part * p.part + r0 * ES + (long long)skip * KSLAB * p.ld;
      room = Kc * p.ld - r0 * ES - (long long)skip * KSLAB * p.ld;
      along = 0;
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        const int byte = (wave * NL + i) * 1024 + lane * 16, k = byte / ROW, piece = byte % ROW / 16;
        const int from = piece ^ turn(k);
        offset[i] = (int)(k * p.ld) + from * 16;
      }
#pragma unroll
      for (int i = 0; i < T; ++i) {
        const int first = side * (BT / 2) + i * 32;
        if (ES == 2) {
          const int l16 = lane & 15, k = 8 * g + (l16 >> 2), col = first + 16 * (c >> 4) + 4 * (l16 & 3);
          at[i] = k * ROW + (((col >> 3) ^ turn(k)) << 4) + (col & 7) * 2;
        } else {
          const int col = first + c;
          at[i] = 4 * g * ROW + (((col >> 2) ^ turn(4 * g)) << 4) + (col & 3) * 4;
        }
      }
    } else {
      base = p.p + part * p.part + r0 * p.ld;
      along = skip * 128;
      row = p.row;
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        const int r = wave * (BT / 4) + i * 8 + (lane >> 3);
        piece[i & 1] = ((lane & 7) ^ ((r >> 1) & 7)) * 16;       // (the same for every second load)
        offset[i] = (int)((r0 + r < rows ? r : rows - 1 - r0) * p.ld) + piece[i & 1];
      }
#pragma unroll
      for (int step = 0; step < 4; ++step) at[step] = (side * (BT / 2) + c) * 128 + (((2 * step + g) ^ ((c >> 1) & 7)) << 4);
    }
  }
  __device__ __forceinline__ void load(int i, unsigned slab, int wave) const {
    // (rows along k: offsets stay below 2^31 - 2^16, see wide_sizes; a piece behind the row's end is asked for from further on.  Tiles of
    // 256 have whole slabs only: these two instructions for a load cost them 2 %)
    const unsigned most = KS ? 0xffffffffu : 0x7fff0000u;
    const int from = KS || BT == 256 || along + piece[i & 1] < row ? offset[i] : 0x7ffffff0;
    to_lds(base, from, along, KS && room < (long long)most ? (unsigned)room : most, slab + (wave * NL + i) * 1024);
  }
  __device__ __forceinline__ void next(const Plane& p) {
    if (KS) { base += KSLAB * p.ld; room -= KSLAB * p.ld; }
    else along += 128;
  }
  // back by `slabs`, and `parts` parts further
  __device__ __forceinline__ void again(const Plane& p, int slabs, int parts) {
    if (KS) { base -= (long long)slabs * KSLAB * p.ld; room += (long long)slabs * KSLAB * p.ld; }
    else along -= slabs * 128;
    base += parts * p.part;
  }
  // fragment of tile i in step `step`
  __device__ __forceinline__ Frag read(const unsigned char* slab, int step, int i) const {
    if constexpr (!KS) {
      return *reinterpret_cast<const Frag*>(slab + at[step] + i * 32 * 128);
    } else if constexpr (ES == 2) {
      // a sixteenth of the wavefront hands in 4 k x 16 rows and each lane gets four k of its row
      typedef __attribute__((address_space(3))) short4v* Lds4;
      const unsigned char* q = slab + at[i] + step * 16 * ROW;
      const bf16x4 lo = __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds4)(q)));
      const bf16x4 hi = __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds4)(q + 4 * ROW)));
      return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    } else {
      const unsigned char* q = slab + at[i] + step * 8 * ROW;
      Frag f;
#pragma unroll
      for (int j = 0; j < 4; ++j) f[j] = *reinterpret_cast<const float*>(q + j * ROW);
      return f;
    }
  }
};

// Tile of BT x BT outputs, four wavefronts with a quarter each.  While one slab is multiplied in four steps, the next one and A's part of
// the one after that are on their way into LDS.  Behind the last step's reads a barrier says that nobody needs the old slab
// any more and that the next one has arrived.  Bound by the matrix instructions: busy 73 % of the cycles at 8192^3 bf16 (829 us, 1326
// TFLOP/s; a library's product 683), the rest at the slabs' barriers and the tiles' ends, 16 us each.
template <typename CT, int BT, typename OT, bool AS, bool BS>
__device__ __forceinline__ void product_wide(const WideArgs& a, long long L, int share, unsigned char* lds) {
  typedef typename Mma<CT>::Frag Frag;
  constexpr int T = BT / 64, NL = BT / 32, SLAB = BT * 128;       // 32 x 32 tiles along a wavefront's side; loads per operand and slab
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), wi = wave >> 1, wj = wave & 1;
  // tiles in groups of GM rows of tiles, so that the tiles that an XCD works on at a time share few panels of both operands
  constexpr int GM = 4;
  const long long ti = (a.I + BT - 1) / BT, tj = (a.J + BT - 1) / BT;
  const long long group = L / (GM * tj), first = group * GM, size = ti - first < GM ? ti - first : GM, in = L - group * GM * tj;
  const long long i0 = (first + in % size) * BT, j0 = in / size * BT;

  // Where workgroups share a tile each takes a piece of the contraction, through all passes: with a product's passes in different
  // sums, one part too many rounded up could overflow before the others come in.
  const int s0 = share * a.per, slabs = s0 + a.per < a.slabs ? a.per : a.slabs - s0, total = slabs * a.passes;
  Stream<CT, BT, AS> sa;
  Stream<CT, BT, BS> sb;
  // the pass of either operand's next slab, and its slabs that are left; parts by pass
  int passA = 0, passB = 0;
  auto part = [](unsigned parts, int pass) { return (int)(parts >> (4 * pass) & 15u); };
  sa.init(a.A, i0, a.I, a.Kc, part(a.partA, 0), s0, wave, lane, wi);
  sb.init(a.B, j0, a.J, a.Kc, part(a.partB, 0), s0, wave, lane, wj);
  int leftA = slabs, leftB = slabs;
  const unsigned lds_at = (unsigned)(unsigned long long)(LdsPtr*)lds;
  auto nextA = [&]() {
    sa.next(a.A);
    if (--leftA == 0) { leftA = slabs; sa.again(a.A, slabs, part(a.partA, passA + 1) - part(a.partA, passA)); ++passA; }
  };
  auto nextB = [&]() {
    sb.next(a.B);
    if (--leftB == 0) { leftB = slabs; sb.again(a.B, slabs, part(a.partB, passB + 1) - part(a.partB, passB)); ++passB; }
  };
  const int c = lane & 31, g = lane >> 5;
  Frag fa[2][T], fb[2][T];
  // places in LDS: three of A's slabs, then two of B's
  auto read = [&](int pa, int pb, int step, int i) {             // tile i's fragments
    fa[step & 1][i] = sa.read(lds + pa, step, i);
    fb[step & 1][i] = sb.read(lds + pb, step, i);
  };
  floatx16 acc[T][T];
#pragma unroll
  for (int i = 0; i < T; ++i)
#pragma unroll
    for (int j = 0; j < T; ++j) acc[i][j] = zero16();

  // One slab.  In every step the reads of the next one are spread over the first half of the multiplications; the order is fixed
  // in NG groups of MG multiplications.  Loads are spread over all steps, a quarter of a slab's in each, because the address unit takes 16
  // cycles for one of four wavefronts and a wavefront that waits for it multiplies nothing (all of them in two steps: 8192^3 bf16
  // 828 us): B's of the slab after the next from step 3 on, behind the barrier that frees their place, and in the next slab's
  // step 0, A's in steps 1 and 2.
  constexpr int NG = T == 1 ? 1 : 2 * T, MG = T * T / NG, HALF = NL / 2;
  int pa = 0, pb = 3 * SLAB;                                     // of the slab that is multiplied
  auto multiply = [&](auto more, auto last) {
    const int pa1 = pa == 2 * SLAB ? 0 : pa + SLAB, pa2 = pa1 == 2 * SLAB ? 0 : pa1 + SLAB, pb1 = 7 * SLAB - pb;
#pragma unroll
    for (int step = 0; step < 4; ++step) {
      // what this slab's last reads asked for, and the next slab: all loads but those of steps 1 and 2
      if (step == 3 && more) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" :: "n"(NL) : "memory");
      if (step == 3 && !more) asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
#pragma unroll
      for (int n = 0; n < NG; ++n) {
        if (n < T && !(step == 3 && last)) read(step < 3 ? pa : pa1, step < 3 ? pb : pb1, (step + 1) & 3, n);
        if (n * HALF % NG < HALF) {                               // every NG / HALF'th group: load k of the step's half
          const int k = n * HALF / NG;
          if (step == 0 && !last) sb.load(HALF + k, lds_at + pb1, wave);
          if (step == 1 && more) sa.load(k, lds_at + pa2, wave);
          if (step == 2 && more) sa.load(HALF + k, lds_at + pa2, wave);
          if (step == 3 && more) sb.load(k, lds_at + pb, wave);
        }
#pragma unroll
        for (int k = 0; k < MG; ++k) {
          const int m = n * MG + k;
          Mma<CT>::go(fb[step & 1][m % T], fa[step & 1][m / T], acc[m / T][m % T]);     // (B first: see the end)
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      if (step == 0 && !last) nextB();
      if (step == 2 && more) nextA();
    }
    pa = pa1;
    pb = pb1;
  };
  constexpr std::true_type yes{};
  constexpr std::false_type no{};
#pragma unroll
  for (int i = 0; i < NL; ++i) { sa.load(i, lds_at, wave); sb.load(i, lds_at + 3 * SLAB, wave); }
  nextA();
  nextB();
  if (total > 1) {
#pragma unroll
    for (int i = 0; i < NL; ++i) sa.load(i, lds_at + SLAB, wave);
#pragma unroll
    for (int i = 0; i < HALF; ++i) sb.load(i, lds_at + 4 * SLAB, wave);
    nextA();
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" :: "n"(NL + HALF) : "memory");
  } else {
    asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
  }
#pragma unroll
  for (int i = 0; i < T; ++i) read(pa, pb, 0, i);
  // Passes come in the order of their scale, the largest first, and the sums are brought to that of the next pass where it is another,
  // at last to 1: exact, and every bit of a float arrives (4096 x 1024 x 4096 float rows on bf16
  // weights 107 us without, 112 so; two float operands 186 and 190).
  int pass = 0, left = slabs;                                     // of the slab that is multiplied, and how many of it are left
  auto scale_of = [&](int p) { return (int)(a.scales >> (5 * p) & 31u) - 2; };
  auto shrink = [&](int by) {
    if (by == 0) return;
    const float f = two_to(-by);
    // Where all accumulation registers are taken the compiler moves them to vector registers at once, and that through memory; so in
    // assembly, four at a time.  It does not see to the waits there: they stand before the first and behind the last.
    if constexpr (T == 4) asm volatile("s_nop 15\n\ts_nop 7" ::: "memory");
#pragma unroll
    for (int i = 0; i < T; ++i)
#pragma unroll
      for (int j = 0; j < T; ++j)
#pragma unroll
        for (int k = 0; k < 16; k += 4) {
          if constexpr (T == 4) {
            float x0 = acc[i][j][k], x1 = acc[i][j][k + 1], x2 = acc[i][j][k + 2], x3 = acc[i][j][k + 3], y0, y1, y2, y3;
            asm volatile("v_accvgpr_read_b32 %4, %0\n\tv_accvgpr_read_b32 %5, %1\n\tv_accvgpr_read_b32 %6, %2\n\tv_accvgpr_read_b32 %7, %3\n\t"
                         "v_mul_f32 %4, %8, %4\n\tv_mul_f32 %5, %8, %5\n\tv_mul_f32 %6, %8, %6\n\tv_mul_f32 %7, %8, %7\n\t"
                         "v_accvgpr_write_b32 %0, %4\n\tv_accvgpr_write_b32 %1, %5\n\tv_accvgpr_write_b32 %2, %6\n\tv_accvgpr_write_b32 %3, %7"
                         : "+a"(x0), "+a"(x1), "+a"(x2), "+a"(x3), "=&v"(y0), "=&v"(y1), "=&v"(y2), "=&v"(y3) : "v"(f));
            acc[i][j][k] = x0; acc[i][j][k + 1] = x1; acc[i][j][k + 2] = x2; acc[i][j][k + 3] = x3;
          } else {
#pragma unroll
            for (int l = 0; l < 4; ++l) acc[i][j][k + l] *= f;
          }
        }
    if constexpr (T == 4) asm volatile("s_nop 7" ::: "memory");
  };
  auto done = [&]() {
    if (--left) return;
    left = slabs;
    if constexpr (sizeof(CT) == 2) shrink(scale_of(pass) - scale_of(pass + 1));          // (float operands have one part)
    ++pass;
  };
  for (int t = 0; t < total - 2; ++t) {
    multiply(yes, no);
    done();
  }
  if (total > 1) {
    multiply(no, no);
    done();
  }
  multiply(no, yes);
  const float unscale = two_to(sizeof(CT) == 2 ? -scale_of(pass) : 0);

  // Through LDS, 32 rows of the wavefront's quarter at a time, so that a lane has eight entries of a row in its hands.  With B as the
  // instructions' first operand a lane has four consecutive columns of one row of every tile, which it writes at once.  Strips are
  // a loop, and the unrolled code of a strip's rows is one for each kind of epilogue, of which a call runs one: with everything unrolled the
  // epilogue is 300 KB of instructions, and fetching those costs more than what they do (8192 x 1024 x 4096 bf16: 109 us, a loop
  // over rows 89).  The residual of a strip's rows is asked for at once (8192 x 4096 x 4096 bf16 with tanh, residual and factors: 294 us
  // with two rows' at a time, 250 so).
  constexpr int W = BT / 2, PITCH = W + 4, STEP = 512 / W, IT = 32 / STEP;
  const int lc = lane % (W / 8) * 8, lr = lane / (W / 8);
  const long long col = j0 + wj * W + lc, n = a.I * a.J;
  const bool whole = col + 8 <= a.J, residual = a.e.fwd && a.e.R && whole;
  const bool inside = i0 + BT <= a.I && j0 + BT <= a.J && !a.partial;
  const long long row0 = i0 + wi * W + lr;
  float bias[8] = {};
  if (a.e.fwd && a.e.bias && !a.partial) {
#pragma unroll
    for (int k = 0; k < 8; ++k) bias[k] = a.e.bias[col + k < a.J ? col + k : a.J - 1];
  }
#pragma unroll 1
  for (int i = 0; i < T; ++i) {
    Raw8<OT> ahead[IT];
    if (inside && residual) {
#pragma unroll
      for (int k = 0; k < IT; ++k) ahead[k].load(static_cast<const OT*>(a.e.R) + (row0 + i * 32 + k * STEP) * a.J + col);
    }
    // (two strips in turn: what is read of one does not hold up the next one's writes)
    float* strip = reinterpret_cast<float*>(lds) + (wave * 2 + (i & 1)) * 32 * PITCH;
#pragma unroll
    for (int m = 0; m < T; ++m) {
      if (m != i) continue;                                       // (registers have no index)
#pragma unroll
      for (int j = 0; j < T; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          *reinterpret_cast<floatx4*>(strip + c * PITCH + j * 32 + 8 * q + 4 * g) =
              floatx4{acc[m][j][4 * q] * unscale, acc[m][j][4 * q + 1] * unscale, acc[m][j][4 * q + 2] * unscale, acc[m][j][4 * q + 3] * unscale};
    }
    __builtin_amdgcn_wave_barrier();
    const float* from = strip + lr * PITCH + lc;
    long long row = row0 + i * 32;
    if (inside) {
      // all rows and columns exist: the strip's rows one behind the other, the residual of all of them loaded before
      auto rows = [&](auto kind) {
        constexpr int KIND = decltype(kind)::value;
#pragma unroll
        for (int k = 0; k < IT; ++k) {
          float v[8];
          *reinterpret_cast<floatx4*>(v) = *reinterpret_cast<const floatx4*>(from + k * STEP * PITCH);
          *reinterpret_cast<floatx4*>(v + 4) = *reinterpret_cast<const floatx4*>(from + k * STEP * PITCH + 4);
          finish8_whole<OT, KIND>(a.e, (row + k * STEP) * a.J + col, v, bias, ahead[k]);
        }
      };
      if (!a.e.fwd) rows(std::integral_constant<int, PLAIN>{});
      else if (a.e.act == ACT_TANH) rows(std::integral_constant<int, ACT_TANH>{});
      else if (a.e.act == ACT_RELU) rows(std::integral_constant<int, ACT_RELU>{});
      else rows(std::integral_constant<int, ACT_IDENT>{});
    } else {
#pragma unroll 1
      for (int k = 0; k < IT; ++k, row += STEP, from += STEP * PITCH) {
        const long long at = row * a.J + col;
        if (row >= a.I) continue;
        Raw8<OT> r = {};
        if (residual && !a.partial) r.load(static_cast<const OT*>(a.e.R) + at);
        float v[8];
        *reinterpret_cast<floatx4*>(v) = *reinterpret_cast<const floatx4*>(from);
        *reinterpret_cast<floatx4*>(v + 4) = *reinterpret_cast<const floatx4*>(from + 4);
        if (a.partial) put8(a.partial + share * n + at, v, whole, a.J - col);
        else finish8<OT>(a.e, at, v, bias, r, whole, a.J - col);
      }
    }
    __builtin_amdgcn_wave_barrier();
  }
}
constexpr int wide_waves(int bt) { return bt == 256 ? 1 : bt == 128 ? 2 : 4; }          // workgroups of a compute unit
template <typename CT, int BT, typename OT, bool AS, bool BS>
__global__ __launch_bounds__(256, wide_waves(BT)) void product_wide_kernel(WideArgs a) {
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  product_wide<CT, BT, OT, AS, BS>(a, logical_block(), blockIdx.y, lds);
}
// Both products of a backward pass, where one alone leaves compute units idle: dW (w, `first` workgroups) and dX.
template <typename CT, int BT, typename OT>
__global__ __launch_bounds__(256, wide_waves(BT)) void product_pair_kernel(WideArgs w, WideArgs x, unsigned first, unsigned tiles_w, unsigned tiles_x) {
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  const unsigned b = blockIdx.x;
  if (b < first) product_wide<CT, BT, float, true, true>(w, b % tiles_w, b / tiles_w, lds);
  else product_wide<CT, BT, OT, false, true>(x, (b - first) % tiles_x, (b - first) / tiles_x, lds);
}

// Operand -> planes of CT: rows x (k padded to ldo with zeros), PARTS of them: 1 as it is (or widened); 2: the product of two bf16
// values, which has 16 significant bits, as the sum of two; 3: a float as the sum of three, all as large as Scale says
// (the bf16 instructions take subnormal values as they are).  A thread has eight columns of every eighth row of a workgroup's
// span x 256 entries.  With `sums` the columns' sums over the span as well (of the gradient, for the bias), and PARTS = 0 is
// those alone.  Bound by memory: 8192 x 4096 bf16 with factors into two parts, with sums, 268 MB in 45 us.  All that a call lays out goes in one launch, one job for each array.
struct LayJob {
  const void* p;  const void* f;
  void* out;  float* sums;
  long long rows, K, ldo;
  int span, kind;                     // kind: type + 2 * (CT is bf16) + 4 * (there are factors) + 8 * (no planes, sums only) + 16 * (p8 or f8)
  float scale;
  unsigned first;                     // workgroup
  Packed packed;                      // p (without factors) or f in 8 bits
};
struct LayJobs { LayJob j[4]; int n; };
template <typename T, typename CT, int PARTS, bool HF, bool EIGHT = false>
__device__ __forceinline__ void lay_out(const LayJob& a, unsigned block, float (&sh)[8][256]) {
  const T *p = static_cast<const T*>(a.p), *f = static_cast<const T*>(a.f);
  CT* out = static_cast<CT*>(a.out);
  const long long K = a.K, ldo = a.ldo, tiles = ((PARTS ? ldo : K) + 255) / 256, L = block - a.first, chunk = L / tiles;
  const int t = threadIdx.x;
  const long long k = L % tiles * 256 + t % 32 * 8, r0 = chunk * a.span, r1 = r0 + a.span < a.rows ? r0 + a.span : a.rows;
  const long long left = K - k;
  const bool whole = left >= 8;
  float s[8] = {};
  if (k < (PARTS ? ldo : K)) {
    for (long long r = r0 + t / 32; r < r1; r += 8) {
      const long long at = r * K + k;
      float v[8], b[8];
      if (EIGHT && !HF) {
        load8(a.packed, r, k, left, v);
      } else if (whole) {
        load8(p + at, v);
        if (HF && !EIGHT) load8(f + at, b);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          v[j] = j < left ? widen(p[at + j]) : 0.0f;
          if (HF && !EIGHT) b[j] = j < left ? widen(f[at + j]) : 0.0f;
        }
      }
      if (HF && EIGHT) load8(a.packed, r, k, left, b);       // (codes and scales reach as far as ldo)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (HF) v[j] *= b[j];
        s[j] += v[j];
      }
      if constexpr (PARTS > 0) {
        CT* o = out + r * ldo + k;
        if constexpr (PARTS >= 2) {
          float lo[8], least[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            split2(v[j], Scale<PARTS>::S0, Scale<PARTS>::S1, &v[j], &lo[j]);
            if constexpr (PARTS == 3) split2(lo[j], 0, Scale<3>::S2 - Scale<3>::S1, &lo[j], &least[j]);
          }
          store8(o + a.rows * ldo, lo);
          if (PARTS == 3) store8(o + 2 * a.rows * ldo, least);
        }
        store8(o, v);
      }
    }
  }
  if (!a.sums) return;
#pragma unroll
  for (int j = 0; j < 8; ++j) sh[t / 32][t % 32 * 8 + j] = s[j];
  __syncthreads();
  const long long col = L % tiles * 256 + t;
  if (col >= K) return;
  float x = sh[0][t];
#pragma unroll
  for (int i = 1; i < 8; ++i) x += sh[i][t];
  a.sums[chunk * K + col] = a.scale * x;
}
__global__ __launch_bounds__(256) void lay_out_kernel(LayJobs jobs, unsigned before) {
  __shared__ float sh[8][256];
  const unsigned block = before + blockIdx.x;    // of all launches
  int i = 0;
  while (i + 1 < jobs.n && block >= jobs.j[i + 1].first) ++i;
  const LayJob a = jobs.j[i];
  switch (a.kind) {
    case 0: lay_out<float, float, 1, false>(a, block, sh); break;
    case 1: lay_out<__bf16, float, 1, false>(a, block, sh); break;
    case 2: lay_out<float, __bf16, 3, false>(a, block, sh); break;
    case 3: lay_out<__bf16, __bf16, 1, false>(a, block, sh); break;
    case 4: lay_out<float, float, 1, true>(a, block, sh); break;
    case 5: lay_out<__bf16, float, 1, true>(a, block, sh); break;
    case 6: lay_out<float, __bf16, 3, true>(a, block, sh); break;
    case 7: lay_out<__bf16, __bf16, 2, true>(a, block, sh); break;
    case 8: lay_out<float, float, 0, false>(a, block, sh); break;
    case 9: lay_out<__bf16, float, 0, false>(a, block, sh); break;
    case 12: lay_out<float, float, 0, true>(a, block, sh); break;
    case 13: lay_out<__bf16, float, 0, true>(a, block, sh); break;
    case 17: lay_out<__bf16, float, 1, false, true>(a, block, sh); break;
    case 19: lay_out<__bf16, __bf16, 1, false, true>(a, block, sh); break;
    case 20: lay_out<float, float, 1, true, true>(a, block, sh); break;
    case 21: lay_out<__bf16, float, 1, true, true>(a, block, sh); break;
    case 22: lay_out<float, __bf16, 3, true, true>(a, block, sh); break;
    case 23: lay_out<__bf16, __bf16, 2, true, true>(a, block, sh); break;
    case 28: lay_out<float, float, 0, true, true>(a, block, sh); break;
    case 29: lay_out<__bf16, float, 0, true, true>(a, block, sh); break;
  }
}
// out[col] = sum over the chunks; 64 columns and sixteen sets of chunks per workgroup
__global__ __launch_bounds__(1024) void add_chunks_kernel(const float* part, int chunks, long long F, float* out) {
  __shared__ float sh[16][64];
  const int lane = threadIdx.x & 63, set = threadIdx.x >> 6;
  for (long long col0 = blockIdx.x * 64LL; col0 < F; col0 += gridDim.x * 64LL) {
    const long long col = col0 + lane;
    float s = 0.0f;
    if (col < F)
      for (int c = set; c < chunks; c += 16) s += part[c * F + col];
    sh[set][lane] = s;
    __syncthreads();
    if (set == 0 && col < F) {
#pragma unroll
      for (int i = 1; i < 16; ++i) s += sh[i][lane];
      out[col] = s;
    }
    __syncthreads();
  }
}
hipError_t add_chunks(const float* part, int chunks, long long F, float* out, hipStream_t s) {
  const long long blocks = (F + 63) / 64;
  hipLaunchKernelGGL(add_chunks_kernel, dim3((unsigned)(blocks < 65536 ? blocks : 65536)), dim3(1024), 0, s, part, chunks, F, out);
  return hipGetLastError();
}

__global__ __launch_bounds__(256) void zero_kernel(float* out, long long n) {
  for (long long i = blockIdx.x * 256LL + threadIdx.x; i < n; i += gridDim.x * 256LL) out[i] = 0.0f;
}

inline size_t up(size_t x) { return (x + 255) / 256 * 256; }

// Rows of a chunk of sums: 8, and more where that makes over 256 chunks
int sum_span(long long rows) { const long long n = (rows + 255) / 256; return (int)((n + 7) / 8 * 8); }
int chunks_of(long long rows) { const int s = sum_span(rows); return (int)((rows + s - 1) / s); }
// ... and of an array that is laid out alone: 8, up to 64 where that still makes two thousand workgroups
int lay_span(long long rows, long long tiles) {
  const long long n = rows * tiles / 2048 / 8 * 8;
  return (int)(n < 8 ? 8 : n > 64 ? 64 : n);
}

// ---- which matrix instructions, and which operands have to be laid out
// Two bf16 operands go to the bf16 instructions, and a float A against a bf16 B may if the product is large: three parts hold
// a float's 24 bits, and three passes of the bf16 instructions take less than one of the float ones, by more than the two planes' worth
// of bytes that laying it out in parts costs over widening B.
// us on the float / the bf16 instructions, float rows on bf16 weights: 256 x 1024 x 1024 18.1 / 18.0, 512 x 1024 x 1024 24.7 / 22.0, 1024^3
// 28.6 / 25.1 (with its backward pass, whose two products then no longer share a launch, 75 / 76), 4096 x 1024 x 4096 263 / 114.
constexpr double SPLIT = 1.0e9;
// Two float operands, six passes, on the float / the bf16 instructions: 2048 x 1024 x 2048 70 / 70, 2048^3 129 / 123 and its backward pass
// 258 / 228, 4096 x 1024 x 4096 273 / 195, 4096^3 936 / 656; backward of 2048 x 1000 x 1000 82 / 131.
constexpr double SPLIT2 = 6.0e9;
// Beyond these sizes the estimates of both ways decide (product_us), because parts are bytes, too: where a side is short they cost more than
// the instructions save (us on the float / the bf16 instructions: 8192 x 8192 x 100 float 142 / 305, backward of 6282 x 56 x 20295 with factors
// 640 / 1010, of 8192 x 56 x 8192 float states on bf16 weights 297 / 538, but of 8192 x 256 x 8192 float 656 / 599).
inline bool may_bf16(const Product& q) {                        // of a product whose operands are not laid out yet
  const double size = (double)q.I * (double)q.J * (double)q.Kc;
  return q.A.type ? q.B.type : size >= (q.B.type ? SPLIT : SPLIT2);
}
inline bool may_float(const Product& q) { return !q.A.type || !q.B.type; }
constexpr double COPY = 5.3e6;                                  // bytes a us that layouts and reads of whole operands reach
constexpr double AHEAD = 1.03;                                  // by which the float instructions have to be ahead, which are less exact
inline int bf16_parts(int type, const void* factors) { return type ? (factors ? 2 : 1) : 3; }
inline int slab_of(bool bf16) { return bf16 ? 64 : 32; }
// Rows along k need whole 16-byte pieces, and whole slabs where 256 x 256 tiles read them: a product with few of those takes smaller ones
// and its operands as they are (us with a copy / so: 181 x 1100 x 6311 float 52 / 41, 2000 x 1000 x 1000 bf16 18.6 / 12.6).
inline bool few_tiles(const Product& q) { return (q.I + 255) / 256 * ((q.J + 255) / 256) < 128; }
inline bool whole_slabs(const Operand& o, bool bf16) { return o.kslow || o.ld % slab_of(bf16) == 0; }
inline bool in_place(const Operand& o, bool bf16, long long Kc, bool any_pieces) {
  if (o.f || o.p8 || (o.type != 0) != bf16) return false;
  return o.ld % (bf16 ? 8 : 4) == 0 && (o.kslow || ((any_pieces || whole_slabs(o, bf16)) && (o.ld == Kc || o.padded)));
}
// The launch that lays out, as it comes together, and what it takes of the workspace
struct Layout {
  LayJobs jobs;
  char* base;
  size_t bytes;
  long long blocks;
  double moved;                       // bytes read and written

  char* take(size_t n) { char* p = base + bytes; bytes += up(n); return p; }
  // (ldo 0: no planes, sums only.  Not `out`, which may be null where sizes alone are asked for)
  void add(const void* p, const void* f, int type, bool bf16, long long rows, long long K, void* out, long long ldo, int span, float scale, float* sums,
           const Packed* packed) {
    const bool planes = ldo > 0;
    LayJob& j = jobs.j[jobs.n++];
    j = LayJob{p, f, out, sums, rows, K, ldo, span, type + 2 * (planes && bf16) + (f ? 4 : 0) + (planes ? 0 : 8) + (packed ? 16 : 0), scale, (unsigned)blocks,
               packed ? *packed : Packed{}};
    blocks += ((planes ? ldo : K) + 255) / 256 * ((rows + span - 1) / span);
    moved += (double)rows * ((double)K * (type ? 2 : 4) * (f ? 2 : 1) + (double)ldo * (bf16 ? 2 * bf16_parts(type, f) : 4));
  }
  // the operand itself, or its plane in the workspace
  Operand plane(const Operand& o, bool bf16, long long rows, long long Kc, bool any_pieces) {
    if (in_place(o, bf16, Kc, any_pieces)) return o;
    // (row length: whole slabs along k; with k slow whole 16-byte pieces, of which 8 entries are some)
    const long long m = o.kslow ? 8 : slab_of(bf16), r = o.kslow ? Kc : rows, k = o.kslow ? rows : Kc, ld = (k + m - 1) / m * m;
    Operand n = {};
    n.parts = bf16 ? bf16_parts(o.type, o.f) : 1;
    n.p = take((size_t)n.parts * r * ld * (bf16 ? 2 : 4));
    n.ld = ld; n.type = bf16; n.kslow = o.kslow; n.padded = 1; n.part = r * ld;
    add(o.p, o.f, o.type, bf16, r, k, const_cast<void*>(n.p), ld, lay_span(r, (ld + 255) / 256), 1.0f, nullptr, o.f ? o.f8 : o.p8);
    return n;
  }
  hipError_t launch(hipStream_t s) const {
    for (long long b = 0; b < blocks; b += MOST_BLOCKS)
      hipLaunchKernelGGL(lay_out_kernel, dim3((unsigned)(blocks - b < MOST_BLOCKS ? blocks - b : MOST_BLOCKS)), dim3(256), 0, s, jobs, (unsigned)b);
    return hipGetLastError();
  }
};

// ---- which tiles
// (32-bit offsets within a tile's rows, or within a slab's where k is slow; tiles of 128 and their 256 threads in one launch)
constexpr long long MOST_TILES = (1LL << 24) - 1;
inline bool wide_sizes(const Product& q) {
  const long long most = 1LL << 20;
  return (q.A.kslow ? q.I <= 4 * most : q.Kc <= most) && (q.B.kslow ? q.J <= 4 * most : q.Kc <= most) && q.Kc <= (1LL << 30) &&
         (q.I + 127) / 128 * ((q.J + 127) / 128) <= MOST_TILES;
}
struct WidePlan {
  bool bf16;
  int bt, slabs, passes, parts;       // parts: workgroups that share a tile's contraction
  size_t bytes;                       // of their sums
  double us;                          // the estimate
};
// The tile and the number of parts whose time is estimated lowest: tiles run one to a compute unit at a time or share it without
// getting faster; us for a slab by what the loop reaches (256: 1380 TFLOP/s bf16, 150 float), the start and end of a tile, and the
// launch and the traffic that join the parts.
WidePlan wide_plan(const Product& q) {
  WidePlan w = {};
  w.bf16 = q.A.type != 0;                                       // (they are planes of one type)
  w.passes = q.B.parts > 1 ? 6 : q.A.parts > 1 ? q.A.parts : 1;
  w.slabs = (int)((q.Kc + slab_of(w.bf16) - 1) / slab_of(w.bf16));
  double best = 0.0;
  for (int bt = whole_slabs(q.A, w.bf16) && whole_slabs(q.B, w.bf16) ? 256 : 128; bt >= 64; bt /= 2) {
    const long long tiles = (q.I + bt - 1) / bt * ((q.J + bt - 1) / bt);
    if (tiles > MOST_TILES) continue;
    const double slab = w.bf16 ? (bt == 256 ? 1.6 : bt == 128 ? 0.55 : 0.2) : (bt == 256 ? 7.2 : bt == 128 ? 1.9 : 0.55), ends = bt == 256 ? 6.0 : bt == 128 ? 3.0 : 2.0;
    for (int parts = 1; parts <= 32 && (parts == 1 || (parts <= w.slabs && 2 * parts <= w.slabs * w.passes && tiles * parts <= 2048)); ++parts) {
      const int piece = (w.slabs + parts - 1) / parts, per = piece * w.passes;
      if (parts > 1 && (w.slabs + piece - 1) / piece != parts) continue;
      const long long rounds = (tiles * parts + 255) / 256;
      const double join = parts > 1 ? 4.0 + (double)q.I * q.J * 4.0 * (2 * parts) / 4.0e6 : 0.0;
      const double us = (double)rounds * (per * slab + (bt == 256 ? ends : 0.0)) + (bt == 256 ? 0.0 : ends) + join;
      if (best == 0.0 || us < best) { best = us; w.bt = bt; w.parts = parts; }
    }
  }
  w.bytes = w.parts > 1 ? (size_t)w.parts * q.I * q.J * sizeof(float) : 0;
  w.us = best;
  return w;
}
// Estimated time of a product of planes, for the choice of instructions: the tiles' or that of the planes' bytes, each read once in
// every pass.  The large tiles' results are written with nothing beside them, which tells where the contraction is short.
double product_us(const Product& q) {
  const WidePlan w = wide_plan(q);
  const long long rounds = ((q.I + 255) / 256 * ((q.J + 255) / 256) * w.parts + 255) / 256;
  const double tiles = w.us + (w.bt == 256 ? 6.0 * (double)rounds : 0.0);
  const double bytes = (double)w.passes * (w.bf16 ? 2.0 : 4.0) * (double)q.Kc * (double)(q.I + q.J) / COPY;
  return tiles > bytes ? tiles : bytes;
}
double layout_us(const Layout& l) { return l.jobs.n ? 3.0 + l.moved / COPY : 0.0; }

// Room for the sums of the parts of a product whose operands are where they will be read
size_t parts_workspace(const Product& q) {
  if (wide_sizes(q)) return wide_plan(q).bytes;
  const int parts = parts_of(q);
  return parts > 1 ? (size_t)parts * (size_t)q.I * (size_t)q.J * sizeof(float) : 0;
}

template <typename CT, int BT, typename OT, bool AS, bool BS>
hipError_t launch_wide_tiles(const WideArgs& a, int parts, hipStream_t s) {
  static LdsOptIn opt;
  const size_t smem = 5 * BT * 128;
  const hipError_t e = opt.raise(reinterpret_cast<const void*>(&product_wide_kernel<CT, BT, OT, AS, BS>), smem);
  if (e != hipSuccess) return e;
  const long long tiles = (a.I + BT - 1) / BT * ((a.J + BT - 1) / BT);
  hipLaunchKernelGGL((product_wide_kernel<CT, BT, OT, AS, BS>), dim3((unsigned)tiles, (unsigned)parts), dim3(256), smem, s, a);
  return hipGetLastError();
}
template <typename CT, int BT>
hipError_t launch_wide_out(const WideArgs& a, bool as, bool bs, int parts, hipStream_t s) {
  if (as) return launch_wide_tiles<CT, BT, float, true, true>(a, parts, s);            // dW is float
  if (bs) return a.e.otype ? launch_wide_tiles<CT, BT, __bf16, false, true>(a, parts, s) : launch_wide_tiles<CT, BT, float, false, true>(a, parts, s);
  return a.e.otype ? launch_wide_tiles<CT, BT, __bf16, false, false>(a, parts, s) : launch_wide_tiles<CT, BT, float, false, false>(a, parts, s);
}

// Both operands are planes of the same type
bool ready(const Product& q) {
  const bool bf16 = q.A.type != 0;
  return q.B.type == q.A.type && in_place(q.A, bf16, q.Kc, true) && in_place(q.B, bf16, q.Kc, true);
}
WideArgs wide_args(const Product& q, const WidePlan& w, void* partial) {
  const long long es = w.bf16 ? 2 : 4;
  WideArgs a = {};
  auto plane = [&](const Operand& o) { return Plane{static_cast<const char*>(o.p), o.ld * es, o.part * es, o.kslow ? 0 : (int)(o.ld * es)}; };
  a.A = plane(q.A);
  a.B = plane(q.B);
  a.e = q.e;
  a.I = q.I; a.J = q.J; a.Kc = q.Kc;
  a.slabs = w.slabs;
  a.passes = w.passes;
  // A's parts each against B; of three parts each, the six pairs that make up a float product: the three that are left out are
  // at most 2^-23 of it together.  The smallest first: added to the sum of the large ones, each of them would round that once
  // more (1024^3 float: 6.7e-7 off with the largest first, 1.8e-7 so, the float instructions 5.7e-7).
  a.partA = w.passes == 6 ? 0x001120u : w.passes == 3 ? 0x012u : w.passes == 2 ? 0x01u : 0u;
  a.partB = w.passes == 6 ? 0x010102u : 0u;
  auto scale = [](int parts, unsigned i) {
    if (parts < 2) return 0;
    const int s[2][3] = {{Scale<2>::S0, Scale<2>::S1, Scale<2>::S2}, {Scale<3>::S0, Scale<3>::S1, Scale<3>::S2}};
    return s[parts - 2][i];
  };
  for (int i = 0; i < w.passes; ++i)
    a.scales |= (unsigned)(scale(q.A.parts, a.partA >> (4 * i) & 15u) + scale(q.B.parts, a.partB >> (4 * i) & 15u) + 2) << (5 * i);
  a.per = (w.slabs + w.parts - 1) / w.parts;
  a.partial = w.parts > 1 ? static_cast<float*>(partial) : nullptr;
  return a;
}
// The product of operands that are in place or laid out
hipError_t launch_wide_product(const Product& q, void* partial, hipStream_t s) {
  if (!ready(q)) return hipErrorInvalidValue;
  const WidePlan w = wide_plan(q);
  const WideArgs a = wide_args(q, w, partial);
  hipError_t e;
  const bool as = q.A.kslow, bs = q.B.kslow;
  if (w.bf16) e = w.bt == 256 ? launch_wide_out<__bf16, 256>(a, as, bs, w.parts, s) : w.bt == 128 ? launch_wide_out<__bf16, 128>(a, as, bs, w.parts, s)
                                                                                  : launch_wide_out<__bf16, 64>(a, as, bs, w.parts, s);
  else e = w.bt == 256 ? launch_wide_out<float, 256>(a, as, bs, w.parts, s) : w.bt == 128 ? launch_wide_out<float, 128>(a, as, bs, w.parts, s)
                                                                           : launch_wide_out<float, 64>(a, as, bs, w.parts, s);
  return e != hipSuccess || w.parts == 1 ? e : join_parts(q, a.partial, w.parts, s);
}
template <typename CT, int BT>
hipError_t launch_pair_tiles(const WideArgs& w, const WideArgs& x, int parts_w, int parts_x, hipStream_t s) {
  static LdsOptIn opt[2];
  const size_t smem = 5 * BT * 128;
  const hipError_t e = x.e.otype ? opt[1].raise(reinterpret_cast<const void*>(&product_pair_kernel<CT, BT, __bf16>), smem)
                                 : opt[0].raise(reinterpret_cast<const void*>(&product_pair_kernel<CT, BT, float>), smem);
  if (e != hipSuccess) return e;
  const unsigned tw = (unsigned)((w.I + BT - 1) / BT * ((w.J + BT - 1) / BT)), tx = (unsigned)((x.I + BT - 1) / BT * ((x.J + BT - 1) / BT));
  const dim3 grid(tw * parts_w + tx * parts_x);
  if (x.e.otype) hipLaunchKernelGGL((product_pair_kernel<CT, BT, __bf16>), grid, dim3(256), smem, s, w, x, tw * parts_w, tw, tx);
  else hipLaunchKernelGGL((product_pair_kernel<CT, BT, float>), grid, dim3(256), smem, s, w, x, tw * parts_w, tw, tx);
  return hipGetLastError();
}
// Whether both products of a backward pass go in one launch: same type, same small tiles, and fewer than four workgroups of one
// of them for a compute unit.
bool pairs(const Product& w, const Product& x) {
  const WidePlan a = wide_plan(w), b = wide_plan(x);
  const long long tw = (w.I + a.bt - 1) / a.bt * ((w.J + a.bt - 1) / a.bt) * a.parts, tx = (x.I + b.bt - 1) / b.bt * ((x.J + b.bt - 1) / b.bt) * b.parts;
  return a.bf16 == b.bf16 && a.bt == b.bt && a.bt <= 128 && (tw < 1024 || tx < 1024) && tw + tx <= MOST_TILES;
}
hipError_t launch_wide_pair(const Product& qw, const Product& qx, char* partial_w, char* partial_x, hipStream_t s) {
  if (!ready(qw) || !ready(qx)) return hipErrorInvalidValue;
  const WidePlan pw = wide_plan(qw), px = wide_plan(qx);
  const WideArgs w = wide_args(qw, pw, partial_w), x = wide_args(qx, px, partial_x);
  hipError_t e = pw.bf16 ? (pw.bt == 128 ? launch_pair_tiles<__bf16, 128>(w, x, pw.parts, px.parts, s) : launch_pair_tiles<__bf16, 64>(w, x, pw.parts, px.parts, s))
                         : (pw.bt == 128 ? launch_pair_tiles<float, 128>(w, x, pw.parts, px.parts, s) : launch_pair_tiles<float, 64>(w, x, pw.parts, px.parts, s));
  if (e == hipSuccess && pw.parts > 1) e = join_parts(qw, w.partial, pw.parts, s);
  if (e == hipSuccess && px.parts > 1) e = join_parts(qx, x.partial, px.parts, s);
  return e;
}

// Which instructions a single product takes
double forward_us(const Product& q, bool bf16) {
  Layout l = {};
  Product p = q;
  p.A = l.plane(q.A, bf16, q.I, q.Kc, few_tiles(q));
  p.B = l.plane(q.B, bf16, q.J, q.Kc, few_tiles(q));
  return layout_us(l) + product_us(p);
}
bool forward_bf16(const Product& q) {
  return may_bf16(q) && (!may_float(q) || forward_us(q, true) <= AHEAD * forward_us(q, false));
}

// ---- the backward pass: G = dY * D is laid out once for both products where a large tile reads it and it is not there already
Product input_product(const BackwardArgs& b) {
  Product q = {};
  q.A = Operand{b.dY, b.D, b.F, b.ytype, 0};
  if (b.D && b.D8.codes) q.A.f8 = &b.D8;
  q.B = Operand{b.W, nullptr, b.K, b.wtype, 1};
  q.e = Epilogue{0, 0, b.dxtype, b.scale, nullptr, nullptr, b.dX, nullptr};
  q.I = b.M; q.J = b.K; q.Kc = b.F;
  return q;
}
Product weight_product(const BackwardArgs& b) {
  Product q = {};
  q.A = Operand{b.dY, b.D, b.F, b.ytype, 1};
  q.B = Operand{b.X, nullptr, b.K, b.xtype, 1};
  if (b.X8.codes) q.B.p8 = &b.X8;
  if (b.D && b.D8.codes) q.A.f8 = &b.D8;
  q.e = Epilogue{0, 0, 0, b.scale, nullptr, nullptr, b.dW, nullptr};
  q.I = b.F; q.J = b.K; q.Kc = b.M;
  return q;
}
struct BackwardPlan {
  Product x, w;                       // with their operands where the launches find them
  Layout lay;
  float* sums;                        // of chunks of rows, for db
  int chunks;
  bool pair;                          // dW and dX in one launch
  char *partial_x, *partial_w;
  size_t bytes;
};
// Operands and layouts with the given instructions.  base: the workspace, or null for sizes alone
BackwardPlan lay_backward(const BackwardArgs& b, char* base, bool x_bf16, bool w_bf16) {
  BackwardPlan p = {};
  p.lay.base = base;
  p.x = input_product(b);
  p.w = weight_product(b);
  p.chunks = chunks_of(b.M);
  p.sums = p.chunks > 1 ? reinterpret_cast<float*>(p.lay.take((size_t)p.chunks * b.F * sizeof(float))) : b.db;
  const bool x = b.dX && wide_sizes(p.x), w = b.dW && wide_sizes(p.w);
  bool summed = !b.db;
  Operand G[2] = {};                  // [bf16]
  for (int bf16 = 0; bf16 < 2; ++bf16) {
    const bool for_x = x && x_bf16 == (bf16 != 0) && !in_place(p.x.A, bf16, p.x.Kc, few_tiles(p.x));
    const bool for_w = w && w_bf16 == (bf16 != 0) && !in_place(p.w.A, bf16, p.w.Kc, few_tiles(p.w));
    if (!for_x && !for_w) continue;
    Operand& g = G[bf16];
    const int m = slab_of(bf16);
    g.ld = (b.F + m - 1) / m * m;
    g.type = bf16; g.padded = 1; g.parts = bf16 ? bf16_parts(b.ytype, b.D) : 1; g.part = b.M * g.ld;
    g.p = p.lay.take((size_t)g.parts * g.part * (bf16 ? 2 : 4));
    p.lay.add(b.dY, b.D, b.ytype, bf16, b.M, b.F, const_cast<void*>(g.p), g.ld, summed ? lay_span(b.M, (g.ld + 255) / 256) : sum_span(b.M), b.scale,
              summed ? nullptr : p.sums, b.D && b.D8.codes ? &b.D8 : nullptr);
    summed = true;
    if (for_x) p.x.A = g;
    if (for_w) { p.w.A = g; p.w.A.kslow = 1; }
  }
  if (!summed) p.lay.add(b.dY, b.D, b.ytype, false, b.M, b.F, nullptr, 0, sum_span(b.M), b.scale, p.sums, b.D && b.D8.codes ? &b.D8 : nullptr);
  if (x) p.x.B = p.lay.plane(p.x.B, x_bf16, p.x.J, p.x.Kc, few_tiles(p.x));
  if (w) p.w.B = p.lay.plane(p.w.B, w_bf16, p.w.J, p.w.Kc, few_tiles(p.w));
  return p;
}
BackwardPlan backward_plan(const BackwardArgs& b, char* base) {
  const Product qx = input_product(b), qw = weight_product(b);
  const bool x = b.dX && wide_sizes(qx), w = b.dW && wide_sizes(qw);
  // the instructions of both products together: they share the layouts of G
  bool x_bf16 = may_bf16(qx), w_bf16 = may_bf16(qw);
  if ((x && x_bf16 && may_float(qx)) || (w && w_bf16 && may_float(qw))) {
    double best = 0.0;
    for (int c = 3; c >= 0; --c) {
      const bool xb = c & 1, wb = c & 2;
      if (x ? !(xb ? may_bf16(qx) : may_float(qx)) : xb) continue;
      if (w ? !(wb ? may_bf16(qw) : may_float(qw)) : wb) continue;
      const BackwardPlan p = lay_backward(b, nullptr, xb, wb);
      const double us = (layout_us(p.lay) + (x ? product_us(p.x) : 0.0) + (w ? product_us(p.w) : 0.0)) *
                        ((x && !xb && may_bf16(qx)) || (w && !wb && may_bf16(qw)) ? AHEAD : 1.0);
      if (best == 0.0 || us < best) { best = us; x_bf16 = xb; w_bf16 = wb; }
    }
  }
  BackwardPlan p = lay_backward(b, base, x_bf16, w_bf16);
  p.pair = x && w && pairs(p.w, p.x);
  const size_t nx = b.dX ? up(parts_workspace(p.x)) : 0, nw = b.dW ? up(parts_workspace(p.w)) : 0;
  p.partial_x = base + p.lay.bytes;
  p.partial_w = p.partial_x + (p.pair ? nx : 0);
  p.bytes = p.lay.bytes + (p.pair ? nx + nw : nx > nw ? nx : nw);
  return p;
}

// ---- thin gradients: at most 16 columns or rows of G
struct ThinPlan {
  bool thin, by_column;
  int chunk, chunks;
  size_t bytes, sums;                 // of the chunks' sums; where those of db begin
};
// Chunks of the long side: about a thousand workgroups with the blocks of 256 k, and no fewer than 32 rows each, 8 per wavefront.
ThinPlan thin_plan(const BackwardArgs& b) {
  ThinPlan p = {};
  const long long nt = b.F < b.M ? b.F : b.M, rows = b.F < b.M ? b.M : b.F, blocks = (b.K + 255) / 256;
  p.thin = nt <= 16;
  if (!p.thin) return p;
  p.by_column = b.F < b.M;
  long long chunks = blocks >= 1024 ? 1 : 1024 / blocks;
  if (chunks > (rows + 31) / 32) chunks = (rows + 31) / 32;
  long long chunk = ((rows + chunks - 1) / chunks + 3) / 4 * 4;
  if (chunk > THIN_ROWS) chunk = THIN_ROWS;
  p.chunk = (int)chunk;
  p.chunks = (int)((rows + chunk - 1) / chunk);
  if (p.chunks > 1) {
    p.sums = up((size_t)p.chunks * nt * b.K * sizeof(float));
    p.bytes = p.sums + (p.by_column ? up((size_t)p.chunks * b.F * sizeof(float)) : 0);
  }
  return p;
}
template <typename TS, typename TT, typename TY>
hipError_t launch_thin_sizes(const ThinArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)((a.K + 255) / 256 * a.chunks));
  if (a.nt <= 4) hipLaunchKernelGGL((thin_backward_kernel<TS, TT, TY, 4>), grid, dim3(256), 0, s, a);
  else if (a.nt <= 8) hipLaunchKernelGGL((thin_backward_kernel<TS, TT, TY, 8>), grid, dim3(256), 0, s, a);
  else if (a.nt <= 12) hipLaunchKernelGGL((thin_backward_kernel<TS, TT, TY, 12>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((thin_backward_kernel<TS, TT, TY, 16>), grid, dim3(256), 0, s, a);
  return hipGetLastError();
}
template <typename TS, typename TT>
hipError_t launch_thin_y(const ThinArgs& a, int ytype, hipStream_t s) {
  return ytype ? launch_thin_sizes<TS, TT, __bf16>(a, s) : launch_thin_sizes<TS, TT, float>(a, s);
}
hipError_t launch_thin(const BackwardArgs& b, const ThinPlan& p, char* ws, hipStream_t s) {
  ThinArgs a = {};
  const bool c = p.by_column;
  a.S = c ? b.X : b.W;  a.T = c ? b.W : b.X;  a.g = b.dY;  a.f = b.D;
  void* outT = c ? static_cast<void*>(b.dW) : b.dX;
  a.outS = c ? b.dX : static_cast<void*>(b.dW);
  a.outT = outT && p.chunks > 1 ? ws : outT;
  a.sum = b.db && c && p.chunks > 1 ? reinterpret_cast<float*>(ws + p.sums) : b.db;
  a.rows = c ? b.M : b.F;  a.K = b.K;  a.F = b.F;
  a.nt = (int)(c ? b.F : b.M);  a.by_column = c;
  a.chunk = p.chunk;  a.chunks = p.chunks;
  a.outS_type = c ? b.dxtype : 0;  a.outT_type = c ? 0 : b.dxtype;
  a.scale = b.scale;
  const int ts = c ? b.xtype : b.wtype, tt = c ? b.wtype : b.xtype;
  a.kept = b.X8;
  a.f8 = b.D8;
  hipError_t e;
  if (b.X8.codes) e = c ? (tt ? launch_thin_y<Mx8, __bf16>(a, b.ytype, s) : launch_thin_y<Mx8, float>(a, b.ytype, s))
                          : (ts ? launch_thin_y<__bf16, Mx8>(a, b.ytype, s) : launch_thin_y<float, Mx8>(a, b.ytype, s));
  else e = ts ? (tt ? launch_thin_y<__bf16, __bf16>(a, b.ytype, s) : launch_thin_y<__bf16, float>(a, b.ytype, s))
                    : (tt ? launch_thin_y<float, __bf16>(a, b.ytype, s) : launch_thin_y<float, float>(a, b.ytype, s));
  if (e != hipSuccess || p.chunks == 1) return e;
  if (outT) {
    Product q = {};
    q.e = Epilogue{0, 0, a.outT_type, 1.0f, nullptr, nullptr, outT, nullptr};
    q.I = a.nt; q.J = b.K;
    e = join_parts(q, static_cast<const float*>(a.outT), p.chunks, s);
  }
  if (e == hipSuccess && b.db && c) e = add_chunks(a.sum, p.chunks, b.F, b.db, s);
  return e;
}

}  // namespace

hipError_t join_parts(const Epilogue& e, const float* partial, int parts, long long I, long long J, hipStream_t s) {
  const long long n = I * J, per = parts >= 16 ? 64 : 256, blocks = (n + per - 1) / per;
  const dim3 grid((unsigned)(blocks < 4096 ? blocks : 4096));
  if (parts >= 16) hipLaunchKernelGGL(join_parts_kernel<16>, grid, dim3(1024), 0, s, e, partial, parts, n, J);
  else hipLaunchKernelGGL(join_parts_kernel<1>, grid, dim3(256), 0, s, e, partial, parts, n, J);
  return hipGetLastError();
}


size_t product_workspace(const Product& q) {
  const FewPlan f = few_plan(q);
  if (f.few) return f.parts > 1 ? (size_t)f.parts * (size_t)q.I * (size_t)q.J * sizeof(float) : 0;
  if (!wide_sizes(q)) return parts_workspace(q);
  Layout l = {};
  Product p = q;
  const bool bf16 = forward_bf16(q);
  p.A = l.plane(q.A, bf16, q.I, q.Kc, few_tiles(q));
  p.B = l.plane(q.B, bf16, q.J, q.Kc, few_tiles(q));
  return l.bytes + parts_workspace(p);
}

hipError_t launch_product(const Product& q, void* ws, hipStream_t s) {
  const FewPlan f = few_plan(q);
  if (f.few) {
    const hipError_t e = launch_few(q, f, static_cast<float*>(ws), s);
    return e != hipSuccess || f.parts == 1 ? e : join_parts(q, static_cast<float*>(ws), f.parts, s);
  }
  if (!wide_sizes(q)) return launch_any_product(q, ws, s);
  Layout l = {};
  l.base = static_cast<char*>(ws);
  Product p = q;
  const bool bf16 = forward_bf16(q);
  p.A = l.plane(q.A, bf16, q.I, q.Kc, few_tiles(q));
  p.B = l.plane(q.B, bf16, q.J, q.Kc, few_tiles(q));
  const hipError_t e = l.launch(s);
  return e != hipSuccess ? e : launch_wide_product(p, l.base + l.bytes, s);
}

// What the calls with these sizes and types need, whichever outputs are wanted (the pointers say only whether one is there)
size_t backward_workspace(const BackwardArgs& b) {
  const ThinPlan t = thin_plan(b);
  if (t.thin) return t.bytes;
  size_t n = 0;
  for (int wanted = 0; wanted < 8; ++wanted) {
    BackwardArgs a = b;
    if (!(wanted & 1)) a.dX = nullptr;
    if (!(wanted & 2)) a.dW = nullptr;
    if (!(wanted & 4)) a.db = nullptr;
    const size_t m = backward_plan(a, nullptr).bytes;
    n = n > m ? n : m;
  }
  return n;
}

bool backward_reads_kept(const BackwardArgs& b) {
  // (the tiles for offsets beyond 32 bits read their operands as they lie)
  return thin_plan(b).thin || (wide_sizes(input_product(b)) && wide_sizes(weight_product(b)));
}

hipError_t launch_backward(const BackwardArgs& b, void* ws, hipStream_t s) {
  const ThinPlan t = thin_plan(b);
  if (t.thin) return launch_thin(b, t, static_cast<char*>(ws), s);
  const BackwardPlan p = backward_plan(b, static_cast<char*>(ws));
  hipError_t e = p.lay.launch(s);
  if (e == hipSuccess && b.db && p.chunks > 1) e = add_chunks(p.sums, p.chunks, b.F, b.db, s);
  if (e != hipSuccess) return e;
  if (p.pair) return launch_wide_pair(p.w, p.x, p.partial_w, p.partial_x, s);
  if (b.dX) e = wide_sizes(p.x) ? launch_wide_product(p.x, p.partial_x, s) : launch_any_product(p.x, p.partial_x, s);
  if (e == hipSuccess && b.dW) e = wide_sizes(p.w) ? launch_wide_product(p.w, p.partial_w, s) : launch_any_product(p.w, p.partial_w, s);
  return e;
}

hipError_t launch_zero(float* out, long long n, hipStream_t s) {
  const long long blocks = (n + 255) / 256;
  if (n > 0) hipLaunchKernelGGL(zero_kernel, dim3((unsigned)(blocks < 4096 ? blocks : 4096)), dim3(256), 0, s, out, n);
  return hipGetLastError();
}

}  // namespace mgrit
