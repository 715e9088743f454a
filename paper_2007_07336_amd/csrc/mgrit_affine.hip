// End layers: matrix products with bias, activation and residual in the epilogue, and the products and sums of their
// backward pass.  Every one of them is C[i][j] = sum_k A(i, k) B(j, k) in some order of its operands (mgrit_ops.h).
#include "mgrit_device.h"
#include "mgrit_ops.h"

namespace mgrit {

namespace {

// ------------------------------------------------------------------------------------------ values
__device__ __forceinline__ float widen(float v) { return v; }
__device__ __forceinline__ float widen(__bf16 v) { return static_cast<float>(v); }
template <typename T> __device__ __forceinline__ T narrow(float v) { return static_cast<T>(v); }   // to nearest, ties to even

// tanh(z) and 1 - tanh(z)^2 to about 2e-7 relative.  With e = exp(-2 |z|): tanh |z| = (1 - e) / (1 + e), and 1 - tanh^2 =
// 4 e / (1 + e)^2, which loses nothing near saturation; below 0.35, where 1 - e cancels, the odd series up to z^11.
__device__ __forceinline__ float tanh_with_slope(float z, float* slope) {
  const float a = fabsf(z);
  const float e = __builtin_amdgcn_exp2f(a * -2.885390081777927f);
  const float r = __builtin_amdgcn_rcpf(1.0f + e);
  const float q = z * z;
  const float series = z + z * q * (-0.33333333333f + q * (0.13333333333f + q * (-0.05396825397f + q * (0.02186948854f - q * 0.00886323552f))));
  *slope = 4.0f * e * r * r;
  return a < 0.35f ? series : copysignf((1.0f - e) * r, z);
}

struct Out { float y, d; };
// act(z) and act'(z); a NaN stays one
__device__ __forceinline__ Out activate(float z, int act) {
  Out o;
  if (act == ACT_TANH) {
    o.y = tanh_with_slope(z, &o.d);
  } else if (act == ACT_RELU) {
    o.y = z <= 0.0f ? 0.0f : z;
    o.d = z > 0.0f ? 1.0f : z != z ? z : 0.0f;
  } else {
    o.y = z;
    o.d = 1.0f;
  }
  return o;
}

template <typename OT>
__device__ __forceinline__ void finish(const Epilogue& e, long long at, long long col, float sum) {
  OT* out = static_cast<OT*>(e.out);
  if (!e.fwd) {
    out[at] = narrow<OT>(e.scale * sum);
    return;
  }
  const Out o = activate(e.bias ? sum + e.bias[col] : sum, e.act);
  const float y = e.scale * o.y;
  out[at] = narrow<OT>(e.R ? static_cast<const OT*>(e.R)[at] + y : y);
  if (e.D) static_cast<OT*>(e.D)[at] = narrow<OT>(e.scale * o.d);
}

// ------------------------------------------------------------------------------------------ any size, any order
// Tile of 64 x 64 outputs, four wavefronts with 32 x 32 of them each; slabs of the contraction go through registers (the
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

// blockIdx.x: tile; blockIdx.y: part of the contraction (kpart long).  One part: the epilogue here; more: sums to
// partial[part][i][j].
template <typename TA, typename TB, typename CT, bool HF, bool AS, bool BS>
__global__ __launch_bounds__(256) void product_tile_kernel(Product q, long long kpart, float* partial) {
  __shared__ __attribute__((aligned(16))) CT As[GT * Slab<CT>::ST], Bs[GT * Slab<CT>::ST];
  const long long tj = (q.J + GT - 1) / GT;
  const int L = logical_block();
  const long long i0 = L / tj * GT, j0 = L % tj * GT;
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

__global__ __launch_bounds__(256) void join_parts_kernel(Epilogue e, const float* partial, int parts, long long n, long long J) {
  for (long long at = blockIdx.x * 256LL + threadIdx.x; at < n; at += gridDim.x * 256LL) {
    float s = partial[at];
    for (int k = 1; k < parts; ++k) s += partial[k * n + at];
    if (e.otype) finish<__bf16>(e, at, at % J, s);
    else finish<float>(e, at, at % J, s);
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
  hipLaunchKernelGGL((product_tile_kernel<TA, TB, CT, HF, AS, BS>), dim3((unsigned)tiles_of(q), (unsigned)parts), dim3(256), 0, s, q,
                     kpart, parts > 1 ? partial : nullptr);
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

// ------------------------------------------------------------------------------------------ sums of columns
// Workgroup (64 columns, chunk of rows): four wavefronts take every fourth row; then the chunks are added up.
constexpr int CHUNK = 256;
template <typename T>
__global__ __launch_bounds__(256) void column_sum_kernel(const T* g, const T* f, long long M, long long F, float scale, float* out) {
  __shared__ float part[4][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const long long col = blockIdx.x * 64LL + lane, m0 = blockIdx.y * (long long)CHUNK, m1 = m0 + CHUNK < M ? m0 + CHUNK : M;
  float s = 0.0f;
  if (col < F)
    for (long long m = m0 + wave; m < m1; m += 4) s += f ? widen(g[m * F + col]) * widen(f[m * F + col]) : widen(g[m * F + col]);
  part[wave][lane] = s;
  __syncthreads();
  if (wave == 0 && col < F) out[blockIdx.y * F + col] = scale * ((part[0][lane] + part[1][lane]) + (part[2][lane] + part[3][lane]));
}
__global__ __launch_bounds__(256) void add_chunks_kernel(const float* part, long long chunks, long long F, float* out) {
  const long long col = blockIdx.x * 256LL + threadIdx.x;
  if (col >= F) return;
  float s = 0.0f;
  for (long long c = 0; c < chunks; ++c) s += part[c * F + col];
  out[col] = s;
}

__global__ __launch_bounds__(256) void zero_kernel(float* out, long long n) {
  for (long long i = blockIdx.x * 256LL + threadIdx.x; i < n; i += gridDim.x * 256LL) out[i] = 0.0f;
}

}  // namespace

size_t product_workspace(const Product& q) {
  const int parts = parts_of(q);
  return parts > 1 ? (size_t)parts * (size_t)q.I * (size_t)q.J * sizeof(float) : 0;
}

hipError_t launch_product(const Product& q, void* ws, hipStream_t s) {
  const int parts = parts_of(q);
  float* partial = static_cast<float*>(ws);
  hipError_t e;
  if (!q.A.kslow && !q.B.kslow) e = launch_types<false, false, false>(q, partial, parts, s);
  else if (!q.A.kslow) e = q.A.f ? launch_types<true, false, true>(q, partial, parts, s) : launch_types<false, false, true>(q, partial, parts, s);
  else e = q.A.f ? launch_types<true, true, true>(q, partial, parts, s) : launch_types<false, true, true>(q, partial, parts, s);
  if (e != hipSuccess || parts == 1) return e;
  const long long n = q.I * q.J, blocks = (n + 255) / 256;
  hipLaunchKernelGGL(join_parts_kernel, dim3((unsigned)(blocks < 4096 ? blocks : 4096)), dim3(256), 0, s, q.e, partial, parts, n, q.J);
  return hipGetLastError();
}

size_t column_sum_workspace(long long M, long long F) {
  const long long chunks = (M + CHUNK - 1) / CHUNK;
  return chunks > 1 ? (size_t)chunks * (size_t)F * sizeof(float) : 0;
}

hipError_t launch_column_sum(const Operand& G, long long M, long long F, float scale, float* db, void* ws, hipStream_t s) {
  const long long chunks = (M + CHUNK - 1) / CHUNK;
  float* out = chunks > 1 ? static_cast<float*>(ws) : db;
  // (a grid's second dimension ends at 65535 chunks: the rows of taller layers are handed over in several launches)
  for (long long c = 0; c < chunks; c += 65535) {
    const long long n = chunks - c < 65535 ? chunks - c : 65535, rows = M - c * CHUNK, at = c * CHUNK * F;
    const dim3 grid((unsigned)((F + 63) / 64), (unsigned)n);
    if (G.type)
      hipLaunchKernelGGL(column_sum_kernel<__bf16>, grid, dim3(256), 0, s, static_cast<const __bf16*>(G.p) + at,
                         G.f ? static_cast<const __bf16*>(G.f) + at : nullptr, rows, F, scale, out + c * F);
    else
      hipLaunchKernelGGL(column_sum_kernel<float>, grid, dim3(256), 0, s, static_cast<const float*>(G.p) + at,
                         G.f ? static_cast<const float*>(G.f) + at : nullptr, rows, F, scale, out + c * F);
  }
  if (chunks > 1) hipLaunchKernelGGL(add_chunks_kernel, dim3((unsigned)((F + 255) / 256)), dim3(256), 0, s, out, chunks, F, db);
  return hipGetLastError();
}

hipError_t launch_zero(float* out, long long n, hipStream_t s) {
  const long long blocks = (n + 255) / 256;
  if (n > 0) hipLaunchKernelGGL(zero_kernel, dim3((unsigned)(blocks < 4096 ? blocks : 4096)), dim3(256), 0, s, out, n);
  return hipGetLastError();
}

}  // namespace mgrit
