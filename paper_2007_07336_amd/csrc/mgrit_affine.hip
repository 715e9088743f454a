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

// Eight results of one row.  whole: all eight exist and lie on a multiple of eight
template <typename T> struct Eight { T v[8]; };
__device__ __forceinline__ void load8(const float* p, float (&v)[8]) {
  *reinterpret_cast<floatx4*>(v) = *reinterpret_cast<const floatx4*>(p);
  *reinterpret_cast<floatx4*>(v + 4) = *reinterpret_cast<const floatx4*>(p + 4);
}
__device__ __forceinline__ void load8(const __bf16* p, float (&v)[8]) {
  const bf16x8 b = *reinterpret_cast<const bf16x8*>(p);
#pragma unroll
  for (int k = 0; k < 8; ++k) v[k] = widen(b[k]);
}
__device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
  *reinterpret_cast<floatx4*>(p) = floatx4{v[0], v[1], v[2], v[3]};
  *reinterpret_cast<floatx4*>(p + 4) = floatx4{v[4], v[5], v[6], v[7]};
}
__device__ __forceinline__ void store8(__bf16* p, const float (&v)[8]) {
  bf16x8 b;
#pragma unroll
  for (int k = 0; k < 8; ++k) b[k] = narrow<__bf16>(v[k]);
  *reinterpret_cast<bf16x8*>(p) = b;
}
template <typename OT>
__device__ __forceinline__ void put8(OT* p, const float (&v)[8], bool whole, long long left) {
  if (whole) {
    store8(p, v);
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (k < left) p[k] = narrow<OT>(v[k]);
  }
}
template <typename OT>
__device__ __forceinline__ void finish8(const Epilogue& e, long long at, float (&v)[8], const float (&bias)[8], bool whole, long long left) {
  OT* out = static_cast<OT*>(e.out) + at;
  if (!e.fwd) {
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] *= e.scale;
    put8(out, v, whole, left);
    return;
  }
  float d[8], r[8];
  if (e.R) {
    const OT* R = static_cast<const OT*>(e.R) + at;
    if (whole) {
      load8(R, r);
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k) r[k] = k < left ? widen(R[k]) : 0.0f;
    }
  }
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const Out o = activate(v[k] + bias[k], e.act);
    v[k] = e.R ? r[k] + e.scale * o.y : e.scale * o.y;
    d[k] = e.scale * o.d;
  }
  put8(out, v, whole, left);
  if (e.D) put8(static_cast<OT*>(e.D) + at, d, whole, left);
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

// ------------------------------------------------------------------------------------------ large products
// Operands as planes: rows along k, padded with zeros to whole slabs of 128 bytes (64 bf16 or 32 float), 16-byte pieces.  What the
// caller has in this form is read in place; anything else -- transposed, ragged, with a factor, of another type -- is laid
// out in the workspace first (lay_out_kernel), which costs a pass over the operand and keeps the multiplying loop free of
// everything but multiplications.
typedef __attribute__((address_space(3))) void LdsPtr;
// 16 bytes per lane from base + each lane's offset + along to `to` and the 1008 bytes behind it, in lane order
__device__ __forceinline__ void to_lds(const char* base, int offset, int along, unsigned char* to) {
  __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(base), 0, -1, 0x00020000);
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (LdsPtr*)to, 16, offset, along, 0, 0);
}

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
  const void* p;
  long long ld;                // bytes from row to row
  long long part;              // bytes from part to part
};
struct WideArgs {
  Plane A, B;
  Epilogue e;
  long long I, J;
  int slabs;                   // of one pass over the contraction
  int passes;                  // A's parts, each of which is multiplied with B
  int per;                     // slabs that one workgroup takes (blockIdx.y: which), all passes counted
  float* partial;              // several workgroups: their sums
};

// Tile of BT x BT outputs, four wavefronts with a quarter each.  A slab of both operands is 2 BT rows of 128 bytes in LDS, its
// 16-byte pieces in the order piece ^ (row & 7): the hardware writes LDS in lane order, so the lanes pick their pieces in that
// order from memory, and eight lanes that read the same piece of eight rows meet different banks.  Two slabs are in LDS: while one
// is multiplied in four steps, the next one is on its way.  Behind the last step's reads a barrier says that nobody needs the old slab
// any more and that the next one has arrived; the loads of the one after go out at once and have a whole slab's time.
template <typename CT, int BT, typename OT>
__global__ __launch_bounds__(256, BT == 256 ? 1 : 2) void product_wide_kernel(WideArgs a) {
  typedef typename Mma<CT>::Frag Frag;
  constexpr int T = BT / 64, NL = BT / 32, SLAB = BT * 128;       // 32 x 32 tiles along a wavefront's side; loads per operand and slab
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), wi = wave >> 1, wj = wave & 1;
  // tiles in groups of GM rows of tiles, so that the tiles that an XCD works on at a time share few panels of both operands
  constexpr int GM = 4;
  const long long ti = (a.I + BT - 1) / BT, tj = (a.J + BT - 1) / BT;
  const long long L = logical_block(), group = L / (GM * tj), first = group * GM, size = ti - first < GM ? ti - first : GM, in = L - group * GM * tj;
  const long long i0 = (first + in % size) * BT, j0 = in / size * BT;

  const int total = a.slabs * a.passes, t0 = (int)blockIdx.y * a.per, t1 = t0 + a.per < total ? t0 + a.per : total;
  int offA[NL], offB[NL];
#pragma unroll
  for (int i = 0; i < NL; ++i) {
    const int r = wave * (BT / 4) + i * 8 + (lane >> 3), piece = (lane & 7) ^ ((r >> 1) & 7);
    const long long ra = i0 + r < a.I ? r : a.I - 1 - i0, rb = j0 + r < a.J ? r : a.J - 1 - j0;
    offA[i] = (int)(ra * a.A.ld) + piece * 16;
    offB[i] = (int)(rb * a.B.ld) + piece * 16;
  }
  const char* baseA = static_cast<const char*>(a.A.p) + i0 * a.A.ld;
  const char* baseB = static_cast<const char*>(a.B.p) + j0 * a.B.ld;
  // the next slab to load: of which pass (A's parts, each against B from its start), and how far along the rows
  int left = a.slabs - t0 % a.slabs, along = t0 % a.slabs * 128;
  baseA += t0 / a.slabs * a.A.part;
  auto load = [&](int buf, int i) {                              // load i of 2 NL
    unsigned char* to = lds + buf * 2 * SLAB + wave * (BT / 4) * 128 + (i < NL ? i * 1024 : SLAB + (i - NL) * 1024);
    to_lds(i < NL ? baseA : baseB, i < NL ? offA[i % NL] : offB[i % NL], along, to);
  };
  auto next = [&]() {
    along += 128;
    if (--left == 0) { left = a.slabs; along = 0; baseA += a.A.part; }
  };
  const int c = lane & 31, g = lane >> 5;
  const unsigned char* readA = lds + (wi * (BT / 2) + c) * 128;
  const unsigned char* readB = lds + SLAB + (wj * (BT / 2) + c) * 128;
  int piece[4];
#pragma unroll
  for (int step = 0; step < 4; ++step) piece[step] = ((2 * step + g) ^ ((c >> 1) & 7)) << 4;
  Frag fa[2][T], fb[2][T];
  auto read = [&](int buf, int step, int n) {                    // fragment n of 2 T
    const int at = buf * 2 * SLAB + piece[step] + (n / 2) * 32 * 128;
    if (n & 1) fb[step & 1][n / 2] = *reinterpret_cast<const Frag*>(readB + at);
    else       fa[step & 1][n / 2] = *reinterpret_cast<const Frag*>(readA + at);
  };
  floatx16 acc[T][T];
#pragma unroll
  for (int i = 0; i < T; ++i)
#pragma unroll
    for (int j = 0; j < T; ++j) acc[i][j] = zero16();

  // One slab.  In every step the reads of the next one are spread over the first half of the multiplications; the order is fixed
  // in groups of T / 2 multiplications.  The loads of the slab after the next begin behind the barrier and are spread over SPREAD
  // steps: the address unit takes 16 cycles for one, and a wavefront that waits for it multiplies nothing.
  constexpr int SPREAD = 3, PER = (2 * NL + 2 * T * SPREAD - 1) / (2 * T * SPREAD);       // loads in a group
  auto multiply = [&](int buf, auto rest, auto more, auto last) {
#pragma unroll
    for (int step = 0; step < 4; ++step) {
      if (step == 3) asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
#pragma unroll
      for (int n = 0; n < 2 * T; ++n) {
        if (n < T && !(step == 3 && last)) {
          read(step < 3 ? buf : buf ^ 1, (step + 1) & 3, 2 * n);
          read(step < 3 ? buf : buf ^ 1, (step + 1) & 3, 2 * n + 1);
        }
        const int group = (step + 1) % 4 * 2 * T + n;
#pragma unroll
        for (int k = group * PER; k < (group + 1) * PER && k < 2 * NL; ++k) {
          if (step == 3 && more) load(buf, k);
          if (step < 3 && rest) load(buf ^ 1, k);
        }
#pragma unroll
        for (int k = 0; k < T / 2; ++k) {
          const int m = n * (T / 2) + k;
          Mma<CT>::go(fa[step & 1][m / T], fb[step & 1][m % T], acc[m / T][m % T]);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      if (step == SPREAD - 2 && rest) next();
    }
  };
  constexpr std::true_type yes{};
  constexpr std::false_type no{};
#pragma unroll
  for (int i = 0; i < 2 * NL; ++i) load(0, i);
  next();
  asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
  if (t0 + 1 < t1) {
#pragma unroll
    for (int i = 0; i < 2 * T * PER && i < 2 * NL; ++i) load(1, i);
  }
#pragma unroll
  for (int n = 0; n < 2 * T; ++n) read(0, 0, n);
  int buf = 0;
  for (int t = t0; t < t1 - 2; ++t, buf ^= 1) multiply(buf, yes, yes, no);
  if (t0 + 1 < t1) { multiply(buf, yes, no, no); buf ^= 1; }
  multiply(buf, no, no, yes);

  // Through LDS, 32 rows of the wavefront's quarter at a time, so that a lane has eight entries of a row in its hands
  constexpr int W = BT / 2, PITCH = W + 4;
  float* strip = reinterpret_cast<float*>(lds) + wave * 32 * PITCH;
  const int lc = lane % (W / 8) * 8, lr = lane / (W / 8);
  const long long col = j0 + wj * W + lc;
  const long long n = a.I * a.J;
  const bool whole = a.J % 8 == 0 && col + 8 <= a.J;
  float bias[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) bias[k] = a.e.fwd && a.e.bias && !a.partial && col + k < a.J ? a.e.bias[col + k] : 0.0f;
#pragma unroll
  for (int i = 0; i < T; ++i) {
#pragma unroll
    for (int j = 0; j < T; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) strip[((r & 3) + 8 * (r >> 2) + 4 * g) * PITCH + j * 32 + c] = acc[i][j][r];
    __builtin_amdgcn_wave_barrier();
    for (int r = lr; r < 32; r += 512 / W) {
      const long long row = i0 + wi * W + i * 32 + r, at = row * a.J + col;
      float v[8];
      *reinterpret_cast<floatx4*>(v) = *reinterpret_cast<const floatx4*>(strip + r * PITCH + lc);
      *reinterpret_cast<floatx4*>(v + 4) = *reinterpret_cast<const floatx4*>(strip + r * PITCH + lc + 4);
      if (row < a.I) {
        if (a.partial) put8(a.partial + blockIdx.y * n + at, v, whole, a.J - col);
        else finish8<OT>(a.e, at, v, bias, whole, a.J - col);
      }
    }
    __builtin_amdgcn_wave_barrier();
  }
}

// Operand -> planes: rows x (k padded to whole slabs) of CT, PARTS of them: 1 as it is (or widened); 2: the product of two bf16
// values, 16 significant bits, is the sum of two.  Workgroup: 64 rows x 64 k; where rows are the fast index in memory they
// change places in LDS.
template <typename T, typename CT, int PARTS, bool HF, bool KSLOW>
__global__ __launch_bounds__(256) void lay_out_kernel(const T* p, const T* f, long long ld, long long rows, long long Kc, CT* out, long long ldo, long long part) {
  __shared__ float tile[64][65];
  const long long kt = (ldo + 63) / 64, L = blockIdx.x;
  const long long r0 = L / kt * 64, k0 = L % kt * 64;
  const int t = threadIdx.x;
  if (KSLOW) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = t % 16 * 4, k = t / 16 + 16 * i;
      const long long at = (k0 + k) * ld + r0 + r, left = k0 + k < Kc ? rows - r0 - r : 0;
      Four<T> a, b;
      if (ld % 4 == 0 && left >= 4) {
        a = *reinterpret_cast<const Four<T>*>(__builtin_assume_aligned(p + at, 4 * sizeof(T)));
        if (HF) b = *reinterpret_cast<const Four<T>*>(__builtin_assume_aligned(f + at, 4 * sizeof(T)));
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          a.v[j] = j < left ? p[at + j] : T(0.0f);
          if (HF) b.v[j] = j < left ? f[at + j] : T(0.0f);
        }
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) tile[k][r + j] = HF ? widen(a.v[j]) * widen(b.v[j]) : widen(a.v[j]);
    }
    __syncthreads();
  }
  for (int n = t; n < 512; n += 256) {             // eight k of a row
    const int r = n / 8, k = n % 8 * 8;
    if (r0 + r >= rows || k0 + k >= ldo) continue;
    float v[8];
    if (KSLOW) {
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = tile[k + j][r];
    } else {
      const long long at = (r0 + r) * ld + k0 + k, left = Kc - k0 - k;
      float b[8];
      if (ld % 8 == 0 && left >= 8) {
        load8(p + at, v);
        if (HF) load8(f + at, b);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          v[j] = j < left ? widen(p[at + j]) : 0.0f;
          if (HF) b[j] = j < left ? widen(f[at + j]) : 0.0f;
        }
      }
      if (HF)
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] *= b[j];
    }
    CT* o = out + (r0 + r) * ldo + k0 + k;
    store8(o, v);
    if (PARTS == 2) {
      float lo[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) lo[j] = v[j] - widen(narrow<CT>(v[j]));
      store8(o + part, lo);
    }
  }
}

template <typename CT> constexpr int slab_of() { return 128 / (int)sizeof(CT); }

struct WidePlan {
  bool wide, bf16;
  int bt, slabs, passes, parts;       // parts: workgroups that share a tile's contraction
  bool copyA, copyB;
  long long ldp;                      // entries from row to row of a laid out plane
  size_t offB, offP, bytes;
};
inline bool in_place(const Operand& o, bool bf16, long long Kc) {
  const int slab = bf16 ? 64 : 32;
  return !o.kslow && !o.f && (o.type != 0) == bf16 && Kc % slab == 0 && o.ld == Kc;
}
WidePlan wide_plan(const Product& q) {
  WidePlan w = {};
  const long long t128 = (q.I + 127) / 128 * ((q.J + 127) / 128);
  w.wide = q.I >= 128 && q.J >= 128 && q.Kc >= 64 && t128 >= 16 && q.Kc <= (1LL << 20) && t128 < (1LL << 30);
  if (!w.wide) return w;
  w.bf16 = q.A.type && q.B.type;
  const int slab = w.bf16 ? 64 : 32;
  const long long t256 = (q.I + 255) / 256 * ((q.J + 255) / 256);
  w.bt = t256 >= 192 ? 256 : 128;
  w.passes = w.bf16 && q.A.f ? 2 : 1;
  w.slabs = (int)((q.Kc + slab - 1) / slab);
  w.ldp = (long long)w.slabs * slab;
  const long long tiles = w.bt == 256 ? t256 : t128;
  const int total = w.slabs * w.passes;
  long long parts = tiles >= 256 ? 1 : 512 / tiles;
  if (parts > total / 8) parts = total / 8 > 0 ? total / 8 : 1;
  w.parts = (int)parts;
  w.copyA = !in_place(q.A, w.bf16, q.Kc);
  w.copyB = !in_place(q.B, w.bf16, q.Kc);
  const size_t es = w.bf16 ? 2 : 4;
  auto up = [](size_t x) { return (x + 255) / 256 * 256; };
  w.offB = w.copyA ? up((size_t)w.passes * q.I * w.ldp * es) : 0;
  w.offP = w.offB + (w.copyB ? up((size_t)q.J * w.ldp * es) : 0);
  w.bytes = w.offP + (w.parts > 1 ? (size_t)w.parts * q.I * q.J * sizeof(float) : 0);
  return w;
}

template <typename T, typename CT, int PARTS, bool HF>
hipError_t lay_out(const Operand& o, long long rows, long long Kc, void* out, long long ldp, hipStream_t s) {
  const dim3 grid((unsigned)((rows + 63) / 64 * ((ldp + 63) / 64)));
  const T *p = static_cast<const T*>(o.p), *f = static_cast<const T*>(o.f);
  if (o.kslow) hipLaunchKernelGGL((lay_out_kernel<T, CT, PARTS, HF, true>), grid, dim3(256), 0, s, p, f, o.ld, rows, Kc, static_cast<CT*>(out), ldp, rows * ldp);
  else hipLaunchKernelGGL((lay_out_kernel<T, CT, PARTS, HF, false>), grid, dim3(256), 0, s, p, f, o.ld, rows, Kc, static_cast<CT*>(out), ldp, rows * ldp);
  return hipGetLastError();
}
hipError_t lay_out(const Operand& o, bool bf16, long long rows, long long Kc, void* out, long long ldp, hipStream_t s) {
  if (bf16) return o.f ? lay_out<__bf16, __bf16, 2, true>(o, rows, Kc, out, ldp, s) : lay_out<__bf16, __bf16, 1, false>(o, rows, Kc, out, ldp, s);
  if (o.type) return o.f ? lay_out<__bf16, float, 1, true>(o, rows, Kc, out, ldp, s) : lay_out<__bf16, float, 1, false>(o, rows, Kc, out, ldp, s);
  return o.f ? lay_out<float, float, 1, true>(o, rows, Kc, out, ldp, s) : lay_out<float, float, 1, false>(o, rows, Kc, out, ldp, s);
}

template <typename CT, int BT, typename OT>
hipError_t launch_wide_tiles(const WideArgs& a, int parts, hipStream_t s) {
  static LdsOptIn opt;
  const size_t smem = 4 * BT * 128;
  const hipError_t e = opt.raise(reinterpret_cast<const void*>(&product_wide_kernel<CT, BT, OT>), smem);
  if (e != hipSuccess) return e;
  const long long tiles = (a.I + BT - 1) / BT * ((a.J + BT - 1) / BT);
  hipLaunchKernelGGL((product_wide_kernel<CT, BT, OT>), dim3((unsigned)tiles, (unsigned)parts), dim3(256), smem, s, a);
  return hipGetLastError();
}
template <typename CT, int BT>
hipError_t launch_wide_out(const WideArgs& a, int parts, hipStream_t s) {
  return a.e.otype ? launch_wide_tiles<CT, BT, __bf16>(a, parts, s) : launch_wide_tiles<CT, BT, float>(a, parts, s);
}

hipError_t join_parts(const Product& q, const float* partial, int parts, hipStream_t s) {
  const long long n = q.I * q.J, blocks = (n + 255) / 256;
  hipLaunchKernelGGL(join_parts_kernel, dim3((unsigned)(blocks < 4096 ? blocks : 4096)), dim3(256), 0, s, q.e, partial, parts, n, q.J);
  return hipGetLastError();
}

hipError_t launch_wide_product(const Product& q, const WidePlan& w, void* ws, hipStream_t s) {
  char* base = static_cast<char*>(ws);
  const long long es = w.bf16 ? 2 : 4;
  hipError_t e = hipSuccess;
  if (w.copyA) e = lay_out(q.A, w.bf16, q.I, q.Kc, base, w.ldp, s);
  if (e == hipSuccess && w.copyB) e = lay_out(q.B, w.bf16, q.J, q.Kc, base + w.offB, w.ldp, s);
  if (e != hipSuccess) return e;
  WideArgs a = {};
  a.A = w.copyA ? Plane{base, w.ldp * es, q.I * w.ldp * es} : Plane{q.A.p, q.A.ld * es, 0};
  a.B = w.copyB ? Plane{base + w.offB, w.ldp * es, 0} : Plane{q.B.p, q.B.ld * es, 0};
  a.e = q.e;
  a.I = q.I; a.J = q.J;
  a.slabs = w.slabs;
  a.passes = w.passes;
  a.per = (w.slabs * w.passes + w.parts - 1) / w.parts;
  const int parts = (w.slabs * w.passes + a.per - 1) / a.per;          // none of them empty
  a.partial = parts > 1 ? reinterpret_cast<float*>(base + w.offP) : nullptr;
  if (w.bf16) e = w.bt == 256 ? launch_wide_out<__bf16, 256>(a, parts, s) : launch_wide_out<__bf16, 128>(a, parts, s);
  else e = w.bt == 256 ? launch_wide_out<float, 256>(a, parts, s) : launch_wide_out<float, 128>(a, parts, s);
  if (e != hipSuccess || parts == 1) return e;
  return join_parts(q, a.partial, parts, s);
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
  const WidePlan w = wide_plan(q);
  if (w.wide) return w.bytes;
  const int parts = parts_of(q);
  return parts > 1 ? (size_t)parts * (size_t)q.I * (size_t)q.J * sizeof(float) : 0;
}

hipError_t launch_product(const Product& q, void* ws, hipStream_t s) {
  const WidePlan w = wide_plan(q);
  if (w.wide) return launch_wide_product(q, w, ws, s);
  const int parts = parts_of(q);
  float* partial = static_cast<float*>(ws);
  hipError_t e;
  if (!q.A.kslow && !q.B.kslow) e = launch_types<false, false, false>(q, partial, parts, s);
  else if (!q.A.kslow) e = q.A.f ? launch_types<true, false, true>(q, partial, parts, s) : launch_types<false, false, true>(q, partial, parts, s);
  else e = q.A.f ? launch_types<true, true, true>(q, partial, parts, s) : launch_types<false, true, true>(q, partial, parts, s);
  if (e != hipSuccess || parts == 1) return e;
  return join_parts(q, partial, parts, s);
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
