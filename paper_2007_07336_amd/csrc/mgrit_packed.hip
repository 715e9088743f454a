// Values in few bits: packing and unpacking of microscaled arrays, and products with weights in 4 bits.
#include "mgrit_epilogue.h"

namespace mgrit {

namespace {

constexpr long long MOST_BLOCKS = 1LL << 22;                     // of one launch: fewer than 2^32 threads
constexpr int MX8 = MGRIT_MX8, MX4 = MGRIT_MX4;
constexpr int SLAB = 256;                                        // columns of a slab: 8 blocks, 128 bytes of 4-bit codes

inline size_t up(size_t x) { return (x + 255) / 256 * 256; }

// Where block b's scale lies among its slab's eight: lanes of one half of a wavefront take blocks 0 2 4 6 in turn, those of the other 1 3 5 7
__device__ __forceinline__ int place_of(int b) { return (b & 1) * 4 + (b >> 1); }
// 2^(byte - 127) as a float (byte 0: a subnormal one)
__device__ __forceinline__ float scale_of(unsigned byte) { return __builtin_bit_cast(float, byte ? byte << 23 : 0x00400000u); }
// The scale of a block whose largest magnitude has these bits: with top = m 2^x, 1 <= m < 2, and the largest value l 2^e it is 2^(x - e),
// twice that if m > l; subnormal tops get the least scale, for which everything is small enough
template <int FORMAT> __device__ __forceinline__ unsigned scale_byte(unsigned top) {
  constexpr unsigned E = FORMAT == MX8 ? 8 : 2, L = FORMAT == MX8 ? 0x600000u : 0x400000u;
  if (top >= 0x7f800000u) return 255u;
  const unsigned x = (top >> 23) + ((top & 0x7fffffu) > L ? 1u : 0u);
  return x > E ? x - E : 0u;
}
__device__ __forceinline__ unsigned codes4(const float (&v)[8], float scale) {                     // eight 4-bit codes
  unsigned c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, v[0], v[1], scale, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[2], v[3], scale, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[4], v[5], scale, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[6], v[7], scale, 3);
}
typedef short short2v __attribute__((ext_vector_type(2)));
__device__ __forceinline__ unsigned codes8(float a, float b, float c, float d, float scale) {     // four 8-bit codes
  short2v r = {0, 0};
  r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, a, b, scale, false);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, c, d, scale, true);
  return __builtin_bit_cast(unsigned, r);
}

// Eight columns a thread, four lanes a block.  Bound by memory: 8192 x 4096 bf16 into 4 bits 17 us (85 MB, 5.0 TB/s), into 8 bits 23 (102 MB).
template <typename T, int FORMAT>
__global__ __launch_bounds__(256) void pack_kernel(Packed p, const T* X, long long first) {
  const unsigned per = (unsigned)(p.slabs * (SLAB / 8));         // eights of a row
  const long long base = (first + blockIdx.x) * 256;
  const unsigned off = (unsigned)(base % per) + threadIdx.x;
  const long long row = base / per + off / per;
  if (row >= p.rows) return;                                     // (whole blocks of 32 at a time: rows have a multiple of them)
  const unsigned e = off % per;
  const long long k = e * 8LL, left = p.cols - k;
  const T* x = X + row * p.cols + k;
  float v[8];
  if (left >= 8) {
    load8(x, v);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = j < left ? widen(x[j]) : 0.0f;
  }
  unsigned top = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const unsigned u = __builtin_bit_cast(unsigned, v[j]) & 0x7fffffffu;
    top = u > top ? u : top;
  }
#pragma unroll
  for (int d = 1; d < 4; d <<= 1) {
    const unsigned u = (unsigned)__shfl_xor((int)top, d);
    top = u > top ? u : top;
  }
  const unsigned byte = scale_byte<FORMAT>(top);
  if (byte == 255u) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = 0.0f;
  }
  const float scale = scale_of(byte == 255u ? 127u : byte);
  if constexpr (FORMAT == MX4) {
    *reinterpret_cast<unsigned*>(p.codes + row * p.pitch + e * 4LL) = codes4(v, scale);
  } else {
    *reinterpret_cast<uint2*>(p.codes + row * p.pitch + e * 8LL) = make_uint2(codes8(v[0], v[1], v[2], v[3], scale), codes8(v[4], v[5], v[6], v[7], scale));
  }
  if ((e & 3) == 0) {
    const unsigned b = e / 4;
    p.scales[((long long)(b / 8) * p.rows + row) * 8 + place_of(b & 7)] = (unsigned char)byte;
  }
}

typedef float floatx2v __attribute__((ext_vector_type(2)));
// Eight values of codes, in float
template <int FORMAT> __device__ __forceinline__ void values8(const unsigned char* at, unsigned byte, float (&v)[8]) {
  const float scale = byte == 255u ? NAN : scale_of(byte);
  floatx2v a[4];
  if constexpr (FORMAT == MX4) {
    const unsigned c = *reinterpret_cast<const unsigned*>(at);
    a[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 0);
    a[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 1);
    a[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 2);
    a[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, 1.0f, 3);
  } else {
    const uint2 c = *reinterpret_cast<const uint2*>(at);
    a[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c.x, 1.0f, false);
    a[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c.x, 1.0f, true);
    a[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c.y, 1.0f, false);
    a[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(c.y, 1.0f, true);
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = a[j / 2][j % 2] * scale;    // (by the instructions of ordinary floats, which keep subnormal results)
}
template <typename T, int FORMAT>
__device__ __forceinline__ void unpack(const Unpack& u, long long base) {
  const Packed& p = u.from;
  const unsigned per = (unsigned)((u.ld + 7) / 8);               // eights of a row of out
  const unsigned off = (unsigned)(base % per) + threadIdx.x;
  const long long row = base / per + off / per;
  if (row >= p.rows) return;
  const unsigned e = off % per;
  float v[8] = {};
  if (e * 8LL < p.cols) {
    const unsigned b = e / 4;
    const unsigned byte = p.scales[((long long)(b / 8) * p.rows + row) * 8 + place_of(b & 7)];
    values8<FORMAT>(p.codes + row * p.pitch + e * (FORMAT == MX4 ? 4LL : 8LL), byte, v);
    if (byte == 255u) {                                          // (what lies behind the last column is zero all the same)
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (e * 8LL + j >= p.cols) v[j] = 0.0f;
    }
  }
  put8(static_cast<T*>(u.out) + row * u.ld + e * 8LL, v, u.ld - e * 8LL >= 8, u.ld - e * 8LL);
}
// Two arrays: the second one's workgroups from `second` on
struct Unpacks { Unpack u[2]; long long second; };
__global__ __launch_bounds__(256) void unpack_kernel(Unpacks a, long long first) {
  const long long block = first + blockIdx.x;
  const bool other = block >= a.second;
  const Unpack& u = a.u[other ? 1 : 0];
  const long long base = (other ? block - a.second : block) * 256;
  if (u.from.format == MX8) { if (u.type) unpack<__bf16, MX8>(u, base); else unpack<float, MX8>(u, base); }
  else { if (u.type) unpack<__bf16, MX4>(u, base); else unpack<float, MX4>(u, base); }
}

// out[row][0 .. ld) <- X rounded to bf16, zeros from cols on (ld a multiple of 8)
template <typename T>
__global__ __launch_bounds__(256) void round_kernel(const T* X, __bf16* out, long long rows, long long cols, long long ld, long long first) {
  const unsigned per = (unsigned)(ld / 8);
  const long long base = (first + blockIdx.x) * 256;
  const unsigned off = (unsigned)(base % per) + threadIdx.x;
  const long long row = base / per + off / per;
  if (row >= rows) return;
  const long long k = (off % per) * 8LL, left = cols - k;
  float v[8];
  if (left >= 8) {
    load8(X + row * cols + k, v);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = j < left ? widen(X[row * cols + k + j]) : 0.0f;
  }
  store8(out + row * ld + k, v);
}
template <typename F> hipError_t in_launches(long long threads, F launch) {
  const long long blocks = (threads + 255) / 256;
  for (long long b = 0; b < blocks; b += MOST_BLOCKS) launch(dim3((unsigned)(blocks - b < MOST_BLOCKS ? blocks - b : MOST_BLOCKS)), b);
  return hipGetLastError();
}

// ------------------------------------------------------------------------------------------ both operands in 4 bits
typedef int int8v __attribute__((ext_vector_type(8)));
typedef unsigned uint4v __attribute__((ext_vector_type(4)));
// One operand's codes or scales: rows `ld` bytes apart
struct Codes {
  const char* p;
  const char* scales;
  long long rows;
};
struct FourArgs {
  Codes A, B;                // X and W
  Epilogue e;
  long long I, J, pitch;     // pitch: bytes of a row of codes of either
  int slabs, per;            // of the contraction; of one workgroup
  float* partial;            // several workgroups share a tile: their sums
};
template <int STEP> __device__ __forceinline__ void multiply4(uint4v a, uint4v b, unsigned sa, unsigned sb, floatx16& c) {
  const int8v x = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0}, y = {(int)b[0], (int)b[1], (int)b[2], (int)b[3], 0, 0, 0, 0};
  c = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x, y, c, 4, 4, STEP, (int)sa, STEP, (int)sb);
}

// Tile of BT x BT outputs, four wavefronts with a quarter each.  A slab is 256 k: 128 bytes of a row, in LDS in the order piece ^ (row / 2 & 7),
// as the larger types' (so that 16 rows' pieces of one k meet different banks), and 8 scales of a row, one behind the other as they lie in memory.
// While one slab is multiplied the next one is on its way.  Bound by what a compute unit takes from L2, 68 KB a slab of 256 in 1.9 us where its matrix
// instructions take 0.9; and by the epilogue of two rounds of tiles, whose residual and results come from and go to memory with nothing beside them:
// 8192 x 4096 x 4096 bf16 with tanh and residual 115 us, 61 of them in the slabs, 8192^3 311 us (3.5 PFLOP/s).  Slabs of 128 k, four of them on their way: 72 us where
// these take 61, as rows of 64 bytes arrive no faster than those of 128.  (The 8-bit matrix instructions are no way to more exact activations: they align
// the products of an instruction to the largest and drop what is 2^-12 of it; those of 4-bit values lose nothing.)
template <int BT, typename OT>
__global__ __launch_bounds__(256, BT == 256 ? 1 : 2) void product_four_kernel(FourArgs a) {
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  constexpr int T = BT / 64, NL = BT / 32, CODES = BT * 128, SC = BT * 8 < 1024 ? 1024 : BT * 8, PLACE = 2 * (CODES + SC);     // NL: loads of either's codes per wavefront
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), wi = wave >> 1, wj = wave & 1;
  const int c = lane & 31, g = lane >> 5;
  constexpr int GM = 4;                                           // tiles in groups of GM rows of tiles: few panels of both operands at a time
  const long long L = logical_block(), ti = (a.I + BT - 1) / BT, tj = (a.J + BT - 1) / BT;
  const long long group = L / (GM * tj), firstg = group * GM, size = ti - firstg < GM ? ti - firstg : GM, in = L - group * GM * tj;
  const long long i0 = (firstg + in % size) * BT, j0 = in / size * BT;
  const int s0 = (int)blockIdx.y * a.per, slabs = s0 + a.per < a.slabs ? a.per : a.slabs - s0;

  // rows behind the last one read as zeros
  int offA[NL], offB[NL];
#pragma unroll
  for (int i = 0; i < NL; ++i) {
    const int r = wave * (BT / 4) + i * 8 + (lane >> 3), piece = ((lane & 7) ^ ((r >> 1) & 7)) * 16;
    offA[i] = i0 + r < a.I ? (int)(r * a.pitch) + piece : 0x7ffffff0;
    offB[i] = j0 + r < a.J ? (int)(r * a.pitch) + piece : 0x7ffffff0;
  }
  const char *pa = a.A.p + i0 * a.pitch, *pb = a.B.p + j0 * a.pitch;
  const char *qa = a.A.scales + i0 * 8, *qb = a.B.scales + j0 * 8;
  const long long stepA = a.A.rows * 8, stepB = a.B.rows * 8;
  // bytes of a slab's scales, in whole loads (the array has room for that; what belongs to no row meets codes that are zero and results that are not written)
  const unsigned roomA = (unsigned)((a.I - i0 < BT ? a.I - i0 : BT) * 8 + 15) & ~15u, roomB = (unsigned)((a.J - j0 < BT ? a.J - j0 : BT) * 8 + 15) & ~15u;
  const unsigned lds_at = (unsigned)(unsigned long long)(LdsPtr*)lds;
  auto load = [&](int t, int place) {
    const unsigned to = lds_at + place * PLACE;
    const int along = (s0 + t) * 128;
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      to_lds(pa, offA[i], along, 0x7fff0000u, to + (wave * NL + i) * 1024);
      to_lds(pb, offB[i], along, 0x7fff0000u, to + CODES + (wave * NL + i) * 1024);
    }
    // scales: BT rows of 8 bytes are BT / 128 instructions for either operand
    if (wave < SC / 1024) to_lds(qa + (s0 + t) * stepA, wave * 1024 + lane * 16, 0, roomA, to + 2 * CODES + wave * 1024);
    else if (wave - 2 >= 0 && wave - 2 < SC / 1024) to_lds(qb + (s0 + t) * stepB, (wave - 2) * 1024 + lane * 16, 0, roomB, to + 2 * CODES + SC + (wave - 2) * 1024);
  };
  floatx16 acc[T][T];
#pragma unroll
  for (int i = 0; i < T; ++i)
#pragma unroll
    for (int j = 0; j < T; ++j) acc[i][j] = zero16();
  const int rowA = wi * (BT / 2) + c, rowB = wj * (BT / 2) + c, turn = (c >> 1) & 7;
  load(0, 0);
  for (int t = 0; t < slabs; ++t) {
    // the slab has arrived, for all wavefronts, and nobody reads the other place any more
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    if (t + 1 < slabs) load(t + 1, (t + 1) & 1);
    const unsigned char* at = lds + (t & 1) * PLACE;
    unsigned sa[T], sb[T];
#pragma unroll
    for (int i = 0; i < T; ++i) {
      sa[i] = *reinterpret_cast<const unsigned*>(at + 2 * CODES + (rowA + i * 32) * 8 + g * 4);
      sb[i] = *reinterpret_cast<const unsigned*>(at + 2 * CODES + SC + (rowB + i * 32) * 8 + g * 4);
    }
    auto step = [&](auto number) {
      constexpr int STEP = decltype(number)::value;
      uint4v fa[T], fb[T];
#pragma unroll
      for (int i = 0; i < T; ++i) {
        fa[i] = *reinterpret_cast<const uint4v*>(at + (rowA + i * 32) * 128 + (((2 * STEP + g) ^ turn) << 4));
        fb[i] = *reinterpret_cast<const uint4v*>(at + CODES + (rowB + i * 32) * 128 + (((2 * STEP + g) ^ turn) << 4));
      }
#pragma unroll
      for (int i = 0; i < T; ++i)
#pragma unroll
        for (int j = 0; j < T; ++j) multiply4<STEP>(fb[j], fa[i], sb[j], sa[i], acc[i][j]);      // (B first: a lane has four columns of a row, see the end)
    };
    step(std::integral_constant<int, 0>{});
    step(std::integral_constant<int, 1>{});
    step(std::integral_constant<int, 2>{});
    step(std::integral_constant<int, 3>{});
  }
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");

  // Through LDS, 32 rows of the wavefront's quarter at a time, so that a lane has eight entries of a row in its hands
  constexpr int W = BT / 2, PITCH = W + 4, STEP = 512 / W, IT = 32 / STEP;
  const int lc = lane % (W / 8) * 8, lr = lane / (W / 8);
  const long long col = j0 + wj * W + lc, n = a.I * a.J;
  const bool whole = col + 8 <= a.J, residual = a.e.R && whole;
  const bool inside = i0 + BT <= a.I && j0 + BT <= a.J && !a.partial;
  float bias[8] = {};
  if (a.e.bias && !a.partial) {
#pragma unroll
    for (int k = 0; k < 8; ++k) bias[k] = a.e.bias[col + k < a.J ? col + k : a.J - 1];
  }
#pragma unroll 1
  for (int i = 0; i < T; ++i) {
    const long long row0 = i0 + wi * W + i * 32 + lr;
    Raw8<OT> ahead[IT];
    if (inside && residual) {
#pragma unroll
      for (int k = 0; k < IT; ++k) ahead[k].load(static_cast<const OT*>(a.e.R) + (row0 + k * STEP) * a.J + col);
    }
    float* strip = reinterpret_cast<float*>(lds) + (wave * 2 + (i & 1)) * 32 * PITCH;
#pragma unroll
    for (int m = 0; m < T; ++m) {
      if (m != i) continue;                                       // (registers have no index)
#pragma unroll
      for (int j = 0; j < T; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          *reinterpret_cast<floatx4*>(strip + c * PITCH + j * 32 + 8 * q + 4 * g) =
              floatx4{acc[m][j][4 * q], acc[m][j][4 * q + 1], acc[m][j][4 * q + 2], acc[m][j][4 * q + 3]};
    }
    __builtin_amdgcn_wave_barrier();
    const float* from = strip + lr * PITCH + lc;
    if (inside) {
      auto rows = [&](auto kind) {
        constexpr int KIND = decltype(kind)::value;
#pragma unroll
        for (int k = 0; k < IT; ++k) {
          float v[8];
          *reinterpret_cast<floatx4*>(v) = *reinterpret_cast<const floatx4*>(from + k * STEP * PITCH);
          *reinterpret_cast<floatx4*>(v + 4) = *reinterpret_cast<const floatx4*>(from + k * STEP * PITCH + 4);
          finish8_whole<OT, KIND>(a.e, (row0 + k * STEP) * a.J + col, v, bias, ahead[k]);
        }
      };
      if (a.e.act == ACT_TANH) rows(std::integral_constant<int, ACT_TANH>{});
      else if (a.e.act == ACT_RELU) rows(std::integral_constant<int, ACT_RELU>{});
      else rows(std::integral_constant<int, ACT_IDENT>{});
    } else {
#pragma unroll 1
      for (int k = 0; k < IT; ++k) {
        const long long row = row0 + k * STEP, at = row * a.J + col;
        if (row >= a.I) continue;
        Raw8<OT> r = {};
        if (residual && !a.partial) r.load(static_cast<const OT*>(a.e.R) + at);
        float v[8];
        *reinterpret_cast<floatx4*>(v) = *reinterpret_cast<const floatx4*>(from + k * STEP * PITCH);
        *reinterpret_cast<floatx4*>(v + 4) = *reinterpret_cast<const floatx4*>(from + k * STEP * PITCH + 4);
        if (a.partial) put8(a.partial + blockIdx.y * n + at, v, whole, a.J - col);
        else finish8<OT>(a.e, at, v, bias, r, whole, a.J - col);
      }
    }
    __builtin_amdgcn_wave_barrier();
  }
}
constexpr size_t four_lds(int bt) {
  const int sc = bt * 8 < 1024 ? 1024 : bt * 8, slabs = 4 * (bt * 128 + sc), strips = 8 * 32 * (bt / 2 + 4) * 4;
  return slabs > strips ? slabs : strips;
}

struct FourPlan { int bt, parts; };
// The tile and the number of workgroups that share its contraction whose time is estimated lowest
FourPlan four_plan(long long I, long long J, int slabs) {
  FourPlan p = {};
  double best = 0.0;
  for (int bt = 256; bt >= 64; bt /= 2) {
    const long long tiles = (I + bt - 1) / bt * ((J + bt - 1) / bt);
    if (tiles > (1LL << 24) - 1) continue;
    const int fit = bt == 256 ? 1 : bt == 128 ? 2 : 4;            // workgroups on a compute unit
    const double slab = bt == 256 ? 1.5 : bt == 128 ? 0.6 : 0.3, ends = bt == 256 ? 20.0 : bt == 128 ? 5.0 : 3.0;
    for (int parts = 1; parts <= 32 && parts <= slabs && (parts == 1 || tiles * parts <= 1024); ++parts) {
      const int per = (slabs + parts - 1) / parts;
      if ((slabs + per - 1) / per != parts) continue;
      const double rounds = (double)((tiles * parts + 255) / 256);
      const double join = parts > 1 ? 4.0 + (double)I * J * 8.0 * parts / 4.0e6 : 0.0;
      const double us = rounds * per * slab + ends * (rounds > fit ? rounds / fit : 1.0) + join;
      if (best == 0.0 || us < best) { best = us; p.bt = bt; p.parts = parts; }
    }
  }
  return p;
}
template <int BT, typename OT>
hipError_t launch_four_tiles(const FourArgs& a, int parts, hipStream_t s) {
  static LdsOptIn opt;
  const hipError_t e = opt.raise(reinterpret_cast<const void*>(&product_four_kernel<BT, OT>), four_lds(BT));
  if (e != hipSuccess) return e;
  const long long tiles = (a.I + BT - 1) / BT * ((a.J + BT - 1) / BT);
  hipLaunchKernelGGL((product_four_kernel<BT, OT>), dim3((unsigned)tiles, (unsigned)parts), dim3(256), four_lds(BT), s, a);
  return hipGetLastError();
}
template <typename OT>
hipError_t launch_four(const FourArgs& a, const FourPlan& p, hipStream_t s) {
  return p.bt == 256 ? launch_four_tiles<256, OT>(a, p.parts, s) : p.bt == 128 ? launch_four_tiles<128, OT>(a, p.parts, s) : launch_four_tiles<64, OT>(a, p.parts, s);
}

// ------------------------------------------------------------------------------------------ few bf16 rows on 4-bit weights
struct FewArgs {
  const char* X;             // bf16, rows `ldx` bytes apart of which `row` count, whole 16-byte pieces
  const char* W;
  const char* scales;
  Epilogue e;
  long long M, F, ldx, pitch;
  int row, slabs, per;       // slabs of the contraction; of one workgroup
  float* partial;
};
template <int SEL> __device__ __forceinline__ void widen2(unsigned c, float scale, bf16x8& v) {
  const bf16x2 p = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, scale, SEL);
  v[2 * SEL] = p[0];
  v[2 * SEL + 1] = p[1];
}
// At most 16 FB rows on many weights.  Bound by reading the weights once: a workgroup has 64 of their rows, 16 for each wavefront, and slabs of 256 k
// of them, of their scales and of all of X on their way into LDS, PLACES of them in turn.  A lane takes a whole block of 32 codes of its row and widens
// it to bf16 (exact) for four matrix instructions; their k are in another order, which is X's too.
// 1 row on 32768 x 4096 weights: 71 MB in 13.4 us with its launch, 5.3 TB/s (unpacked to bf16 first, and multiplied by the kernel for few bf16 rows: 110).  X through
// LDS for four wavefronts at once, because it is more bytes than the weights from 8 rows on.
template <int FB> constexpr int few_places() { return FB == 1 ? 3 : FB == 2 ? 2 : 3; }
template <int FB> constexpr int few_place() { return 64 * 128 + 4 * 1024 + FB * 8192; }
template <int FB>
__global__ __launch_bounds__(256, FB <= 2 ? 2 : 1) void product_few_four_kernel(FewArgs a, int first) {
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  constexpr int PLACES = few_places<FB>(), PLACE = few_place<FB>(), SCALES = 64 * 128, XS = SCALES + 4096, LOADS = 3 + 2 * FB;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), r16 = lane & 15, g = lane >> 4;
  const long long j0 = ((long long)first + logical_block()) * 64;
  const int s0 = (int)blockIdx.y * a.per, slabs = s0 + a.per < a.slabs ? a.per : a.slabs - s0;
  // rows behind the last one, and pieces behind the end of X's, read as zeros
  int offW[2], offX[2 * FB], pieceX[2 * FB];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int r = wave * 16 + 8 * h + (lane >> 3), piece = ((lane & 7) ^ ((r >> 1) & 7)) * 16;
    offW[h] = j0 + r < a.F ? (int)(r * a.pitch) + piece : 0x7ffffff0;
  }
  // X's instruction n of 8 FB: 8 rows of one panel of 64 k; wavefront w takes 2 FB w ..
#pragma unroll
  for (int i = 0; i < 2 * FB; ++i) {
    const int n = wave * 2 * FB + i, block = n >> 3, panel = n >> 1 & 3, r = 8 * (n & 1) + (lane >> 3);
    pieceX[i] = panel * 128 + ((lane & 7) ^ ((r >> 1) & 7)) * 16;
    offX[i] = block * 16 + r < a.M ? (int)((block * 16 + r) * a.ldx) + pieceX[i] : 0x7ffffff0;
  }
  const char* pw = a.W + j0 * a.pitch;
  const char* ps = a.scales + (j0 + wave * 16) * 8;
  const unsigned room = j0 + wave * 16 < a.F ? (unsigned)((a.F - j0 - wave * 16 < 16 ? a.F - j0 - wave * 16 : 16) * 8 + 15) & ~15u : 0u;
  const unsigned lds_at = (unsigned)(unsigned long long)(LdsPtr*)lds;
  auto load = [&](int t) {
    const unsigned to = lds_at + t % PLACES * PLACE;
    const int k = s0 + t;
#pragma unroll
    for (int h = 0; h < 2; ++h) to_lds(pw, offW[h], k * 128, 0x7fff0000u, to + wave * 2048 + h * 1024);
    to_lds(ps + (long long)k * a.F * 8, lane * 16, 0, room, to + SCALES + wave * 1024);
#pragma unroll
    for (int i = 0; i < 2 * FB; ++i)
      to_lds(a.X, k * 512 + pieceX[i] < a.row ? offX[i] : 0x7ffffff0, k * 512, 0x7fff0000u, to + XS + (wave * 2 * FB + i) * 1024);
  };
  floatx4 acc[FB];
#pragma unroll
  for (int i = 0; i < FB; ++i) acc[i] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
  unsigned nans = 0;                 // whether a block of this lane's row is NaN
#pragma unroll
  for (int t = 0; t < PLACES - 1; ++t)
    if (t < slabs) load(t);
  const int turn = (r16 >> 1) & 7;
  for (int t = 0; t < slabs; ++t) {
    // slab t has arrived, for all wavefronts, and nobody reads the one before it any more
    if (t + PLACES - 2 < slabs) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" :: "n"(LOADS * (PLACES - 2)) : "memory");
    else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    if (t + PLACES - 1 < slabs) load(t + PLACES - 1);
    const unsigned char* at = lds + t % PLACES * PLACE;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint4v codes = *reinterpret_cast<const uint4v*>(at + wave * 2048 + r16 * 128 + (((4 * h + g) ^ turn) << 4));
      const unsigned byte = at[SCALES + wave * 1024 + r16 * 8 + (g & 1) * 4 + 2 * h + (g >> 1)];
      nans |= byte == 255u;
      const float scale = scale_of(byte == 255u ? 127u : byte);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        bf16x8 w;
        widen2<0>(codes[j], scale, w);
        widen2<1>(codes[j], scale, w);
        widen2<2>(codes[j], scale, w);
        widen2<3>(codes[j], scale, w);
#pragma unroll
        for (int b = 0; b < FB; ++b) {
          const bf16x8 x = *reinterpret_cast<const bf16x8*>(at + XS + (b * 4 + 2 * h + (g >> 1)) * 2048 + r16 * 128 + ((((g & 1) * 4 + j) ^ turn) << 4));
          acc[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, w, acc[b], 0, 0, 0);
        }
      }
    }
  }
  nans |= __shfl_xor(nans, 16);
  nans |= __shfl_xor(nans, 32);
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
  // lane: row r16 of the weights, four rows of X
  float* sums = reinterpret_cast<float*>(lds);
  constexpr int PITCH = 64 + 4;
#pragma unroll
  for (int b = 0; b < FB; ++b)
#pragma unroll
    for (int r = 0; r < 4; ++r) sums[(b * 16 + 4 * g + r) * PITCH + wave * 16 + r16] = nans ? NAN : acc[b][r];
  __syncthreads();
  for (int n = threadIdx.x; n < FB * 16 * 64; n += 256) {
    const int m = n >> 6, f = n & 63;
    if (m >= a.M || j0 + f >= a.F) continue;
    const float v = sums[m * PITCH + f];
    const long long col = j0 + f, to = m * a.F + col;
    if (a.partial) a.partial[blockIdx.y * a.M * a.F + to] = v;
    else if (a.e.otype) finish<__bf16>(a.e, to, col, v);
    else finish<float>(a.e, to, col, v);
  }
}
template <int FB>
hipError_t launch_few_four(const FewArgs& a, int parts, hipStream_t s) {
  static LdsOptIn opt;
  constexpr size_t smem = few_places<FB>() * few_place<FB>();
  const hipError_t e = opt.raise(reinterpret_cast<const void*>(&product_few_four_kernel<FB>), smem);
  if (e != hipSuccess) return e;
  const long long blocks = (a.F + 63) / 64;
  for (long long b = 0; b < blocks; b += MOST_BLOCKS)
    hipLaunchKernelGGL(product_few_four_kernel<FB>, dim3((unsigned)(blocks - b < MOST_BLOCKS ? blocks - b : MOST_BLOCKS), (unsigned)parts), dim3(256), smem, s, a,
                       (int)b);
  return hipGetLastError();
}
// Workgroups that share the contraction where there are fewer than one for each of the 256 compute units, two slabs each at least
int few_parts(long long F, int slabs) {
  const long long blocks = (F + 63) / 64;
  if (blocks >= 256) return 1;
  const long long want = (256 + blocks - 1) / blocks, most = slabs / 2 > 1 ? slabs / 2 : 1, parts = want < most ? want : most;
  const int per = (int)((slabs + parts - 1) / parts);
  return (slabs + per - 1) / per;
}

// ------------------------------------------------------------------------------------------ bf16 rows on 4-bit weights
constexpr long long FEW = 64;
// (whole 16-byte pieces of rows, and offsets of 31 bits)
inline bool bf16_in_place(const PackedProduct& q) { return q.xtype && q.K % 8 == 0; }
struct WidePlaces { size_t W, X, bytes; long long ld; Product p; };
// The weights unpacked to bf16 planes in the workspace, and the product of planes
WidePlaces wide_places(const PackedProduct& q, char* base) {
  WidePlaces w = {};
  w.ld = (q.K + 63) / 64 * 64;
  w.W = 0;
  w.X = up((size_t)q.F * w.ld * 2);
  w.bytes = w.X + (q.xtype ? 0 : up((size_t)q.M * w.ld * 2));
  w.p.e = q.e;
  w.p.I = q.M; w.p.J = q.F; w.p.Kc = q.K;
  w.p.A = Operand{q.xtype ? q.X : base + w.X, nullptr, q.xtype ? q.K : w.ld, 1, 0, !q.xtype, 1, 0};
  w.p.B = Operand{base + w.W, nullptr, w.ld, 1, 0, 1, 1, 0};
  return w;
}

}  // namespace

size_t packed_bytes(long long rows, long long cols, int format) {
  const Packed p = packed_view(rows, cols, format, nullptr);
  return up((size_t)rows * p.pitch) + up((size_t)rows * p.slabs * 8);
}
Packed packed_view(long long rows, long long cols, int format, void* at) {
  Packed p = {};
  p.rows = rows; p.cols = cols; p.format = format;
  p.slabs = (cols + SLAB - 1) / SLAB;
  p.pitch = p.slabs * (format == MX4 ? SLAB / 2 : SLAB);
  p.codes = static_cast<unsigned char*>(at);
  p.scales = p.codes + up((size_t)rows * p.pitch);
  return p;
}
hipError_t launch_pack(const Packed& p, const void* X, int type, hipStream_t s) {
  return in_launches(p.rows * p.slabs * (SLAB / 8), [&](dim3 grid, long long b) {
    if (type && p.format == MX8) hipLaunchKernelGGL((pack_kernel<__bf16, MX8>), grid, dim3(256), 0, s, p, static_cast<const __bf16*>(X), b);
    else if (type) hipLaunchKernelGGL((pack_kernel<__bf16, MX4>), grid, dim3(256), 0, s, p, static_cast<const __bf16*>(X), b);
    else if (p.format == MX8) hipLaunchKernelGGL((pack_kernel<float, MX8>), grid, dim3(256), 0, s, p, static_cast<const float*>(X), b);
    else hipLaunchKernelGGL((pack_kernel<float, MX4>), grid, dim3(256), 0, s, p, static_cast<const float*>(X), b);
  });
}
hipError_t launch_unpack(const Unpack* arrays, int n, hipStream_t s) {
  Unpacks a = {};
  long long blocks[2] = {};
  for (int i = 0; i < n; ++i) {
    a.u[i] = arrays[i];
    blocks[i] = (arrays[i].from.rows * ((arrays[i].ld + 7) / 8) + 255) / 256;
  }
  a.second = blocks[0];
  return in_launches((blocks[0] + blocks[1]) * 256, [&](dim3 grid, long long b) { hipLaunchKernelGGL(unpack_kernel, grid, dim3(256), 0, s, a, b); });
}

size_t packed_product_workspace(const PackedProduct& q) {
  if (q.xformat == MX4) {
    const Packed x = packed_view(q.M, q.K, MX4, nullptr);
    const FourPlan f = four_plan(q.M, q.F, (int)x.slabs);
    return up(packed_bytes(q.M, q.K, MX4)) + (f.parts > 1 ? (size_t)f.parts * q.M * q.F * sizeof(float) : 0);
  }
  if (q.M <= FEW) {
    const int parts = few_parts(q.F, (int)packed_view(q.F, q.K, MX4, nullptr).slabs);
    return (bf16_in_place(q) ? 0 : up((size_t)q.M * ((q.K + 7) / 8 * 8) * 2)) + (parts > 1 ? (size_t)parts * q.M * q.F * sizeof(float) : 0);
  }
  const WidePlaces w = wide_places(q, nullptr);
  return w.bytes + product_workspace(w.p);
}
hipError_t launch_packed_product(const PackedProduct& q, void* ws, hipStream_t s) {
  char* base = static_cast<char*>(ws);
  const Packed W = packed_view(q.F, q.K, MX4, const_cast<void*>(q.W));
  if (q.xformat == MX4) {
    const Packed X = packed_view(q.M, q.K, MX4, ws);
    const FourPlan f = four_plan(q.M, q.F, (int)X.slabs);
    hipError_t e = launch_pack(X, q.X, q.xtype, s);
    if (e != hipSuccess) return e;
    FourArgs a = {};
    a.A = Codes{reinterpret_cast<const char*>(X.codes), reinterpret_cast<const char*>(X.scales), q.M};
    a.B = Codes{reinterpret_cast<const char*>(W.codes), reinterpret_cast<const char*>(W.scales), q.F};
    a.e = q.e;
    a.I = q.M; a.J = q.F; a.pitch = X.pitch;
    a.slabs = (int)X.slabs;
    a.per = (a.slabs + f.parts - 1) / f.parts;
    a.partial = f.parts > 1 ? reinterpret_cast<float*>(base + up(packed_bytes(q.M, q.K, MX4))) : nullptr;
    e = q.e.otype ? launch_four<__bf16>(a, f, s) : launch_four<float>(a, f, s);
    return e != hipSuccess || f.parts == 1 ? e : join_parts(q.e, a.partial, f.parts, q.M, q.F, s);
  }
  // X as bf16 with rows of ld entries, zeros behind the last one
  auto lay_out = [&](char* to, long long ld) {
    return in_launches(q.M * (ld / 8), [&](dim3 grid, long long b) {
      __bf16* out = reinterpret_cast<__bf16*>(to);
      if (q.xtype) hipLaunchKernelGGL(round_kernel<__bf16>, grid, dim3(256), 0, s, static_cast<const __bf16*>(q.X), out, q.M, q.K, ld, b);
      else hipLaunchKernelGGL(round_kernel<float>, grid, dim3(256), 0, s, static_cast<const float*>(q.X), out, q.M, q.K, ld, b);
    });
  };
  if (q.M <= FEW) {
    const long long ld = (q.K + 7) / 8 * 8;
    const size_t laid = bf16_in_place(q) ? 0 : up((size_t)q.M * ld * 2);
    hipError_t e = laid ? lay_out(base, ld) : hipSuccess;
    if (e != hipSuccess) return e;
    const int parts = few_parts(q.F, (int)W.slabs);
    FewArgs a = {};
    a.X = laid ? base : static_cast<const char*>(q.X);
    a.W = reinterpret_cast<const char*>(W.codes);
    a.scales = reinterpret_cast<const char*>(W.scales);
    a.e = q.e;
    a.M = q.M; a.F = q.F; a.ldx = ld * 2; a.pitch = W.pitch;
    a.row = (int)(ld * 2);
    a.slabs = (int)W.slabs;
    a.per = (a.slabs + parts - 1) / parts;
    a.partial = parts > 1 ? reinterpret_cast<float*>(base + laid) : nullptr;
    e = q.M <= 16 ? launch_few_four<1>(a, parts, s) : q.M <= 32 ? launch_few_four<2>(a, parts, s) : q.M <= 48 ? launch_few_four<3>(a, parts, s)
                                                                                                  : launch_few_four<4>(a, parts, s);
    return e != hipSuccess || parts == 1 ? e : join_parts(q.e, a.partial, parts, q.M, q.F, s);
  }
  const WidePlaces w = wide_places(q, base);
  const Unpack weights = {W, base + w.W, 1, w.ld};
  hipError_t e = launch_unpack(&weights, 1, s);
  if (e == hipSuccess && !q.xtype) e = lay_out(base + w.X, w.ld);
  return e != hipSuccess ? e : launch_product(w.p, base + w.bytes, s);
}

}  // namespace mgrit
