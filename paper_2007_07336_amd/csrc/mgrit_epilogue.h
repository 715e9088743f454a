// Values, epilogues and loads that the products of the end layers have in common (mgrit_affine.hip, mgrit_packed.hip).
#pragma once
#include "mgrit_device.h"
#include "mgrit_ops.h"

namespace mgrit {

namespace {

// ------------------------------------------------------------------------------------------ values
__device__ __forceinline__ float widen(float v) { return v; }
__device__ __forceinline__ float widen(__bf16 v) { return static_cast<float>(v); }
template <typename T> __device__ __forceinline__ T narrow(float v) { return static_cast<T>(v); }   // to nearest, ties to even

// tanh(z) and 1 - tanh(z)^2 to about 4e-7 relative.  With e = exp(-2 |z|): tanh |z| = (1 - e) / (1 + e), and 1 - tanh^2 =
// 4 e / (1 + e)^2, which loses nothing near saturation; below 0.35, where 1 - e cancels, the odd series up to z^11.  The exponent
// -2 log2(e) |z| is taken in two floats, because an error of it is one of e: rounded once it is 1e-6 off at |z| = 10 and 4e-6 at 40.
// That is enough where results are rounded to bf16, and the second float costs 3 % there (8192 x 4096 x 4096: 254 us without, 261 with it).
template <typename OT>
__device__ __forceinline__ float tanh_with_slope(float z, float* slope) {
  const float a = fabsf(z);
  const float c = 2.885390081777927f, c_rest = (float)(2.885390081777926814 - (double)c), p = a * c;
  float e = __builtin_amdgcn_exp2f(-p);
  // exp2(-p - rest) = e (1 - log(2) rest), rest = a c - p + a c_rest
  if (sizeof(OT) == 4 && e > 0.0f) e -= e * 0.6931471805599453f * __builtin_fmaf(a, c_rest, __builtin_fmaf(a, c, -p));
  const float r = __builtin_amdgcn_rcpf(1.0f + e);
  const float q = z * z;
  const float series = z + z * q * (-0.33333333333f + q * (0.13333333333f + q * (-0.05396825397f + q * (0.02186948854f - q * 0.00886323552f))));
  *slope = 4.0f * e * r * r;
  return a < 0.35f ? series : copysignf((1.0f - e) * r, z);
}

struct Out { float y, d; };
// act(z) and act'(z), for results of type OT; a NaN stays one
template <typename OT>
__device__ __forceinline__ Out activate(float z, int act) {
  Out o;
  if (act == ACT_TANH) {
    o.y = tanh_with_slope<OT>(z, &o.d);
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
  const Out o = activate<OT>(e.bias ? sum + e.bias[col] : sum, e.act);
  const float y = e.scale * o.y;
  out[at] = narrow<OT>(e.R ? static_cast<const OT*>(e.R)[at] + y : y);
  if (e.D) static_cast<OT*>(e.D)[at] = narrow<OT>(e.scale * o.d);
}

// Eight entries of a row, at whatever address: 16-byte accesses of global memory need no alignment.  whole: all eight exist.
typedef __bf16 bf16x8u __attribute__((ext_vector_type(8), aligned(2)));
typedef float floatx4u __attribute__((ext_vector_type(4), aligned(4)));
__device__ __forceinline__ void load8(const float* p, float (&v)[8]) {
  *reinterpret_cast<floatx4*>(v) = *reinterpret_cast<const floatx4u*>(p);
  *reinterpret_cast<floatx4*>(v + 4) = *reinterpret_cast<const floatx4u*>(p + 4);
}
__device__ __forceinline__ void load8(const __bf16* p, float (&v)[8]) {
  const bf16x8 b = *reinterpret_cast<const bf16x8u*>(p);
#pragma unroll
  for (int k = 0; k < 8; ++k) v[k] = widen(b[k]);
}
__device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
  *reinterpret_cast<floatx4u*>(p) = floatx4{v[0], v[1], v[2], v[3]};
  *reinterpret_cast<floatx4u*>(p + 4) = floatx4{v[4], v[5], v[6], v[7]};
}
__device__ __forceinline__ void store8(__bf16* p, const float (&v)[8]) {
  bf16x8 b;
#pragma unroll
  for (int k = 0; k < 8; ++k) b[k] = narrow<__bf16>(v[k]);
  *reinterpret_cast<bf16x8u*>(p) = b;
}
template <typename T> struct Raw8;                               // eight entries as they were loaded
template <> struct Raw8<float> {
  floatx4 a, b;
  __device__ __forceinline__ void load(const float* p) { a = *reinterpret_cast<const floatx4u*>(p); b = *reinterpret_cast<const floatx4u*>(p + 4); }
  __device__ __forceinline__ float at(int k) const { return k < 4 ? a[k & 3] : b[k & 3]; }
};
template <> struct Raw8<__bf16> {
  bf16x8 a;
  __device__ __forceinline__ void load(const __bf16* p) { a = *reinterpret_cast<const bf16x8u*>(p); }
  __device__ __forceinline__ float at(int k) const { return widen(a[k]); }
};
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
// (r: the residual's eight where `whole`, loaded ahead)
template <typename OT>
__device__ __forceinline__ void finish8(const Epilogue& e, long long at, float (&v)[8], const float (&bias)[8], const Raw8<OT>& r, bool whole, long long left) {
  OT* out = static_cast<OT*>(e.out) + at;
  if (!e.fwd) {
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] *= e.scale;
    put8(out, v, whole, left);
    return;
  }
  float d[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const Out o = activate<OT>(v[k] + bias[k], e.act);
    v[k] = e.scale * o.y;
    d[k] = e.scale * o.d;
  }
  if (e.R) {
    const OT* R = static_cast<const OT*>(e.R) + at;
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] += whole ? r.at(k) : k < left ? widen(R[k]) : 0.0f;
  }
  put8(out, v, whole, left);
  if (e.D) put8(static_cast<OT*>(e.D) + at, d, whole, left);
}

// The same of eight that all exist, with the kind of epilogue fixed: an activation of the forward pass, or PLAIN
enum { PLAIN = 3 };
template <typename OT, int KIND>
__device__ __forceinline__ void finish8_whole(const Epilogue& e, long long at, float (&v)[8], const float (&bias)[8], const Raw8<OT>& r) {
  float d[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    if constexpr (KIND == PLAIN) {
      v[k] *= e.scale;
    } else {
      const Out o = activate<OT>(v[k] + bias[k], KIND);
      v[k] = e.scale * o.y;
      d[k] = e.scale * o.d;
    }
  }
  if (KIND != PLAIN && e.R) {
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] += r.at(k);
  }
  store8(static_cast<OT*>(e.out) + at, v);
  if (KIND != PLAIN && e.D) store8(static_cast<OT*>(e.D) + at, d);
}

// ------------------------------------------------------------------------------------------ from memory to LDS
typedef __attribute__((address_space(3))) void LdsPtr;
// 16 bytes per lane from base + each lane's offset + along to LDS address `to` and the 1008 bytes behind it, in lane order; zeros from
// base + room on.  In assembly so that the compiler does not see a load that writes LDS: it would hold back every transposing read
// until all loads have arrived (backward pass of 8192 x 4096 x 4096 bf16: 1781 us).  There is no result register, and what is
// waited for stands in the kernel.
typedef int int4v __attribute__((ext_vector_type(4)));
__device__ __forceinline__ void to_lds(const char* base, int offset, int along, unsigned room, unsigned to) {
  const unsigned long long b = reinterpret_cast<unsigned long long>(base);
  const int4v rsrc = {(int)(unsigned)b, (int)(unsigned)(b >> 32), (int)room, 0x00020000};
  unsigned m0;                       // (an output, so that the compiler knows that it changes; named as overwritten it brings a warning each)
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tbuffer_load_dwordx4 %2, %3, %4 offen lds" : "={m0}"(m0) : "s"(to), "v"(offset), "s"(rsrc), "s"(along) : "memory");
}

}  // namespace

}  // namespace mgrit
