// Device helpers shared by the weight kernels and the 4-bit cache: bf16
// conversions, codes to floats, Eq. 3, and the exact nearest code of a value.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace q4nx {

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// Hides the known bits of a value from the optimizer, so that byte extraction
// of a masked word maps onto v_cvt_f32_ubyte{0..3} (one op per code) instead
// of a per-code AND followed by a convert.
__device__ __forceinline__ uint32_t opaque(uint32_t v) {
  asm volatile("" : "+v"(v));
  return v;
}

__device__ __forceinline__ float bf16_to_f32(uint32_t b) { return __uint_as_float(b << 16); }

__device__ __forceinline__ uint32_t pack_bf16x2(float a, float b) {
  bf16x2 p = __builtin_convertvector((float __attribute__((ext_vector_type(2)))){a, b}, bf16x2);
  return __builtin_bit_cast(uint32_t, p);
}

__device__ __forceinline__ uint16_t f32_to_bf16_bits(float a) {
  return (uint16_t)(pack_bf16x2(a, 0.0f) & 0xFFFFu);
}

// Two code bytes as two float32 values q * 2^-9 (exact) in one conversion.
template <bool HI_WORD>
__device__ __forceinline__ f32x2 codes2_f32(uint32_t bytes) {
  return __builtin_amdgcn_cvt_pk_f32_fp8(bytes, HI_WORD);
}

// Eq. 3 from a scaled code: (q 2^-9) * (d 2^9) is the exact product d*q (both
// scalings are exact powers of two inside the value domain), so one FMA gives
// RN(d*q + m) -- the same bits as the plain definition.
__device__ __forceinline__ float eq3(float q_scaled, float d_times_512, float m) {
  return fmaf(q_scaled, d_times_512, m);
}

// The Eq. 3 levels L_q = fma(q, d, m) are non-decreasing in q, so the exact
// search (quant_code, for the groups the quotient below cannot decide) finds
// the nearest level with two binary searches instead of a scan: c = the number
// of levels below w; the candidates are level c (the first >= w) and the
// first code whose level equals level c-1.
constexpr float kQuantClamp = 1.2676506002282294e30f;  // 2^100

__device__ __forceinline__ uint32_t bf16_rne_flushed(float v) {
  uint32_t b = pack_bf16x2(v, 0.0f) & 0xFFFFu;
  if ((b & 0x7FFFu) < (27u << 7)) b &= 0x8000u;  // |v| < 2^-100 -> signed zero
  return b;
}

// Number of codes q in 0..15 whose level fma(q, d, m) is below v.
__device__ __forceinline__ int levels_below(float v, float d, float m) {
  int c = 0;
#pragma unroll
  for (int s = 8; s >= 1; s >>= 1)
    if (fmaf((float)(c + s - 1), d, m) < v) c += s;
  if (c == 15 && fmaf(15.0f, d, m) < v) c = 16;
  return c;
}

// The exact code of one (clamped) weight; see above.
__device__ __forceinline__ int quant_code(float w, float d, float m) {
  const int cnt = levels_below(w, d, m);
  if (cnt == 0) return 0;
  const float l_lo = fmaf((float)(cnt - 1), d, m);
  // The first code with that level: cnt - 1 unless the level below is the
  // same value (a d small next to m), then the binary search.
  const int q_lo = (cnt == 1 || fmaf((float)(cnt - 2), d, m) < l_lo) ? cnt - 1 : levels_below(l_lo, d, m);
  if (cnt == 16) return q_lo;
  const float l_hi = fmaf((float)cnt, d, m);
  const double dist_hi = (double)l_hi - (double)w;
  const double dist_lo = (double)w - (double)l_lo;
  return dist_hi < dist_lo ? cnt : q_lo;
}

// Where the rounded quotient decides a code: see quantize_kernel.
constexpr float kQuantMaxR = 4194304.0f, kQuantU = 5.9604644775390625e-08f;

}  // namespace q4nx
