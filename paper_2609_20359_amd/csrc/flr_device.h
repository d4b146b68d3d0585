// flr_device.h -- device functions that several of the library's kernels use:
// conversions to and from bf16, and AdamW on 8 elements.
#pragma once

#include "flr_internal.h"

namespace flr {
namespace {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// fp32 -> bf16 bits, round to nearest even; NaN -> quiet NaN, sign kept: the
// conversion instruction (two values at a time), which gives these bits for
// all 2^32 inputs.
__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{lo, hi}, bf16x2));
}

__device__ __forceinline__ uint32_t to_bf16(float x) { return pack_bf16x2(x, 0.f) & 0xFFFFu; }

__device__ __forceinline__ u32x4 pack_bf16x8(const float x[8]) {
  return u32x4{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]),
               pack_bf16x2(x[6], x[7])};
}

// AdamW on 8 elements: p already decayed, g clipped; m, v and p updated.
//
// The division and the two correctly rounded operations before it are a third
// of the step's instructions as the compiler expands them, most of it for
// operands at the ends of the range.  When no lane of the wave has one (kLo,
// kHi below, and s.rbc2, which the host sets when eps and bc2_sqrt allow), the
// same results come cheaper:
//  - sqrt: x * rsq(x) with one correction by its exact residual.  That it is the
//    correctly rounded root rests on the values the instruction returns, so the
//    tests compare every float of the range;
//  - / bc2_sqrt: by its correctly rounded reciprocal and two corrections (the
//    first makes the quotient faithful, the second by Markstein's theorem
//    correctly rounded);
//  - mn / den: reciprocal, one Newton step, two corrections: the operations of
//    the full division where its scaling does nothing.
// Per round: 8B shard (R = 8, A = 4) 29.62 to 29.16 ms, 1 Mi elements (R = 4,
// from cache) 37.8 to 37.1 us; together with the rounding instruction.
constexpr float kMnLo = 0x1p-60f, kMnHi = 0x1p30f, kVnLo = 0x1p-100f, kVnHi = 0x1p60f;

__device__ __forceinline__ void adam8(const AdamScalars& s, const float g[8], float p[8],
                                      float m[8], float v[8]) {
  float m_lo = kMnHi, m_hi = 0.f, v_lo = kVnHi, v_hi = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    m[e] = (s.b1 * m[e]) + (s.omb1 * g[e]);
    v[e] = (s.b2 * v[e]) + (s.omb2 * (g[e] * g[e]));
    const float am = __builtin_fabsf(m[e]);
    m_lo = __builtin_fminf(m_lo, am);
    m_hi = __builtin_fmaxf(m_hi, am);
    v_lo = __builtin_fminf(v_lo, v[e]);
    v_hi = __builtin_fmaxf(v_hi, v[e]);
  }
  // (a NaN is in neither minimum nor maximum; it comes out NaN either way)
  const bool in_range = m_lo >= kMnLo && m_hi <= kMnHi && v_lo >= kVnLo && v_hi <= kVnHi;
  if (s.rbc2 > 0.f && __all(in_range)) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float y = __builtin_amdgcn_rsqf(v[e]);
      float r = v[e] * y;
      r = __builtin_fmaf(__builtin_fmaf(-r, r, v[e]), 0.5f * y, r);
      float q = r * s.rbc2;
      q = __builtin_fmaf(__builtin_fmaf(-s.bc2_sqrt, q, r), s.rbc2, q);
      q = __builtin_fmaf(__builtin_fmaf(-s.bc2_sqrt, q, r), s.rbc2, q);
      const float den = q + s.eps;
      float z = __builtin_amdgcn_rcpf(den);
      z = __builtin_fmaf(__builtin_fmaf(-den, z, 1.0f), z, z);
      float u = m[e] * z;
      u = __builtin_fmaf(__builtin_fmaf(-den, u, m[e]), z, u);
      u = __builtin_fmaf(__builtin_fmaf(-den, u, m[e]), z, u);
      p[e] = p[e] - (s.step_size * u);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float den = (__builtin_sqrtf(v[e]) / s.bc2_sqrt) + s.eps;
      p[e] = p[e] - (s.step_size * (m[e] / den));
    }
  }
}

}  // namespace
}  // namespace flr
