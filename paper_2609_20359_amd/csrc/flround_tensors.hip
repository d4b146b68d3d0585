// flround_tensors.hip -- gfx950 kernels of AdamW over many tensors, with moments in 32
// or in 8 bits.
//
// A stream, bound by memory: a wave takes a unit of 512 elements of one tensor, 4 of
// each half of it to a lane, all of its loads first.  The tensors' addresses are in the
// launch's arguments; a wave finds its tensor by comparing its number with all of their
// first units at once.
//
// States in 8 bits.  A block of 64 elements (16 lanes) shares an exponent byte b, that of
// its largest magnitude.  A code is the top of the element's fp32 pattern after scaling
// by 2^(15 - b) (first moment: a sign, 4 bits of exponent, 3 of mantissa) or 2^(31 - b)
// (second moment, 5 and 3): what the scaling takes into fp32's subnormal range is the
// code's too.  So coding is a scaling, an addition of the rounding and a shift, decoding
// a shift and a scaling, both exact: an unchanged value is held unchanged even when its
// block's exponent moves.
//   - Rounding to nearest stops a slow average: the second moment changes by 1 - beta2 of
//     itself in a step, a code's step is 6 to 12 %.  With random bits below the code
//     instead of half a step, the expected value of what is held is the moment.
//   - A second moment above 0 is never held as 0: the next step would divide by eps.
#include "flr_device.h"
#include "flr_launch.h"
#include "flr_tensors.h"

namespace flr {
namespace {

constexpr int kHalf = kUnit / 2;
constexpr int kTopM = 15, kTopV = 31;   // the largest exponent field of a code
constexpr int kLowExp = 12;             // so that a code's step is above fp32's smallest

typedef f32x4 f32x4_at4 __attribute__((aligned(4)));
typedef u32x2 u32x2_at2 __attribute__((aligned(2)));

// Random bits of element i: two rounds of shifts and products, with constants of a
// published search for little bias.
__device__ __forceinline__ uint32_t random_bits(const TensorsArgs& a, int64_t i) {
  uint32_t x = (uint32_t)i ^ a.key_lo;
  x = (x ^ (x >> 16)) * 0x7FEB352Du;
  x ^= (uint32_t)(i >> 32) + a.key_hi;
  x = (x ^ (x >> 15)) * 0x846CA68Bu;
  return x ^ (x >> 16);
}

template <int kCtrl>
__device__ __forceinline__ uint32_t max_dpp(uint32_t x) {
  const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, kCtrl, 0xF, 0xF, true);
  return x > o ? x : o;
}

// The exponent byte of a block whose lanes hold four elements each.
__device__ __forceinline__ uint32_t block_exp(const float* x) {
  uint32_t most = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint32_t b = __float_as_uint(x[e]) & 0x7FFFFFFFu;
    if (b < 0x7F800000u && b > most) most = b;
  }
  most = max_dpp<0xB1>(most);    // lane ^ 1
  most = max_dpp<0x4E>(most);    // lane ^ 2
  most = max_dpp<0x141>(most);   // the other half of 8
  most = max_dpp<0x140>(most);   // the other half of 16
  // (a mantissa over 1.75 would be rounded to a code that stands for no number)
  const uint32_t b = (most >> 23) + ((most & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return b < kLowExp ? kLowExp : b;
}

// The code of x in a block of exponent b; `bits`: 20 random ones.
template <int kTop, bool kDrawn>
__device__ __forceinline__ uint32_t code_of(float x, int b, uint32_t bits) {
  const uint32_t w = __float_as_uint(x), abs = w & 0x7FFFFFFFu;
  const uint32_t y = __float_as_uint(__builtin_amdgcn_ldexpf(__uint_as_float(abs), kTop - b));
  uint32_t c = (y + (kDrawn ? bits : 0x7FFFFu + ((y >> 20) & 1))) >> 20;
  if (kTop == kTopV && c == 0 && abs != 0) c = 1;
  if (abs >= 0x7F800000u) c = 8 * kTop + 7;
  return kTop == kTopM ? c | (w >> 31) << 7 : c;
}

template <int kTop>
__device__ __forceinline__ float value_of(uint32_t c, int b) {
  const uint32_t k = kTop == kTopM ? c & 127 : c;
  uint32_t w = k == 8 * kTop + 7 ? 0x7FC00000u : k << 20;
  if (kTop == kTopM) w |= (c & 128) << 24;
  return __builtin_amdgcn_ldexpf(__uint_as_float(w), b - kTop);
}

// Four codes of each half, whose exponents the lanes of a block share.
template <int kTop>
__device__ __forceinline__ void load_codes(const uint8_t* codes, const uint8_t* exps, int64_t unit,
                                           int lane, uint32_t w[2], uint32_t b[2]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    w[h] = *reinterpret_cast<const uint32_t*>(codes + unit * kUnit + h * kHalf + lane * 4);
    b[h] = exps[unit * (kUnit / kStateBlock) + h * 4 + lane / 16];
  }
}

template <int kTop>
__device__ __forceinline__ void values(const uint32_t w[2], const uint32_t b[2], float x[8]) {
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int e = 0; e < 4; ++e)
      x[4 * h + e] = value_of<kTop>((w[h] >> (8 * e)) & 255, (int)b[h]);
}

template <int kTop, bool kDrawn>
__device__ __forceinline__ void store_codes(uint8_t* codes, uint8_t* exps, int64_t unit, int lane,
                                            const float x[8], const uint32_t bits[8]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint32_t b = block_exp(x + 4 * h);
    uint32_t w = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      w |= code_of<kTop, kDrawn>(x[4 * h + e], (int)b, bits[4 * h + e]) << (8 * e);
    *reinterpret_cast<uint32_t*>(codes + unit * kUnit + h * kHalf + lane * 4) = w;
    if ((lane & 15) == 0) exps[unit * (kUnit / kStateBlock) + h * 4 + lane / 16] = (uint8_t)b;
  }
}

// Elements lane * 4 .. + 3 of each half of a unit of which n (from the unit's start) are
// the tensor's; `rest` behind them.
__device__ __forceinline__ void load_f32(const float* p, int64_t n, int lane, float x[8],
                                         float rest = 0.f) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int at = h * kHalf + lane * 4;
    if (at + 4 <= n) {
      const f32x4 w = *reinterpret_cast<const f32x4_at4*>(p + at);
      x[4 * h] = w.x, x[4 * h + 1] = w.y, x[4 * h + 2] = w.z, x[4 * h + 3] = w.w;
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) x[4 * h + e] = at + e < n ? p[at + e] : rest;
    }
  }
}

__device__ __forceinline__ void load_bf16(const uint16_t* p, int64_t n, int lane, float x[8]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int at = h * kHalf + lane * 4;
    if (at + 4 <= n) {
      const u32x2 w = *reinterpret_cast<const u32x2_at2*>(p + at);
      x[4 * h] = bf16_lo(w.x), x[4 * h + 1] = bf16_hi(w.x);
      x[4 * h + 2] = bf16_lo(w.y), x[4 * h + 3] = bf16_hi(w.y);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        x[4 * h + e] = at + e < n ? __uint_as_float((uint32_t)p[at + e] << 16) : 0.f;
    }
  }
}

__device__ __forceinline__ void store_f32(float* p, int64_t n, int lane, const float x[8]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int at = h * kHalf + lane * 4;
    if (at + 4 <= n) {
      *reinterpret_cast<f32x4_at4*>(p + at) =
          f32x4{x[4 * h], x[4 * h + 1], x[4 * h + 2], x[4 * h + 3]};
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (at + e < n) p[at + e] = x[4 * h + e];
    }
  }
}

__device__ __forceinline__ void store_bf16(uint16_t* p, int64_t n, int lane, const float x[8]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int at = h * kHalf + lane * 4;
    if (at + 4 <= n) {
      *reinterpret_cast<u32x2_at2*>(p + at) =
          u32x2{pack_bf16x2(x[4 * h], x[4 * h + 1]), pack_bf16x2(x[4 * h + 2], x[4 * h + 3])};
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (at + e < n) p[at + e] = (uint16_t)to_bf16(x[4 * h + e]);
    }
  }
}

template <bool kGradF32, int kBits, bool kDrawn>
__global__ void __launch_bounds__(256) k_tensors(const TensorsArgs a, int64_t units) {
  const int lane = threadIdx.x & 63;
  const int64_t u = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  if (u >= units) return;
  // tensors that begin behind the first one, up to this unit
  static_assert(kMaxTensors > 64 && kMaxTensors <= 128);
  const int more = lane < kMaxTensors - 64 ? a.first[lane + 65] : INT32_MAX;
  const int k = __popcll(__ballot(a.first[lane + 1] <= u)) + __popcll(__ballot(more <= u));
  const int64_t from = (u - a.first[k]) * kUnit;
  const int64_t n = a.numel[k] - from;
  const int64_t unit = a.unit0 + u;
  float* master = a.master[k] + from;
  float p[8], g[8], m[8], v[8];
  load_f32(master, n, lane, p);
  if constexpr (kGradF32)
    load_f32(static_cast<const float*>(a.grad[k]) + from, n, lane, g);
  else
    load_bf16(static_cast<const uint16_t*>(a.grad[k]) + from, n, lane, g);
  float* mf = static_cast<float*>(a.state.m) + unit * kUnit;
  float* vf = static_cast<float*>(a.state.v) + unit * kUnit;
  uint8_t* mc = static_cast<uint8_t*>(a.state.m);
  uint8_t* vc = static_cast<uint8_t*>(a.state.v);
  uint32_t wm[2], bm[2], wv[2], bv[2];
  if constexpr (kBits == 32) {
    load_f32(mf, kUnit, lane, m);
    load_f32(vf, kUnit, lane, v);
  } else {
    load_codes<kTopM>(mc, a.state.m_exp, unit, lane, wm, bm);
    load_codes<kTopV>(vc, a.state.v_exp, unit, lane, wv, bv);
    values<kTopM>(wm, bm, m);
    values<kTopV>(wv, bv, v);
  }
  const float decay = (a.decay[k / 32] >> (k % 32)) & 1 ? a.s.decay : 1.0f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    p[e] = p[e] * decay;
    g[e] = g[e] * a.grad_scale;
  }
  adam8(a.s, g, p, m, v);
  store_f32(master, n, lane, p);
  if (a.working[k]) store_bf16(a.working[k] + from, n, lane, p);
  if constexpr (kBits == 32) {
    store_f32(mf, kUnit, lane, m);
    store_f32(vf, kUnit, lane, v);
  } else {
    uint32_t rm[8], rv[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if constexpr (kDrawn) {
        const uint32_t x = random_bits(a, unit * kUnit + (e / 4) * kHalf + lane * 4 + e % 4);
        rm[e] = x >> 12;
        rv[e] = (x * 0x9E3779B1u) >> 12;
      }
    }
    store_codes<kTopM, kDrawn>(mc, a.state.m_exp, unit, lane, m, rm);
    store_codes<kTopV, kDrawn>(vc, a.state.v_exp, unit, lane, v, rv);
  }
}

template <bool kTo8>
__global__ void __launch_bounds__(256) k_state_convert(const StateDev narrow, const StateDev wide,
                                                       int64_t units) {
  const int lane = threadIdx.x & 63;
  const int64_t u = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  if (u >= units) return;
  float* mf = static_cast<float*>(wide.m) + u * kUnit;
  float* vf = static_cast<float*>(wide.v) + u * kUnit;
  uint8_t* mc = static_cast<uint8_t*>(narrow.m);
  uint8_t* vc = static_cast<uint8_t*>(narrow.v);
  float m[8], v[8];
  if constexpr (kTo8) {
    load_f32(mf, kUnit, lane, m);
    load_f32(vf, kUnit, lane, v);
    const uint32_t none[8] = {};
    store_codes<kTopM, false>(mc, narrow.m_exp, u, lane, m, none);
    store_codes<kTopV, false>(vc, narrow.v_exp, u, lane, v, none);
  } else {
    uint32_t wm[2], bm[2], wv[2], bv[2];
    load_codes<kTopM>(mc, narrow.m_exp, u, lane, wm, bm);
    load_codes<kTopV>(vc, narrow.v_exp, u, lane, wv, bv);
    values<kTopM>(wm, bm, m);
    values<kTopV>(wv, bv, v);
    store_f32(mf, kUnit, lane, m);
    store_f32(vf, kUnit, lane, v);
  }
}

}  // namespace

hipError_t launch_tensors(const TensorsArgs& a, int64_t units, hipStream_t st) {
  auto kernel = a.grad_f32 ? (a.state.bits == 32 ? k_tensors<true, 32, false>
                              : a.drawn          ? k_tensors<true, 8, true>
                                                 : k_tensors<true, 8, false>)
                           : (a.state.bits == 32 ? k_tensors<false, 32, false>
                              : a.drawn          ? k_tensors<false, 8, true>
                                                 : k_tensors<false, 8, false>);
  return launch(kernel, dim3((unsigned)((units + 3) / 4)), 256, 0, st, a, units);
}

hipError_t launch_state_convert(const StateDev& from, const StateDev& to, int64_t units,
                                hipStream_t st) {
  const dim3 grid((unsigned)((units + 3) / 4));
  return to.bits == 8 ? launch(k_state_convert<true>, grid, 256, 0, st, to, from, units)
                      : launch(k_state_convert<false>, grid, 256, 0, st, from, to, units);
}

}  // namespace flr
