// flround_tensors.hip -- gfx950 kernels of AdamW over many tensors, with moments in 32
// or in 8 bits.
//
// A stream, bound by memory: a wave takes a unit of 512 elements of one tensor, 4 of
// each half of it to a lane, all of its loads first and past the caches.  The tensors'
// addresses are in the launch's arguments; a wave finds its tensor by comparing its
// number with all of their first units at once.
//
// States in 8 bits.  A block of 64 elements (16 lanes) shares an exponent byte b, that of
// its largest magnitude.  A code is the top of the element's fp32 pattern after scaling
// by 2^(15 - b) (first moment: a sign, 4 bits of exponent, 3 of mantissa) or 2^(31 - b)
// (second moment, 5 and 3): what the scaling takes into fp32's subnormal range, where it
// rounds to 2^-20 of the smallest code, is the code's too.  So coding is a scaling, an
// addition of the rounding and a shift, decoding a shift and a scaling, both exact: an
// unchanged value is held unchanged even when its block's exponent moves.
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

constexpr uint32_t kInf = 0x7F800000u;

// Random bits of elements i .. i + 3 (i a multiple of 4): two rounds of shifts and
// products.  The two multipliers are from C. Wellons' "Prospecting for Hash Functions"
// (2018), a search for little bias; the multiplier that gives the second moment's bits from
// the first's is a prime next to 2^32 over the golden ratio (D. Knuth, TAOCP 3, 6.4).  The
// four differ in two bits until the first product, so one product gives the others' by
// additions.
__device__ __forceinline__ void random_bits(const TensorsArgs& a, int64_t i, uint32_t x[4]) {
  constexpr uint32_t kFirst = 0x7FEB352Du;
  uint32_t y = (uint32_t)i ^ a.key_lo;
  y ^= y >> 16;
  const uint32_t one = y & 1 ? 0u - kFirst : kFirst, two = y & 2 ? 0u - 2 * kFirst : 2 * kFirst;
  x[0] = y * kFirst;
  x[1] = x[0] + one, x[2] = x[0] + two, x[3] = x[1] + two;
  const uint32_t high = (uint32_t)(i >> 32) + a.key_hi;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    uint32_t z = x[e] ^ high;
    z = (z ^ (z >> 15)) * 0x846CA68Bu;
    x[e] = z ^ (z >> 16);
  }
}

template <int kCtrl>
__device__ __forceinline__ uint32_t max_dpp(uint32_t x) {
  const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, kCtrl, 0xF, 0xF, true);
  return x > o ? x : o;
}

// The largest of a block's 16 lanes' values, in all of them.
__device__ __forceinline__ uint32_t block_max(uint32_t most) {
  most = max_dpp<0xB1>(most);      // lane ^ 1
  most = max_dpp<0x4E>(most);      // lane ^ 2
  most = max_dpp<0x141>(most);     // the other half of 8
  return max_dpp<0x140>(most);     // the other half of 16
}

// The exponent byte of a block whose largest finite magnitude has this pattern.  (A
// mantissa over 1.75 would be rounded to a code that stands for no number: (0x7FFFFF -
// 0x600000) more carries into the exponent for these.)
__device__ __forceinline__ uint32_t block_exp(uint32_t most) {
  const uint32_t b = (most + 0x1FFFFFu) >> 23;
  return b < kLowExp ? kLowExp : b;
}

// What is added to a scaled value's pattern before its low 20 bits are dropped.
template <bool kDrawn>
__device__ __forceinline__ uint32_t rounded(uint32_t y, uint32_t bits) {
  return y + (kDrawn ? bits : 0x7FFFFu + ((y >> 20) & 1));
}

// The codes of 4 elements of each half, and their blocks' exponents; bits: 20 random ones
// for each element.
template <int kTop, bool kDrawn>
__device__ __forceinline__ void store_codes(uint8_t* codes, uint8_t* exps, int64_t unit, int lane,
                                            const float x[8], const uint32_t bits[8]) {
  uint32_t most[2], b[2], c[8];
  float z[8];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    most[h] = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      z[4 * h + e] = x[4 * h + e];
      const uint32_t w = __float_as_uint(x[4 * h + e]) & (kTop == kTopM ? 0x7FFFFFFFu : 0xFFFFFFFFu);
      if (w > most[h]) most[h] = w;
    }
  }
  // (a second moment with a sign, -0 say, is more than any, too: it loses the sign)
  const bool odd = most[0] >= kInf || most[1] >= kInf;
  if (__builtin_expect(__any(odd), 0)) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      most[h] = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t w = __float_as_uint(x[4 * h + e]) & 0x7FFFFFFFu;
        if (w < kInf && w > most[h]) most[h] = w;
        if (kTop == kTopV) z[4 * h + e] = __builtin_fabsf(x[4 * h + e]);
      }
    }
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    b[h] = block_exp(block_max(most[h]));
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int i = 4 * h + e;
      const uint32_t y =
          __float_as_uint(__builtin_amdgcn_ldexpf(z[i], kTop - (int)b[h]));
      c[i] = rounded<kDrawn>(y, bits[i]) >> 20;
      if constexpr (kTop == kTopM) {
        c[i] = (c[i] & 0x7F) | ((y >> 24) & 0x80);   // the sign is y's
      } else {
        const uint32_t w = __float_as_uint(z[i]), least = w < 1 ? w : 1;   // not 0 for v > 0
        c[i] = c[i] > least ? c[i] : least;
      }
    }
  }
  if (__builtin_expect(__any(odd), 0)) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t w = __float_as_uint(x[i]);
      if ((w & 0x7FFFFFFFu) >= kInf) c[i] = (8 * kTop + 7) | (kTop == kTopM ? (w >> 24) & 0x80 : 0);
    }
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint32_t* k = c + 4 * h;
    const uint32_t w = (k[0] | k[1] << 8) | (k[2] << 16 | k[3] << 24);
    __builtin_nontemporal_store(
        w, reinterpret_cast<uint32_t*>(codes + unit * kUnit + h * kHalf + lane * 4));
    if ((lane & 15) == 0) exps[unit * (kUnit / kStateBlock) + h * 4 + lane / 16] = (uint8_t)b[h];
  }
}

// Four codes of each half, whose exponents the lanes of a block share.
struct Codes {
  uint32_t w[2], b[2];
};

__device__ __forceinline__ Codes load_codes(const uint8_t* codes, const uint8_t* exps, int64_t unit,
                                            int lane) {
  Codes c;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    c.w[h] = __builtin_nontemporal_load(
        reinterpret_cast<const uint32_t*>(codes + unit * kUnit + h * kHalf + lane * 4));
    const uint32_t b = exps[unit * (kUnit / kStateBlock) + h * 4 + lane / 16];
    c.b[h] = b < kLowExp ? kLowExp : b;   // (0 before the first step)
  }
  return c;
}

// A first moment's code is an fp8 value of 4 and 3 bits, which the chip converts; a second
// moment's the top of an fp32 pattern.
template <int kTop>
__device__ __forceinline__ void values(const Codes& c, float x[8]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    if constexpr (kTop == kTopM) {
      const float scale = __uint_as_float((c.b[h] - 8) << 23);   // 2^(b - 135)
      const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)c.w[h], false);
      const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)c.w[h], true);
      x[4 * h] = lo[0] * scale, x[4 * h + 1] = lo[1] * scale;
      x[4 * h + 2] = hi[0] * scale, x[4 * h + 3] = hi[1] * scale;
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        x[4 * h + e] = __builtin_amdgcn_ldexpf(
            __uint_as_float(((c.w[h] >> (8 * e)) & 255) << 20), (int)c.b[h] - kTopV);
    }
  }
  if constexpr (kTop == kTopV) {
    // a byte of ones somewhere (or so it may seem)
    auto ones = [](uint32_t w) { return (~w - 0x01010101u) & w & 0x80808080u; };
    if (__builtin_expect(__any((ones(c.w[0]) | ones(c.w[1])) != 0), 0)) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (((c.w[i / 4] >> (8 * (i % 4))) & 255) == 255) x[i] = __builtin_nanf("");
    }
  }
}

// Elements lane * 4 .. + 3 of each half of a unit of which n (from the unit's start) are
// the tensor's, zeros behind them.  kFull: all of them are.
template <bool kFull>
__device__ __forceinline__ void load_f32(const float* p, int n, int lane, float x[8]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int at = h * kHalf + lane * 4;
    if (kFull || at + 4 <= n) {
      const f32x4 w = __builtin_nontemporal_load(reinterpret_cast<const f32x4_at4*>(p + at));
      x[4 * h] = w.x, x[4 * h + 1] = w.y, x[4 * h + 2] = w.z, x[4 * h + 3] = w.w;
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) x[4 * h + e] = at + e < n ? p[at + e] : 0.f;
    }
  }
}

template <bool kFull>
__device__ __forceinline__ void load_bf16(const uint16_t* p, int n, int lane, float x[8]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int at = h * kHalf + lane * 4;
    if (kFull || at + 4 <= n) {
      const u32x2 w = __builtin_nontemporal_load(reinterpret_cast<const u32x2_at2*>(p + at));
      x[4 * h] = bf16_lo(w.x), x[4 * h + 1] = bf16_hi(w.x);
      x[4 * h + 2] = bf16_lo(w.y), x[4 * h + 3] = bf16_hi(w.y);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        x[4 * h + e] = at + e < n ? __uint_as_float((uint32_t)p[at + e] << 16) : 0.f;
    }
  }
}

template <bool kFull, bool kPast = true>
__device__ __forceinline__ void store_f32(float* p, int n, int lane, const float x[8]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int at = h * kHalf + lane * 4;
    if (kFull || at + 4 <= n) {
      const f32x4 w{x[4 * h], x[4 * h + 1], x[4 * h + 2], x[4 * h + 3]};
      if constexpr (kPast) __builtin_nontemporal_store(w, reinterpret_cast<f32x4_at4*>(p + at));
      else *reinterpret_cast<f32x4_at4*>(p + at) = w;
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (at + e < n) p[at + e] = x[4 * h + e];
    }
  }
}

template <bool kFull>
__device__ __forceinline__ void store_bf16(uint16_t* p, int n, int lane, const float x[8]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int at = h * kHalf + lane * 4;
    if (kFull || at + 4 <= n) {
      const u32x2 w{pack_bf16x2(x[4 * h], x[4 * h + 1]), pack_bf16x2(x[4 * h + 2], x[4 * h + 3])};
      __builtin_nontemporal_store(w, reinterpret_cast<u32x2_at2*>(p + at));
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (at + e < n) p[at + e] = (uint16_t)to_bf16(x[4 * h + e]);
    }
  }
}

// One unit: elements `from` on of tensor k, n of them the tensor's.
template <bool kGradF32, int kBits, bool kDrawn, bool kFull>
__device__ __forceinline__ void step_unit(const TensorsArgs& a, int k, int64_t from, int n,
                                          int64_t unit, int lane) {
  float* master = a.master[k] + from;
  float p[8], g[8], m[8], v[8];
  float* mf = static_cast<float*>(a.state.m) + unit * kUnit;
  float* vf = static_cast<float*>(a.state.v) + unit * kUnit;
  uint8_t* mc = static_cast<uint8_t*>(a.state.m);
  uint8_t* vc = static_cast<uint8_t*>(a.state.v);
  Codes cm, cv;
  load_f32<kFull>(master, n, lane, p);
  if constexpr (kGradF32)
    load_f32<kFull>(static_cast<const float*>(a.grad[k]) + from, n, lane, g);
  else
    load_bf16<kFull>(static_cast<const uint16_t*>(a.grad[k]) + from, n, lane, g);
  if constexpr (kBits == 32) {
    load_f32<true>(mf, kUnit, lane, m);
    load_f32<true>(vf, kUnit, lane, v);
  } else {
    cm = load_codes(mc, a.state.m_exp, unit, lane);
    cv = load_codes(vc, a.state.v_exp, unit, lane);
  }
  __builtin_amdgcn_sched_barrier(0);   // all of them before the arithmetic
  uint32_t rm[8], rv[8];
  if constexpr (kDrawn) {   // while the loads are under way
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      random_bits(a, unit * kUnit + h * kHalf + lane * 4, rm + 4 * h);
#pragma unroll
      for (int e = 4 * h; e < 4 * h + 4; ++e) {
        rv[e] = (rm[e] * 0x9E3779B1u) >> 12;
        rm[e] = rm[e] >> 12;
      }
    }
  }
  if constexpr (kBits == 8) {
    values<kTopM>(cm, m);
    values<kTopV>(cv, v);
  }
  const float decay = (a.decay[k / 32] >> (k % 32)) & 1 ? a.s.decay : 1.0f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    p[e] = p[e] * decay;
    g[e] = g[e] * a.grad_scale;
  }
  adam8(a.s, g, p, m, v);
  store_f32<kFull>(master, n, lane, p);
  if (a.working[k]) store_bf16<kFull>(a.working[k] + from, n, lane, p);
  if constexpr (kBits == 32) {
    store_f32<true>(mf, kUnit, lane, m);
    store_f32<true>(vf, kUnit, lane, v);
  } else {
    store_codes<kTopM, kDrawn>(mc, a.state.m_exp, unit, lane, m, rm);
    store_codes<kTopV, kDrawn>(vc, a.state.v_exp, unit, lane, v, rv);
  }
}

// Workgroups of one wave, twelve of which a CU holds at once (by the LDS that they ask for
// and do not use), or of four with seven.  More waves than it takes to keep the memory
// busy only spread what they read and write: 92 M elements with states in 32 bits take 422
// us with 12 waves, 438 with 20, 445 with all 32; the states in 8 bits take more
// arithmetic (620 vector instructions a unit beside 300), and with it 28 waves: 218 M
// elements 578 us, with 16 797.
template <int kBits>
constexpr int kThreads = kBits == 8 ? 256 : 64;
template <int kBits>
constexpr unsigned kLds = kBits == 8 ? 23200 : 13632;

template <bool kGradF32, int kBits, bool kDrawn>
__global__ void __launch_bounds__(kThreads<kBits>) k_tensors(const TensorsArgs a, int64_t units) {
  const int lane = threadIdx.x & 63;
  const int64_t u = (int64_t)blockIdx.x * (kThreads<kBits> / 64) +
                    __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  if (u >= units) return;
  // tensors that begin behind the first one, up to this unit
  static_assert(kMaxTensors > 64 && kMaxTensors <= 128);
  const int more = lane < kMaxTensors - 64 ? a.first[lane + 65] : INT32_MAX;
  const int k = __popcll(__ballot(a.first[lane + 1] <= u)) + __popcll(__ballot(more <= u));
  const int64_t from = (u - a.first[k]) * kUnit;
  const int64_t n = a.numel[k] - from;
  if (__builtin_expect(n >= kUnit, 1))
    step_unit<kGradF32, kBits, kDrawn, true>(a, k, from, kUnit, a.unit0 + u, lane);
  else
    step_unit<kGradF32, kBits, kDrawn, false>(a, k, from, (int)n, a.unit0 + u, lane);
}

// Two waves to a workgroup, eight of which a CU holds at once (218 M elements: 355 us;
// with all that fit 398).
constexpr int kConvertThreads = 128;
constexpr unsigned kConvertLds = 20480;

template <bool kTo8>
__global__ void __launch_bounds__(kConvertThreads)
    k_state_convert(const StateDev narrow, const StateDev wide, int64_t units) {
  const int lane = threadIdx.x & 63;
  const int64_t u = (int64_t)blockIdx.x * (kConvertThreads / 64) +
                    __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  if (u >= units) return;
  float* mf = static_cast<float*>(wide.m) + u * kUnit;
  float* vf = static_cast<float*>(wide.v) + u * kUnit;
  uint8_t* mc = static_cast<uint8_t*>(narrow.m);
  uint8_t* vc = static_cast<uint8_t*>(narrow.v);
  float m[8], v[8];
  if constexpr (kTo8) {
    load_f32<true>(mf, kUnit, lane, m);
    load_f32<true>(vf, kUnit, lane, v);
    const uint32_t none[8] = {};
    store_codes<kTopM, false>(mc, narrow.m_exp, u, lane, m, none);
    store_codes<kTopV, false>(vc, narrow.v_exp, u, lane, v, none);
  } else {
    const Codes cm = load_codes(mc, narrow.m_exp, u, lane);
    const Codes cv = load_codes(vc, narrow.v_exp, u, lane);
    values<kTopM>(cm, m);
    values<kTopV>(cv, v);
    store_f32<true, false>(mf, kUnit, lane, m);
    store_f32<true, false>(vf, kUnit, lane, v);
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
  const int threads = a.state.bits == 8 ? kThreads<8> : kThreads<32>, waves = threads / 64;
  return launch(kernel, dim3((unsigned)((units + waves - 1) / waves)), threads,
                a.state.bits == 8 ? kLds<8> : kLds<32>, st, a, units);
}

hipError_t launch_state_convert(const StateDev& from, const StateDev& to, int64_t units,
                                hipStream_t st) {
  const dim3 grid((unsigned)((units + kConvertThreads / 64 - 1) / (kConvertThreads / 64)));
  return to.bits == 8 ? launch(k_state_convert<true>, grid, kConvertThreads, kConvertLds, st, to,
                               from, units)
                      : launch(k_state_convert<false>, grid, kConvertThreads, kConvertLds, st, from, to,
                               units);
}

}  // namespace flr
