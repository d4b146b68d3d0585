// flr_rows.h -- device functions of kernels that read and write rows of bf16 or
// fp32 values in 16-byte chunks: 8 or 4 elements, on any element's boundary (the
// memory system takes 16 bytes from any address), the last one of a row in part.
#pragma once

#include "flr_device.h"

namespace flr {
namespace {

typedef u32x4 u32x4_at2 __attribute__((aligned(2)));
typedef u32x4 u32x4_at4 __attribute__((aligned(4)));

// A value that a whole wave reads at one address and no kernel writes meanwhile.
template <typename T>
__device__ __forceinline__ T uniform(const T* p) {
  return *(const __attribute__((address_space(4))) T*)(uintptr_t)p;
}

template <typename T>
struct Rows;

template <>
struct Rows<uint16_t> {
  static constexpr int kE = 8;   // elements of a chunk
  static __device__ __forceinline__ u32x4 load_past(const uint16_t* p) {
    return __builtin_nontemporal_load(reinterpret_cast<const u32x4_at2*>(p));
  }
  static __device__ __forceinline__ u32x4 load(const uint16_t* p) {
    return *reinterpret_cast<const u32x4_at2*>(p);
  }
  static __device__ __forceinline__ void store(uint16_t* p, u32x4 w) {
    *reinterpret_cast<u32x4_at2*>(p) = w;
  }
  // past the caches
  static __device__ __forceinline__ void store_past(uint16_t* p, u32x4 w) {
    __builtin_nontemporal_store(w, reinterpret_cast<u32x4_at2*>(p));
  }
  static __device__ __forceinline__ void floats(u32x4 w, float x[8]) {
    x[0] = bf16_lo(w.x), x[1] = bf16_hi(w.x), x[2] = bf16_lo(w.y), x[3] = bf16_hi(w.y);
    x[4] = bf16_lo(w.z), x[5] = bf16_hi(w.z), x[6] = bf16_lo(w.w), x[7] = bf16_hi(w.w);
  }
  static __device__ __forceinline__ u32x4 pack(const float x[8]) { return pack_bf16x8(x); }
  static __device__ __forceinline__ uint16_t one(float x) { return (uint16_t)to_bf16(x); }
  static __device__ __forceinline__ float value(uint16_t x) {
    return __uint_as_float((uint32_t)x << 16);
  }
  // the first n (1 to 7) elements at p; behind them zeros, or with kFill the first one
  template <bool kFill = false>
  static __device__ __forceinline__ u32x4 load_part(const uint16_t* p, int n) {
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < (kFill ? 8 : 7); ++e)
      if (kFill || e < n) w[e / 2] |= (uint32_t)p[e < n ? e : 0] << (16 * (e & 1));
    return u32x4{w[0], w[1], w[2], w[3]};
  }
};

template <>
struct Rows<float> {
  static constexpr int kE = 4;
  static __device__ __forceinline__ u32x4 load_past(const float* p) {
    return __builtin_nontemporal_load(reinterpret_cast<const u32x4_at4*>(p));
  }
  static __device__ __forceinline__ u32x4 load(const float* p) {
    return *reinterpret_cast<const u32x4_at4*>(p);
  }
  static __device__ __forceinline__ void store(float* p, u32x4 w) {
    *reinterpret_cast<u32x4_at4*>(p) = w;
  }
  static __device__ __forceinline__ void store_past(float* p, u32x4 w) {
    __builtin_nontemporal_store(w, reinterpret_cast<u32x4_at4*>(p));
  }
  static __device__ __forceinline__ void floats(u32x4 w, float x[4]) {
    x[0] = __uint_as_float(w.x), x[1] = __uint_as_float(w.y);
    x[2] = __uint_as_float(w.z), x[3] = __uint_as_float(w.w);
  }
  static __device__ __forceinline__ u32x4 pack(const float x[4]) {
    return u32x4{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]),
                 __float_as_uint(x[3])};
  }
  static __device__ __forceinline__ float one(float x) { return x; }
  static __device__ __forceinline__ float value(float x) { return x; }
  template <bool kFill = false>
  static __device__ __forceinline__ u32x4 load_part(const float* p, int n) {
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < (kFill ? 4 : 3); ++e)
      if (kFill || e < n) w[e] = __float_as_uint(p[e < n ? e : 0]);
    return u32x4{w[0], w[1], w[2], w[3]};
  }
};

// Elements [at, at + kE) of a row of n elements; zeros from n on (none where at >= n).
// kPast: what is read once, and more of it than the caches hold.  (A template's argument,
// as the compiler makes one plain access of two that a condition chooses between.)
template <bool kPast = false, typename T>
__device__ __forceinline__ u32x4 load_chunk(const T* row, int64_t at, int64_t n) {
  if (at + Rows<T>::kE <= n) return kPast ? Rows<T>::load_past(row + at) : Rows<T>::load(row + at);
  if (at < n) return Rows<T>::load_part(row + at, (int)(n - at));
  return u32x4{0, 0, 0, 0};
}

template <bool kPast = false, typename T>
__device__ __forceinline__ void store_chunk(T* row, int64_t at, int64_t n, const float* x) {
  if (at + Rows<T>::kE <= n) {
    if constexpr (kPast) Rows<T>::store_past(row + at, Rows<T>::pack(x));
    else Rows<T>::store(row + at, Rows<T>::pack(x));
  } else {
#pragma unroll
    for (int e = 0; e < Rows<T>::kE - 1; ++e)
      if (at + e < n) row[at + e] = Rows<T>::one(x[e]);
  }
}

template <int kCtrl>
__device__ __forceinline__ float add_dpp(float x) {
  return x + __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(
                 0, (int)__float_as_uint(x), kCtrl, 0xF, 0xF, true));
}

// The sum over the wave's 64 lanes, in all of them.
__device__ __forceinline__ float wave_sum_f(float x) {
  x = add_dpp<0xB1>(x);    // lane ^ 1
  x = add_dpp<0x4E>(x);    // lane ^ 2
  x = add_dpp<0x141>(x);   // the other half of 8
  x = add_dpp<0x140>(x);   // the other half of 16
  const int b = (int)__float_as_uint(x);
  auto row = [&](int lane) {
    return __uint_as_float((uint32_t)__builtin_amdgcn_readlane(b, lane));
  };
  return (row(0) + row(16)) + (row(32) + row(48));
}

}  // namespace
}  // namespace flr
