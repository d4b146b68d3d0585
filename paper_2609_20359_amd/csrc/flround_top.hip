// flround_top.hip -- gfx950 kernels of the top logits: the k largest of each
// row with their ids, and the logarithm of the sum of exp(x / tau).
//
// One pass over the logits, bound by HBM.  A workgroup of 512 threads takes a
// segment of a row into registers:
//   * the maxima of its 512 threads give a lower bound on the k-th largest (k
//     threads' maxima are at least their k-th largest), found by bisecting the
//     leading 16 bits;
//   * the 16-byte chunks whose largest value is not below the bound, a few more
//     than k as a rule, are listed in LDS; their values are read again, from L2,
//     and those not below the bound go to a second list; where it would not
//     fit (a row of equal values), the exact k-th largest is found by bisecting
//     (value, id);
//   * a list entry's place is the number of entries above it.
// Rows longer than a segment are joined by a second kernel, in which an entry's
// place is the sum of its places in the segments' sorted lists.
//
// Measured: 64 of 2048 rows of 128256 in bf16, 525 MB, in 119 us (4.4 TB/s; with
// the values kept as floats, 239 registers and one workgroup per SIMD, 330); 100
// of 100 rows of 100003 in fp32 in 23 us; 8 of one row of 50257 in 12 us, most of
// it two launches.  The selection has no loads out; the other workgroups of a CU,
// four in all, cover it.
//
// The order is that of one 64-bit number: the value, then the lower id; so ties
// go to the lowest id and no result depends on the order of the lists.
#include "flr_head.h"

namespace flr {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr float kLn2 = 0.6931471805599453f;
constexpr int kThreads = kTopThreads;
constexpr int kWaves = kThreads / 64;
constexpr int kJoinThreads = 512;
constexpr int kList = 2048;   // entries of the list in LDS

// Larger floats have larger keys, NaN the largest, and -0 that of +0.
__device__ __forceinline__ uint32_t key_of(float x) {
  const int32_t b = (int32_t)__float_as_uint(x + 0.f);
  return x != x ? 0xFFFFFFFFu : (uint32_t)(b ^ ((b >> 31) & 0x7FFFFFFF)) ^ 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t k) {
  const int32_t b = (int32_t)(k ^ 0x80000000u);
  return k == 0xFFFFFFFFu ? NAN : __uint_as_float((uint32_t)(b ^ ((b >> 31) & 0x7FFFFFFF)));
}
__device__ __forceinline__ uint64_t entry(float x, int id) {
  return (uint64_t)key_of(x) << 32 | (0xFFFFFFFFu - (uint32_t)id);
}
__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float log2_(float x) { return __builtin_amdgcn_logf(x); }

// (m, s) stands for s exp(m / tau); nothing is (-inf, 0).  Differences are taken
// before they are scaled: a row masked by the type's lowest value would overflow the
// other way round.  Infinities have none: a maximum of +inf has an s > 0, here +inf,
// whose logarithm changes nothing.
__device__ __forceinline__ void join(float& m, float& s, float pm, float ps, float s2) {
  const float top = fmaxf(m, pm), ref = fabsf(top) == INFINITY ? 0.f : top;
  s = s * exp2_((m - ref) * s2) + ps * exp2_((pm - ref) * s2);
  m = top;
}
__device__ __forceinline__ float lse_of(float m, float s, const TopArgs& a) {
  return m / a.tau + log2_(s) * kLn2;
}

__device__ __forceinline__ void emit(const TopArgs& a, int64_t row, int place, uint64_t e) {
  a.values[row * a.k + place] = value_of((uint32_t)(e >> 32));
  a.ids[row * a.k + place] = (int32_t)(0xFFFFFFFFu - (uint32_t)e);
}

// NC: 16-byte chunks per thread.
template <bool BF16, int NC>
__global__ __launch_bounds__(kThreads) void k_top_segment(const TopArgs a) {
  constexpr int E = BF16 ? 8 : 4;        // elements of a chunk
  constexpr int ES = BF16 ? 2 : 4;
  __shared__ uint64_t list[kList];
  __shared__ uint16_t chunks[kThreads * NC];
  __shared__ uint32_t maxima[kThreads];
  __shared__ float wave_m[kWaves], wave_s[kWaves];
  __shared__ int counts[2][kWaves];
  __shared__ int n_list, n_chunks;
  __shared__ float bound;

  const int tid = threadIdx.x, l = tid & 63, w = tid >> 6;
  const int64_t row = blockIdx.x / a.segs;
  const int seg = (int)(blockIdx.x % a.segs);
  const int vocab = (int)a.vocab;
  // chunks are counted from the 16-byte boundary at or before the row
  const char* src = static_cast<const char*>(a.logits) + row * a.stride * ES;
  const int head = (int)(reinterpret_cast<uintptr_t>(src) & 15) / ES;
  const int first = seg * kThreads * NC * E - head;   // id of the segment's first
  auto element = [&](int id) -> float {
    return BF16 ? __uint_as_float((uint32_t)*reinterpret_cast<const uint16_t*>(src + (int64_t)id * 2) << 16)
                : *reinterpret_cast<const float*>(src + (int64_t)id * 4);
  };

  u32x4 d[NC];
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const int id = first + (c * kThreads + tid) * E;
    if (id >= 0 && id + E <= vocab) {
      d[c] = *reinterpret_cast<const u32x4*>(src + (int64_t)id * ES);
    } else {
      // what is not there reads as -inf, and is told apart by its id
      uint32_t x[E];
#pragma unroll
      for (int e = 0; e < E; ++e)
        x[e] = id + e >= 0 && id + e < vocab ? __float_as_uint(element(id + e)) : 0xFF800000u;
#pragma unroll
      for (int i = 0; i < 4; ++i) d[c][i] = BF16 ? x[2 * i] >> 16 | x[2 * i + 1] : x[i];
    }
  }
  auto value = [&](int c, int e) -> float {
    if (!BF16) return __uint_as_float(d[c][e]);
    const uint32_t u = d[c][e >> 1];
    return __uint_as_float(e & 1 ? u & 0xFFFF0000u : u << 16);
  };

  float top = -INFINITY, tops[NC];
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    tops[c] = -INFINITY;
#pragma unroll
    for (int e = 0; e < E; ++e) tops[c] = fmaxf(tops[c], value(c, e));
    top = fmaxf(top, tops[c]);
  }
  maxima[tid] = key_of(top) >> 16;
  if (tid == 0) n_list = n_chunks = 0;
  float m = top;
#pragma unroll
  for (int x = 32; x; x >>= 1) m = fmaxf(m, __shfl_xor(m, x));
  if (l == 0) wave_m[w] = m;
  __syncthreads();

  // wave 0: the bound; all waves: the sum
  if (w == 0) {
    uint32_t v[kWaves], t = 0;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) v[i] = maxima[i * 64 + l];
    for (int bit = 15; bit >= 0; --bit) {
      const uint32_t x = t | 1u << bit;
      int n = 0;
#pragma unroll
      for (int i = 0; i < kWaves; ++i) n += __popcll(__ballot(v[i] >= x));
      if (n >= a.k) t = x;
    }
    // the least value whose key starts with these bits; as a float it may be a
    // NaN's pattern below -inf, where nothing is below the bound
    if (l == 0) bound = t <= 0x007Fu ? -INFINITY : value_of(t << 16);
  }
  m = wave_m[0];
#pragma unroll
  for (int i = 1; i < kWaves; ++i) m = fmaxf(m, wave_m[i]);
  float s = 0.f;
  const float ref = fabsf(m) == INFINITY ? 0.f : m, ref2 = ref * a.s2;
  // The scaled maximum is rounded, by up to 1/2 where it is 2^24 and by 2^103 in a row
  // of the type's lowest values: from there on (or where it overflows) the difference
  // is taken first.
  const bool far = !(fabsf(ref2) < 0x1p24f);
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    // The values are taken from the registers anew: kept, they would be twice
    // as many, and fewer waves would cover the loads.
    asm volatile("" : "+v"(d[c]));
#pragma unroll
    for (int e = 0; e < E; ++e)
      s += exp2_(far ? (value(c, e) - ref) * a.s2 : __builtin_fmaf(value(c, e), a.s2, -ref2));
  }
  const bool odd = s != s;   // a NaN among them: no chunk is left out
#pragma unroll
  for (int x = 32; x; x >>= 1) s += __shfl_xor(s, x);
  if (l == 0) wave_s[w] = s;
  __syncthreads();

  const float b = bound;
#pragma unroll
  for (int c = 0; c < NC; ++c)
    if (odd || !(tops[c] < b)) chunks[atomicAdd(&n_chunks, 1)] = (uint16_t)(c * kThreads + tid);
  __syncthreads();
  auto each_above = [&](auto f) {
    const int n = n_chunks * E;
    for (int i = tid; i < n; i += kThreads) {
      const int id = first + chunks[i / E] * E + i % E;
      if (id < 0 || id >= vocab) continue;
      const float x = element(id);
      if (!(x < b)) f(entry(x, id));
    }
  };
  each_above([&](uint64_t x) {
    const int at = atomicAdd(&n_list, 1);
    if (at < kList) list[at] = x;
  });
  __syncthreads();
  int all = n_list;
  if (all > kList) {
    // The k-th largest entry itself: the largest number that k entries reach.
    // Ids are below 2^20, so an entry's bits 31 to 20 are ones.
    uint64_t least = 0;
    for (int bit = 63; bit >= 0; --bit) {
      if (bit == 31) {
        least |= 0xFFF00000u;
        bit = 19;
      }
      const uint64_t x = least | (uint64_t)1 << bit;
      int r = 0;
      each_above([&](uint64_t y) { r += y >= x; });
#pragma unroll
      for (int i = 32; i; i >>= 1) r += __shfl_xor(r, i);
      if (l == 0) counts[bit & 1][w] = r;
      __syncthreads();
      r = 0;
#pragma unroll
      for (int i = 0; i < kWaves; ++i) r += counts[bit & 1][i];
      if (r >= a.k) least = x;
    }
    if (tid == 0) n_list = 0;
    __syncthreads();
    each_above([&](uint64_t x) {
      if (x >= least) list[atomicAdd(&n_list, 1)] = x;
    });
    __syncthreads();
    all = a.k;
  }
  const bool last = a.segs == 1;
  uint64_t* out = last ? nullptr : a.lists + (row * a.segs + seg) * a.k;
  for (int i = tid; i < all; i += kThreads) {
    const uint64_t x = list[i];
    int place = 0;
    for (int j = 0; j < all; ++j) place += list[j] > x;
    if (place < a.k) {
      if (last) emit(a, row, place, x);
      else out[place] = x;
    }
  }
  if (!last)
    for (int i = all + tid; i < a.k; i += kThreads) out[i] = 0;   // fewer than k in the segment
  if (tid == 0) {
    s = 0.f;
    for (int i = 0; i < kWaves; ++i) s += wave_s[i];
    if (m == INFINITY && s > 0.f) s = 1.f;   // (a NaN stays)
    if (!last) a.parts[row * a.segs + seg] = make_float2(m, s);
    else if (a.lse) a.lse[row] = lse_of(m, s, a);
  }
}

// Joins a row's segments.  The least of the segments' ceil(k / segs)-th entries
// has k entries at or above it, so only those, a few more than k, are placed:
// an entry's place is how many of its own segment and of the others, by
// bisection, are above it.
__global__ __launch_bounds__(kJoinThreads) void k_top_join(const TopArgs a) {
  extern __shared__ uint64_t lists[];   // segs x k entries, then places and numbers of the kept
  __shared__ int n_kept;
  const int tid = threadIdx.x;
  const int64_t row = blockIdx.x;
  const int n = a.segs * a.k;
  int* place = reinterpret_cast<int*>(lists + n);
  uint16_t* kept = reinterpret_cast<uint16_t*>(place + n);
  for (int i = tid; i < n; i += kJoinThreads) {
    lists[i] = a.lists[row * n + i];
    place[i] = 0;
  }
  if (tid == 0) n_kept = 0;
  __syncthreads();
  if (a.lse && tid < 64) {
    float m = -INFINITY, s = 0.f;
    for (int g = tid; g < a.segs; g += 64) {
      const float2 p = a.parts[row * a.segs + g];
      join(m, s, p.x, p.y, a.s2);
    }
#pragma unroll
    for (int x = 32; x; x >>= 1) join(m, s, __shfl_xor(m, x), __shfl_xor(s, x), a.s2);
    if (tid == 0) a.lse[row] = lse_of(m, s, a);
  }
  const int share = (a.k + a.segs - 1) / a.segs;
  uint64_t least = ~(uint64_t)0;
  for (int g = 0; g < a.segs; ++g) {
    const uint64_t x = lists[g * a.k + share - 1];
    least = x < least ? x : least;
  }
  for (int i = tid; i < n; i += kJoinThreads)
    if (lists[i] != 0 && lists[i] >= least) kept[atomicAdd(&n_kept, 1)] = (uint16_t)i;
  __syncthreads();
  const int pairs = n_kept * a.segs;
  for (int i = tid; i < pairs; i += kJoinThreads) {
    const int e = kept[i / a.segs], g = i % a.segs;
    const uint64_t x = lists[e];
    const uint64_t* p = lists + g * a.k;
    int lo = 0, hi = a.k;   // how many of p are above x
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (p[mid] > x) lo = mid + 1;
      else hi = mid;
    }
    if (lo) atomicAdd(&place[e], lo);
  }
  __syncthreads();
  for (int i = tid; i < n_kept; i += kJoinThreads) {
    const int e = kept[i];
    if (place[e] < a.k) emit(a, row, place[e], lists[e]);
  }
}

template <bool BF16>
hipError_t launch_segment(const TopArgs& a, dim3 grid, hipStream_t st) {
  switch (a.chunks) {
    case 1: return launch(k_top_segment<BF16, 1>, grid, kThreads, 0, st, a);
    case 2: return launch(k_top_segment<BF16, 2>, grid, kThreads, 0, st, a);
    case 4: return launch(k_top_segment<BF16, 4>, grid, kThreads, 0, st, a);
    default: return launch(k_top_segment<BF16, 8>, grid, kThreads, 0, st, a);
  }
}

}  // namespace

hipError_t launch_top(const TopArgs& a, hipStream_t st) {
  const dim3 grid((unsigned)(a.rows * a.segs));
  const hipError_t e = a.bf16 ? launch_segment<true>(a, grid, st) : launch_segment<false>(a, grid, st);
  if (e != hipSuccess || a.segs == 1) return e;
  return launch(k_top_join, dim3((unsigned)a.rows), kJoinThreads, (size_t)a.segs * a.k * 14, st, a);
}

}  // namespace flr
