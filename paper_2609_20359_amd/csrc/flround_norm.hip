// flround_norm.hip -- gfx950 kernels of the layer norm and its gradient.
//
// Both read a row once, hold it in registers as it came (16-byte chunks, spread over
// one to sixteen waves), and write a row: they are bound by memory.  Sums are in
// fp32 in a fixed order.
#include "flr_launch.h"
#include "flr_layers.h"
#include "flr_rows.h"

namespace flr {
namespace {

// The sums of N values over the waves of a row, in all of its threads.  `red` is not
// written again before all have read it: calls take turns between two of them.
template <int W, int N>
__device__ __forceinline__ void row_sums(float (&x)[N], float (*red)[N], int wave) {
#pragma unroll
  for (int k = 0; k < N; ++k) x[k] = wave_sum_f(x[k]);
  if constexpr (W > 1) {
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
      for (int k = 0; k < N; ++k) red[wave][k] = x[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < N; ++k) {
      x[k] = red[0][k];
#pragma unroll
      for (int w = 1; w < W; ++w) x[k] = x[k] + red[w][k];
    }
  }
}

// The largest of the threads' values (none of them NaN) over the waves of a row, in all.
template <int W>
__device__ __forceinline__ float row_max(float x, float (*red)[1], int wave) {
  for (int d = 32; d > 0; d /= 2) x = __builtin_fmaxf(x, __shfl_xor(x, d));
  if constexpr (W > 1) {
    if ((threadIdx.x & 63) == 0) red[wave][0] = x;
    __syncthreads();
    x = red[0][0];
    for (int w = 1; w < W; ++w) x = __builtin_fmaxf(x, red[w][0]);
  }
  return x;
}

// A row whose sum or whose squares are no fp32 numbers (values past 2^60), or whose squares
// lose bits (values below 2^-60 beside an eps as small), from memory again: as the rows
// below, but divided by 2^by, a power close to the row's largest magnitude or to sqrt(eps),
// which is exact where it counts (2^0 for a row of zeros, or with an infinity or NaN).  All
// waves of the row come here.
template <typename T, int W, bool kRms>
__device__ __forceinline__ void norm_scaled(const NormArgs& a, int64_t r, int64_t at,
                                            float (*red)[W][1], int wave) {
  constexpr int E = Rows<T>::kE;
  constexpr int64_t kNext = W * 64 * E;
  const T* row = static_cast<const T*>(a.x) + r * a.ldx;
  const T* wt = static_cast<const T*>(a.weight);
  const T* bs = static_cast<const T*>(a.bias);
  int by = 0;
  // f(element's place, its value / 2^by) for the lane's elements
  auto every = [&](auto f) {
#pragma unroll 1
    for (int64_t k = at; k < a.D; k += kNext) {
      float x[E];
      Rows<T>::floats(load_chunk(row, k, a.D), x);
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (k + e < a.D) f(k + e, __builtin_amdgcn_ldexpf(x[e], -by));
    }
  };
  float most = 0.f, s[1] = {0.f}, q[1] = {0.f};
  every([&](int64_t, float x) {
    most = x == x ? __builtin_fmaxf(most, __builtin_fabsf(x)) : __builtin_inff();
  });
  most = row_max<W>(most, red[0], wave);
  if (most > 0.f && most < __builtin_inff()) {
    by = __builtin_amdgcn_frexp_expf(most);
    const int least = a.eps > 0.f ? __builtin_amdgcn_frexp_expf(a.eps) / 2 : by;
    by = by > least ? by : least;
  }
  if constexpr (!kRms) {
    every([&](int64_t, float x) { s[0] = s[0] + x; });
    row_sums<W>(s, red[1], wave);
  }
  const float n = (float)a.D, mean = kRms ? 0.f : s[0] / n;
  every([&](int64_t, float x) { q[0] = __builtin_fmaf(x - mean, x - mean, q[0]); });
  row_sums<W>(q, red[kRms ? 1 : 0], wave);
  const float rstd = 1.0f / __builtin_sqrtf(q[0] / n + __builtin_amdgcn_ldexpf(a.eps, -2 * by));
  if ((threadIdx.x & 63) == 0 && (W == 1 || wave == 0)) {
    if (a.mean) a.mean[r] = __builtin_amdgcn_ldexpf(mean, by);
    a.rstd[r] = __builtin_amdgcn_ldexpf(rstd, -by);
  }
  T* out = static_cast<T*>(a.y) + r * a.D;
  every([&](int64_t k, float x) {
    float y = (x - mean) * rstd;
    if (wt) y = y * Rows<T>::value(wt[k]);
    if (bs) y = y + Rows<T>::value(bs[k]);
    out[k] = Rows<T>::one(y);
  });
}

// y = (x - mean) rstd w + b.  W waves to a row, K chunks to a lane; outputs larger than the
// L2s go past them, and so do inputs.  (16384 x 4096 bf16, four waves of two chunks: 44 us,
// 6.1 TB/s; 46 through the caches, 45 only with outputs past them.)  Rows at the ends of
// fp32 are left to norm_scaled, which reads them again: kept in registers meanwhile, they
// cost all rows of 16384 columns a quarter more time.
template <typename T, int W, int K, bool kRms, bool kPast>
__global__ void __launch_bounds__(W < 4 ? 256 : 64 * W) k_norm(const NormArgs a) {
  constexpr int E = Rows<T>::kE, kAt = W < 4 ? 4 / W : 1;
  __shared__ float red[2][W][1];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int64_t at = ((W == 1 ? 0 : wave * 64) + lane) * E;
  constexpr int64_t kNext = W * 64 * E;
  const int64_t r = (int64_t)blockIdx.x * kAt + (W == 1 ? wave : 0);
  if (r >= a.T) return;   // (whole waves of W = 1, no barrier behind)
  const T* row = static_cast<const T*>(a.x) + r * a.ldx;
  u32x4 x[K];
#pragma unroll
  for (int k = 0; k < K; ++k) x[k] = load_chunk<kPast>(row, at + k * kNext, a.D);
  const T* wt = static_cast<const T*>(a.weight);
  const T* bs = static_cast<const T*>(a.bias);
  u32x4 w[K] = {}, b[K] = {};
  if (wt) {
#pragma unroll
    for (int k = 0; k < K; ++k) w[k] = load_chunk(wt, at + k * kNext, a.D);
  }
  if (bs) {
#pragma unroll
    for (int k = 0; k < K; ++k) b[k] = load_chunk(bs, at + k * kNext, a.D);
  }
  const float n = (float)a.D;
  float mean = 0.f;
  if constexpr (!kRms) {
    float s[1] = {0.f};
#pragma unroll
    for (int k = 0; k < K; ++k) {
      float f[E];
      Rows<T>::floats(x[k], f);
#pragma unroll
      for (int e = 0; e < E; ++e) s[0] = s[0] + f[e];
    }
    row_sums<W>(s, red[0], wave);
    mean = s[0] / n;
  }
  float q[1] = {0.f};
#pragma unroll
  for (int k = 0; k < K; ++k) {
    float f[E];
    Rows<T>::floats(x[k], f);
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const float d = kRms || at + k * kNext + e < a.D ? f[e] - mean : 0.f;
      q[0] = __builtin_fmaf(d, d, q[0]);
    }
  }
  row_sums<W>(q, red[1], wave);
  const float var = q[0] / n + a.eps;
  const int ends = !(var >= 0x1p-120f && var <= 0x1.fffffep127f);   // (alike in all threads)
  if (__builtin_expect(__builtin_amdgcn_readfirstlane(ends), 0)) {
    norm_scaled<T, W, kRms>(a, r, at, red, wave);
    return;
  }
  const float rstd = 1.0f / __builtin_sqrtf(var);
  if (lane == 0 && (W == 1 || wave == 0)) {
    if (a.mean) a.mean[r] = mean;
    a.rstd[r] = rstd;
  }
  T* out = static_cast<T*>(a.y) + r * a.D;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    float f[E], g[E], h[E];
    Rows<T>::floats(x[k], f);
    Rows<T>::floats(w[k], g);
    Rows<T>::floats(b[k], h);
#pragma unroll
    for (int e = 0; e < E; ++e) {
      float y = (f[e] - mean) * rstd;
      if (wt) y = y * g[e];
      if (bs) y = y + h[e];
      f[e] = y;
    }
    store_chunk<kPast>(out, at + k * kNext, a.D, f);
  }
}

// As load_chunk, but with elements of the row behind its end, too (zeros for a row of no
// elements): the gradient's lanes there have c = 0, and where mean * rstd is no fp32 number
// (a row of one value, 2^100, and eps 2^-60) zeros in x's place would make c xh NaN.
template <bool kPast = false, typename T>
__device__ __forceinline__ u32x4 load_some(const T* row, int64_t at, int64_t n) {
  if (at >= n) at = 0;
  if (at + Rows<T>::kE <= n) return kPast ? Rows<T>::load_past(row + at) : Rows<T>::load(row + at);
  return n > 0 ? Rows<T>::template load_part<true>(row + at, (int)(n - at)) : u32x4{0, 0, 0, 0};
}

// dx = rstd (c - mean(c) - xh mean(c xh)), c = dy w, xh = (x - mean) rstd (the second
// term not for a root mean square), and the workgroup's sums of dy xh and of dy, which it
// holds in registers over all of its rows, R at a time.  kNext: the next rows are asked
// for while these are summed.  (16384 x 4096 bf16, two rows of eight waves, inputs past the
// caches: 68 us, 6.0 TB/s, and 5 for the parts, 70 in all; through the caches 75, and so four
// waves of two chunks 77, without the next rows 79.)
template <typename T, int W, int K, int R, bool kRms, bool kNext, bool kPast>
__global__ void __launch_bounds__(64 * W * R) k_norm_grad(const NormArgs a) {
  constexpr int E = Rows<T>::kE;
  __shared__ float red[2][R][W][2];
  const int lane = threadIdx.x & 63;
  const int all_waves = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int wave = all_waves % W, group = all_waves / W;
  const int64_t at = (wave * 64 + lane) * E;
  constexpr int64_t kStep = W * 64 * E;
  const T* wt = static_cast<const T*>(a.weight);
  float dw[K][E] = {}, db[K][E] = {};
  u32x4 w[K] = {};
  if (wt) {
#pragma unroll
    for (int k = 0; k < K; ++k) w[k] = load_chunk(wt, at + k * kStep, a.D);
  }
  const float per = 1.0f / (float)a.D;
  const int64_t step = (int64_t)gridDim.x * R;
  const T* xs = static_cast<const T*>(a.x);
  const T* ds = static_cast<const T*>(a.dy);
  u32x4 xn[K], dn[K];
  float mean_n, rstd_n;
  // (rows behind the last are zeros, with statistics of zero: they add nothing)
  auto ask = [&](int64_t row) {
    const bool some = row < a.T;
#pragma unroll
    for (int k = 0; k < K; ++k)
      xn[k] = load_some<kPast>(xs + row * a.ldx, at + k * kStep, some ? a.D : 0);
#pragma unroll
    for (int k = 0; k < K; ++k)
      dn[k] = load_chunk<kPast>(ds + row * a.ldy, at + k * kStep, some ? a.D : 0);
    mean_n = !kRms && some ? a.mean_in[row] : 0.f;
    rstd_n = some ? a.rstd_in[row] : 0.f;
  };
  int64_t r = (int64_t)blockIdx.x * R + group;
  if (kNext) ask(r);
  int turn = 0;
  for (int64_t r0 = (int64_t)blockIdx.x * R; r0 < a.T; r0 += step, r += step, turn ^= 1) {
    if (!kNext) ask(r);
    u32x4 x[K], d[K];
#pragma unroll
    for (int k = 0; k < K; ++k) x[k] = xn[k], d[k] = dn[k];
    const float mean = mean_n, rstd = rstd_n;
    if (kNext && r0 + step < a.T) ask(r + step);
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int k = 0; k < K; ++k) {
      float f[E], g[E], h[E];
      Rows<T>::floats(x[k], f);
      Rows<T>::floats(d[k], g);
      Rows<T>::floats(w[k], h);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float xh = (f[e] - mean) * rstd;
        const float c = wt ? g[e] * h[e] : g[e];
        s[0] = __builtin_fmaf(c, xh, s[0]);
        if constexpr (!kRms) s[1] = s[1] + c;
        dw[k][e] = __builtin_fmaf(g[e], xh, dw[k][e]);
        db[k][e] = db[k][e] + g[e];
      }
    }
    row_sums<W>(s, red[turn][group], wave);
    if (r >= a.T) continue;
    const float m0 = s[0] * per, m1 = s[1] * per;
    T* out = static_cast<T*>(a.y) + r * a.D;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      float f[E], g[E], h[E];
      Rows<T>::floats(x[k], f);
      Rows<T>::floats(d[k], g);
      Rows<T>::floats(w[k], h);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float xh = (f[e] - mean) * rstd;
        float c = wt ? g[e] * h[e] : g[e];
        if constexpr (!kRms) c = c - m1;
        f[e] = rstd * __builtin_fmaf(-xh, m0, c);
      }
      store_chunk<kPast>(out, at + k * kStep, a.D, f);
    }
  }
  // the sums of the waves that hold the same columns, halving the groups, then the
  // workgroup's row of parts
  constexpr int kHalf = R > 1 ? R / 2 : 1;
  __shared__ float half[kHalf][R > 1 ? W * 64 * K * E : 1];
  auto leave = [&](float (&sum)[K][E], float* part) {
    const int mine = wave * 64 + lane;
#pragma unroll
    for (int n = R / 2; n > 0; n /= 2) {
      __syncthreads();
      if (group >= n && group < 2 * n) {
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
          for (int e = 0; e < E; ++e) half[group - n][(k * E + e) * W * 64 + mine] = sum[k][e];
      }
      __syncthreads();
      if (group < n) {
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
          for (int e = 0; e < E; ++e)
            sum[k][e] = sum[k][e] + half[group][(k * E + e) * W * 64 + mine];
      }
    }
    if (group > 0) return;
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (at + k * kStep + e < a.D) part[at + k * kStep + e] = sum[k][e];
  };
  float* part = a.parts + blockIdx.x * a.D;
  if (a.dweight) leave(dw, part);
  if (a.dbias) leave(db, part + a.n_parts * a.D);
}

// Few rows take one launch: workgroups for the rows (dx), and for 64 columns each (dw and
// db), which read x and dy again, from the caches, their waves every sixteenth row.
// (300 x 4096 bf16 with a bias: 10.1 us, 13.0 by parts and a second launch; 64 x 1024 9.6
// and 12.7; but 1000 x 1601 fp32 15.7 and 12.7.)
template <typename T, int W, bool kRms>
__global__ void __launch_bounds__(1024) k_norm_grad_few(const NormArgs a, int row_blocks) {
  constexpr int E = Rows<T>::kE, R = 16 / W;
  const int lane = threadIdx.x & 63;
  const int all_waves = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const T* xs = static_cast<const T*>(a.x);
  const T* ds = static_cast<const T*>(a.dy);
  if ((int)blockIdx.x >= row_blocks) {
    __shared__ float sums[2][16][64];
    const int64_t at = (int64_t)((int)blockIdx.x - row_blocks) * 64 + lane;
    float dw = 0.f, db = 0.f;
    if (at < a.D) {
#pragma unroll 8
      for (int r = all_waves; r < (int)a.T; r += 16) {
        const float mean = kRms ? 0.f : uniform(a.mean_in + r), rstd = uniform(a.rstd_in + r);
        const float d = Rows<T>::value(ds[r * a.ldy + at]);
        const float xh = (Rows<T>::value(xs[r * a.ldx + at]) - mean) * rstd;
        dw = __builtin_fmaf(d, xh, dw);
        db = db + d;
      }
    }
    sums[0][all_waves][lane] = dw, sums[1][all_waves][lane] = db;
    __syncthreads();
    if (all_waves > 1 || at >= a.D) return;
    T* out = static_cast<T*>(all_waves == 0 ? a.dweight : a.dbias);
    if (!out) return;
    float s = sums[all_waves][0][lane];
#pragma unroll
    for (int w = 1; w < 16; ++w) s = s + sums[all_waves][w][lane];
    out[at] = Rows<T>::one(s);
    return;
  }
  __shared__ float red[R][W][2];
  const int wave = all_waves % W, group = all_waves / W;
  const int64_t at = (wave * 64 + lane) * E, r = (int64_t)blockIdx.x * R + group;
  const bool some = r < a.T;
  const int64_t n = some ? a.D : 0;
  const u32x4 x = load_some(xs + r * a.ldx, at, n), d = load_chunk(ds + r * a.ldy, at, n);
  u32x4 w{0, 0, 0, 0};
  if (a.weight) w = load_chunk(static_cast<const T*>(a.weight), at, n);
  const float mean = !kRms && some ? a.mean_in[r] : 0.f, rstd = some ? a.rstd_in[r] : 0.f;
  float f[E], g[E], h[E], s[2] = {0.f, 0.f};
  Rows<T>::floats(x, f);
  Rows<T>::floats(d, g);
  Rows<T>::floats(w, h);
#pragma unroll
  for (int e = 0; e < E; ++e) {
    f[e] = (f[e] - mean) * rstd;
    if (a.weight) g[e] = g[e] * h[e];
    s[0] = __builtin_fmaf(g[e], f[e], s[0]);
    if constexpr (!kRms) s[1] = s[1] + g[e];
  }
  row_sums<W>(s, red[group], wave);
  if (!some) return;
  const float m0 = s[0] / (float)a.D, m1 = s[1] / (float)a.D;
#pragma unroll
  for (int e = 0; e < E; ++e) f[e] = rstd * __builtin_fmaf(-f[e], m0, kRms ? g[e] : g[e] - m1);
  store_chunk(static_cast<T*>(a.y) + r * a.D, at, a.D, f);
}

constexpr int kSumWaves = 16;

// The sum of the parts: 64 columns to a workgroup, its waves take every sixteenth part.
template <typename T>
__global__ void __launch_bounds__(64 * kSumWaves) k_norm_sum(const NormArgs a) {
  __shared__ float red[kSumWaves][64];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const bool bias = blockIdx.y == 1 || !a.dweight;
  const int64_t at = (int64_t)blockIdx.x * 64 + lane;
  const float* part = a.parts + (bias ? a.n_parts * a.D : 0) + at;
  float s = 0.f;
  if (at < a.D) {
#pragma unroll 8
    for (int64_t p = wave; p < a.n_parts; p += kSumWaves) s = s + part[p * a.D];
  }
  red[wave][lane] = s;
  __syncthreads();
  if (wave > 0 || at >= a.D) return;
#pragma unroll
  for (int w = 1; w < kSumWaves; ++w) s = s + red[w][lane];
  static_cast<T*>(bias ? a.dbias : a.dweight)[at] = Rows<T>::one(s);
}

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

bool past(const NormArgs& a) { return past_l2(a.T * a.D * (a.bf16 ? 2 : 4)); }

template <typename T, int W, int K, bool kRms>
hipError_t forward(const NormArgs& a, hipStream_t st) {
  const int rows = W < 4 ? 4 / W : 1;
  return launch(past(a) ? k_norm<T, W, K, kRms, true> : k_norm<T, W, K, kRms, false>,
                dim3((unsigned)ceil_div(a.T, rows)), W < 4 ? 256 : 64 * W, 0, st, a);
}

template <typename T, bool kRms>
hipError_t forward(const NormArgs& a, hipStream_t st) {
  const int64_t c = ceil_div(a.D, Rows<T>::kE);
  if (c <= 64) return forward<T, 1, 1, kRms>(a, st);
  if (c <= 128) return forward<T, 1, 2, kRms>(a, st);
  if (c <= 256) return forward<T, 4, 1, kRms>(a, st);
  if (c <= 512) return forward<T, 4, 2, kRms>(a, st);
  if (c <= 1024) return forward<T, 8, 2, kRms>(a, st);
  if (c <= 2048) return forward<T, 16, 2, kRms>(a, st);
  if constexpr (Rows<T>::kE == 8) return forward<T, 16, 4, kRms>(a, st);
  else return c <= 4096 ? forward<T, 16, 4, kRms>(a, st) : forward<T, 16, 8, kRms>(a, st);
}

template <typename T, int W, int K, int R, bool kNext, bool kRms>
hipError_t backward(const NormArgs& a, hipStream_t st) {
  return launch(past(a) ? k_norm_grad<T, W, K, R, kRms, kNext, true>
                        : k_norm_grad<T, W, K, R, kRms, kNext, false>,
                dim3((unsigned)a.n_parts), 64 * W * R, 0, st, a);
}

template <typename T, int W, bool kRms>
hipError_t backward_few(const NormArgs& a, hipStream_t st) {
  const int64_t rows = ceil_div(a.T, 16 / W);
  const int64_t columns = a.dweight || a.dbias ? ceil_div(a.D, 64) : 0;
  return launch(k_norm_grad_few<T, W, kRms>, dim3((unsigned)(rows + columns)), 1024, 0, st, a,
                (int)rows);
}

template <typename T, bool kRms>
hipError_t backward_few(const NormArgs& a, hipStream_t st) {
  const int64_t c = ceil_div(a.D, Rows<T>::kE);
  if (c <= 64) return backward_few<T, 1, kRms>(a, st);
  if (c <= 128) return backward_few<T, 2, kRms>(a, st);
  if (c <= 256) return backward_few<T, 4, kRms>(a, st);
  if (c <= 512) return backward_few<T, 8, kRms>(a, st);
  return backward_few<T, 16, kRms>(a, st);
}

template <typename T, bool kRms>
hipError_t backward(const NormArgs& a, hipStream_t st) {
  const int64_t c = ceil_div(a.D, Rows<T>::kE);
  if (c <= 64) return backward<T, 1, 1, 16, true, kRms>(a, st);
  if (c <= 128) return backward<T, 2, 1, 8, true, kRms>(a, st);
  if (c <= 256) return backward<T, 4, 1, 4, true, kRms>(a, st);
  if (c <= 512) return backward<T, 8, 1, 2, true, kRms>(a, st);
  if (c <= 1024) return backward<T, 16, 1, 1, true, kRms>(a, st);
  if (c <= 2048) return backward<T, 16, 2, 1, false, kRms>(a, st);
  if constexpr (Rows<T>::kE == 8) return backward<T, 16, 4, 1, false, kRms>(a, st);
  else
    return c <= 4096 ? backward<T, 16, 4, 1, false, kRms>(a, st)
                     : backward<T, 16, 8, 1, false, kRms>(a, st);
}

}  // namespace

int norm_rows(int64_t width, bool bf16) {
  const int64_t c = ceil_div(width, bf16 ? 8 : 4);
  return c <= 64 ? 16 : c <= 128 ? 8 : c <= 256 ? 4 : c <= 512 ? 2 : 1;
}

hipError_t launch_norm(const NormArgs& a, hipStream_t st) {
  if (a.bf16) return a.rms ? forward<uint16_t, true>(a, st) : forward<uint16_t, false>(a, st);
  return a.rms ? forward<float, true>(a, st) : forward<float, false>(a, st);
}

hipError_t launch_norm_grad(const NormArgs& a, hipStream_t st) {
  if (norm_few(a.T, a.D, a.bf16)) {
    if (a.bf16)
      return a.rms ? backward_few<uint16_t, true>(a, st) : backward_few<uint16_t, false>(a, st);
    return a.rms ? backward_few<float, true>(a, st) : backward_few<float, false>(a, st);
  }
  if (a.n_parts > 0) {
    const hipError_t e =
        a.bf16 ? (a.rms ? backward<uint16_t, true>(a, st) : backward<uint16_t, false>(a, st))
               : (a.rms ? backward<float, true>(a, st) : backward<float, false>(a, st));
    if (e != hipSuccess) return e;
  }
  if (!a.dweight && !a.dbias) return hipSuccess;
  const dim3 grid((unsigned)ceil_div(a.D, 64), a.dweight && a.dbias ? 2 : 1);
  return a.bf16 ? launch(k_norm_sum<uint16_t>, grid, 64 * kSumWaves, 0, st, a)
                : launch(k_norm_sum<float>, grid, 64 * kSumWaves, 0, st, a);
}

}  // namespace flr
