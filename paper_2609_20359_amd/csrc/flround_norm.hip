// flround_norm.hip -- gfx950 kernels of the layer norm and its gradient.
//
// Both read a row once, hold it in registers as it came (16-byte chunks, spread over
// one, four or sixteen waves), and write a row: they are bound by memory.  Sums are in
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

// y = (x - mean) rstd w + b.  W waves to a row, K chunks to a lane.
template <typename T, int W, int K, bool kRms>
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
  for (int k = 0; k < K; ++k) x[k] = load_chunk(row, at + k * kNext, a.D);
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
  const float rstd = 1.0f / __builtin_sqrtf(q[0] / n + a.eps);
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
    store_chunk(out, at + k * kNext, a.D, f);
  }
}

// dx = rstd (c - mean(c) - xh mean(c xh)), c = dy w, xh = (x - mean) rstd (the second
// term not for a root mean square), and the workgroup's sums of dy xh and of dy, which it
// holds in registers over all of its rows.
template <typename T, int W, int K, bool kRms>
__global__ void __launch_bounds__(W < 4 ? 256 : 64 * W) k_norm_grad(const NormArgs a) {
  constexpr int E = Rows<T>::kE, kAt = W < 4 ? 4 / W : 1;
  __shared__ float red[2][W][2];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int64_t at = ((W == 1 ? 0 : wave * 64) + lane) * E;
  constexpr int64_t kNext = W * 64 * E;
  const T* wt = static_cast<const T*>(a.weight);
  float dw[K][E] = {}, db[K][E] = {};
  u32x4 w[K] = {};
  if (wt) {
#pragma unroll
    for (int k = 0; k < K; ++k) w[k] = load_chunk(wt, at + k * kNext, a.D);
  }
  const float per = 1.0f / (float)a.D;
  int turn = 0;
  for (int64_t r = (int64_t)blockIdx.x * kAt + (W == 1 ? wave : 0); r < a.T;
       r += (int64_t)gridDim.x * kAt, turn ^= 1) {
    const T* xr = static_cast<const T*>(a.x) + r * a.ldx;
    const T* dr = static_cast<const T*>(a.dy) + r * a.ldy;
    u32x4 x[K], d[K];
#pragma unroll
    for (int k = 0; k < K; ++k) x[k] = load_chunk(xr, at + k * kNext, a.D);
#pragma unroll
    for (int k = 0; k < K; ++k) d[k] = load_chunk(dr, at + k * kNext, a.D);
    const float mean = kRms ? 0.f : a.mean_in[r], rstd = a.rstd_in[r];
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
    row_sums<W>(s, red[turn], wave);
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
      store_chunk(out, at + k * kNext, a.D, f);
    }
  }
  // the sums of the waves that hold the same columns, then the workgroup's row of parts
  __shared__ float all[W == 1 ? 3 : 1][W == 1 ? 64 * K * E : 1];
  auto leave = [&](float (&sum)[K][E], float* part) {
    if constexpr (W == 1) {
      __syncthreads();
      if (wave > 0) {
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
          for (int e = 0; e < E; ++e) all[wave - 1][(k * E + e) * 64 + lane] = sum[k][e];
      }
      __syncthreads();
      if (wave > 0) return;
#pragma unroll
      for (int k = 0; k < K; ++k)
#pragma unroll
        for (int e = 0; e < E; ++e)
#pragma unroll
          for (int v = 0; v < 3; ++v) sum[k][e] = sum[k][e] + all[v][(k * E + e) * 64 + lane];
    }
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (at + k * kNext + e < a.D) part[at + k * kNext + e] = sum[k][e];
  };
  float* part = a.parts + blockIdx.x * a.D;
  if (a.dweight) leave(dw, part);
  if (a.dbias) leave(db, part + a.n_parts * a.D);
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

// f.run<W, K>() for the shape.
template <typename F>
hipError_t with_shape(NormShape s, F f) {
  if (s.waves == 1) {
    if (s.chunks == 1) return f.template run<1, 1>();
    if (s.chunks == 2) return f.template run<1, 2>();
    return f.template run<1, 4>();
  }
  if (s.waves == 4) {
    if (s.chunks == 1) return f.template run<4, 1>();
    if (s.chunks == 2) return f.template run<4, 2>();
    return f.template run<4, 4>();
  }
  if (s.chunks == 2) return f.template run<16, 2>();
  if (s.chunks == 4) return f.template run<16, 4>();
  return f.template run<16, 8>();
}

template <typename T, bool kRms>
struct Forward {
  const NormArgs& a;
  hipStream_t st;
  template <int W, int K>
  hipError_t run() {
    const int rows = W < 4 ? 4 / W : 1;
    return launch(k_norm<T, W, K, kRms>, dim3((unsigned)ceil_div(a.T, rows)),
                  W < 4 ? 256 : 64 * W, 0, st, a);
  }
};

template <typename T, bool kRms>
struct Backward {
  const NormArgs& a;
  hipStream_t st;
  template <int W, int K>
  hipError_t run() {
    return launch(k_norm_grad<T, W, K, kRms>, dim3((unsigned)a.n_parts), W < 4 ? 256 : 64 * W, 0,
                  st, a);
  }
};

template <template <typename, bool> class Pass>
hipError_t pass(const NormArgs& a, bool grad, hipStream_t st) {
  const NormShape s = norm_shape(a.T, a.D, a.bf16, grad);
  if (a.bf16)
    return a.rms ? with_shape(s, Pass<uint16_t, true>{a, st})
                 : with_shape(s, Pass<uint16_t, false>{a, st});
  return a.rms ? with_shape(s, Pass<float, true>{a, st}) : with_shape(s, Pass<float, false>{a, st});
}

}  // namespace

NormShape norm_shape(int64_t rows, int64_t width, bool bf16, bool grad) {
  (void)rows, (void)grad;
  const int64_t c = ceil_div(width, bf16 ? 8 : 4);
  if (c <= 64) return {1, 1};
  if (c <= 128) return {1, 2};
  if (c <= 256) return {1, 4};
  if (c <= 512) return {4, 2};
  if (c <= 1024) return {4, 4};
  if (c <= 2048) return {16, 2};
  if (c <= 4096) return {16, 4};
  return {16, 8};
}

hipError_t launch_norm(const NormArgs& a, hipStream_t st) { return pass<Forward>(a, false, st); }

hipError_t launch_norm_grad(const NormArgs& a, hipStream_t st) {
  if (a.n_parts > 0)
    if (const hipError_t e = pass<Backward>(a, true, st)) return e;
  if (!a.dweight && !a.dbias) return hipSuccess;
  const dim3 grid((unsigned)ceil_div(a.D, 64), a.dweight && a.dbias ? 2 : 1);
  return a.bf16 ? launch(k_norm_sum<uint16_t>, grid, 64 * kSumWaves, 0, st, a)
                : launch(k_norm_sum<float>, grid, 64 * kSumWaves, 0, st, a);
}

}  // namespace flr
