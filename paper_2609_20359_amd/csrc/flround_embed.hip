// flround_embed.hip -- gfx950 kernels of the embedding and its gradient.
//
// Both move rows and compute next to nothing, so all that counts is bytes in flight
// and, for the gradient, that no row is summed in an order that depends on timing:
// the tokens are sorted by word without atomics on memory, and each word's rows are
// added in ascending order of its tokens.
#include "flr_launch.h"
#include "flr_layers.h"
#include "flr_rows.h"

namespace flr {
namespace {

// A value that a whole wave reads at one address.
template <typename T>
__device__ __forceinline__ T uniform(const T* p) {
  return *(const __attribute__((address_space(4))) T*)(uintptr_t)p;
}

constexpr int kPiece = 4;   // chunks of a row that a lane holds at a time

// out[t] = scale * weight[ids[t]].  A wave takes a piece of a row, all of its loads
// first.
template <typename T>
__global__ void __launch_bounds__(256) k_embed(const EmbedArgs a, int pieces) {
  constexpr int E = Rows<T>::kE;
  const int lane = threadIdx.x & 63;
  const int64_t w = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int64_t t = w / pieces;
  if (t >= a.T) return;
  const int64_t at = ((w - t * pieces) * kPiece * 64 + lane) * E;
  const int64_t id = uniform(a.ids + t);
  T* out = static_cast<T*>(a.out) + t * a.D;
  u32x4 x[kPiece];
  if (id >= 0 && id < a.V) {
    const T* row = static_cast<const T*>(a.in) + id * a.ld;
#pragma unroll
    for (int i = 0; i < kPiece; ++i) x[i] = load_chunk(row, at + i * 64 * E, a.D);
  }
#pragma unroll
  for (int i = 0; i < kPiece; ++i) {
    float f[E];
    Rows<T>::floats(x[i], f);
#pragma unroll
    for (int e = 0; e < E; ++e)
      f[e] = id < 0 ? 0.f : id >= a.V ? __builtin_nanf("") : f[e] * a.scale;
    store_chunk(out, at + i * 64 * E, a.D, f);
  }
}

// The tokens by word.  A workgroup finds those of a.words words, and where they begin
// among all, by reading every id twice: first each wave counts its share of the tokens
// (a section of them, in order) for each word, and the tokens of all lower words; then,
// from the sums of these counts, it knows where its next token of each word goes.  So
// one launch sorts, stably, and nothing depends on which wave comes first.
__global__ void __launch_bounds__(64 * kEmbedMaxWaves) k_embed_sort(const EmbedArgs a) {
  extern __shared__ int32_t next[];   // [wave][word]
  __shared__ int32_t sums[kEmbedMaxWaves];
  __shared__ int32_t below_all;
  const int waves = blockDim.x / 64, lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int64_t v0 = (int64_t)blockIdx.x * a.words;
  const int nv = (int)(a.V - v0 < a.words ? a.V - v0 : a.words);
  for (int i = threadIdx.x; i < waves * a.words; i += blockDim.x) next[i] = 0;
  if (threadIdx.x == 0) below_all = 0;
  __syncthreads();
  const int64_t share = ((a.T + waves * 64 - 1) / (waves * 64)) * 64;
  const int64_t t0 = wave * share, t1 = t0 + share < a.T ? t0 + share : a.T;
  volatile int32_t* mine = next + wave * a.words;   // (its lanes write for each other)
  int below = 0;
#pragma unroll 4
  for (int64_t t = t0 + lane; t < t1; t += 64) {
    const int64_t id = a.ids[t];
    if (id >= 0 && id < v0) ++below;
    if (id >= v0 && id < v0 + nv) atomicAdd(next + wave * a.words + (id - v0), 1);
  }
  if (below) atomicAdd(&below_all, below);
  __syncthreads();
  // where each word begins: thread j sums words j * per .. + per - 1
  const int per = (nv + blockDim.x - 1) / blockDim.x;
  const int w0 = threadIdx.x * per, w1 = w0 + per < nv ? w0 + per : nv;
  int total = 0;
  for (int w = w0; w < w1; ++w)
    for (int k = 0; k < waves; ++k) total += next[k * a.words + w];
  int upto = total;   // of the threads of this wave up to this one
  for (int d = 1; d < 64; d *= 2) {
    const int o = __shfl_up(upto, d);
    if (lane >= d) upto += o;
  }
  if (lane == 63) sums[wave] = upto;
  __syncthreads();
  int at = below_all + upto - total;
  for (int k = 0; k < wave; ++k) at += sums[k];
  for (int w = w0; w < w1; ++w) {
    a.start[v0 + w] = at;
    for (int k = 0; k < waves; ++k) {
      const int c = next[k * a.words + w];
      next[k * a.words + w] = at;
      at += c;
    }
  }
  if (v0 + nv == a.V && threadIdx.x == 0) {
    int n = below_all;
    for (int k = 0; k < waves; ++k) n += sums[k];
    a.start[a.V] = n;
  }
  __syncthreads();
  for (int64_t t = t0; t < t1; t += 64) {
    const int64_t id = t + lane < t1 ? a.ids[t + lane] : -1;
    const bool here = id >= v0 && id < v0 + nv;
    uint64_t left = __ballot(here);
    const int word = here ? (int)(id - v0) : -1;
    while (left) {   // one word of these 64 tokens at a time
      const int w = __builtin_amdgcn_readlane(word, __builtin_ctzll(left));
      const uint64_t same = __ballot(word == w);
      const int first = mine[w];
      if (word == w)
        a.order[first + __popcll(same & ((1ull << lane) - 1))] = (int32_t)(t + lane);
      if (lane == 0) mine[w] = first + __popcll(same);
      left &= ~same;
    }
  }
}

// scale * sum, beside what stands there, into the gradient's row (from column `at` on).
template <typename T>
__device__ __forceinline__ void write_row(const EmbedArgs& a, int64_t word, int64_t at,
                                          const float acc[Rows<T>::kE]) {
  constexpr int E = Rows<T>::kE;
  T* row = static_cast<T*>(a.out) + word * a.D;
  float f[E];
#pragma unroll
  for (int e = 0; e < E; ++e) f[e] = acc[e] * a.scale;
  if (a.add) {
    float old[E];
    Rows<T>::floats(load_chunk(row, at, a.D), old);
#pragma unroll
    for (int e = 0; e < E; ++e) f[e] = old[e] + f[e];
  }
  store_chunk(row, at, a.D, f);
}

// Sums of the sorted tokens' rows (the first sum_blocks workgroups) and zeros for the
// words without a token (the others).  A wave sums a tile of tokens, one chunk per lane:
// words that lie in the tile are done, those that begin before it or go on beyond it
// leave their part in the slab (rows 0 and 1 of the tile's).
template <typename T>
__global__ void __launch_bounds__(256) k_embed_sum(const EmbedArgs a, int pieces,
                                                   int64_t sum_blocks) {
  constexpr int E = Rows<T>::kE;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  if (blockIdx.x >= sum_blocks) {
    const int64_t v = (blockIdx.x - sum_blocks) * 4 + wave;
    if (v >= a.V || uniform(a.start + v) != uniform(a.start + v + 1)) return;
    const float zero[E] = {};
    T* row = static_cast<T*>(a.out) + v * a.D;
    for (int64_t at = lane * E; at < a.D; at += 64 * E) store_chunk(row, at, a.D, zero);
    return;
  }
  const int64_t w = (int64_t)blockIdx.x * 4 + wave;
  const int64_t tile = w / pieces;
  const int64_t at = ((w - tile * pieces) * 64 + lane) * E;
  const int n = uniform(a.start + a.V);
  const int64_t p0 = tile * a.tile;
  if (p0 >= n) return;
  const int count = (int)(n - p0 < a.tile ? n - p0 : a.tile);
  // lane i: token i of the tile, and its word
  const int token = lane < count ? a.order[p0 + lane] : 0;
  const int word = (int)a.ids[token];
  const T* in = static_cast<const T*>(a.in);
  float acc[E] = {};
  int now = __builtin_amdgcn_readlane(word, 0);
  bool whole = uniform(a.start + now) >= p0;   // it begins in this tile
  float* slab = a.slab + 2 * tile * a.D;
  auto park = [&](int slot) {
    if (at < a.D) {
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (at + e < a.D) slab[slot * a.D + at + e] = acc[e];
    }
  };
  constexpr int kAhead = 8;
  for (int i0 = 0; i0 < count; i0 += kAhead) {
    u32x4 x[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int t = __builtin_amdgcn_readlane(token, (i0 + i) & 63);
      if (i0 + i < count) x[i] = load_chunk(in + t * a.ld, at, a.D);
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      if (i0 + i >= count) break;
      const int next = __builtin_amdgcn_readlane(word, i0 + i);
      if (next != now) {
        if (whole) {
          if (at < a.D) write_row<T>(a, now, at, acc);
        } else {
          park(0);
        }
        now = next, whole = true;
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] = 0.f;
      }
      float f[E];
      Rows<T>::floats(x[i], f);
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] = acc[e] + f[e];
    }
  }
  if (uniform(a.start + now + 1) > p0 + count) park(whole ? 1 : 0);
  else if (!whole) park(0);
  else if (at < a.D) write_row<T>(a, now, at, acc);
}

// A word that begins in a tile and goes on beyond it: its parts in ascending order.
template <typename T>
__global__ void __launch_bounds__(256) k_embed_join(const EmbedArgs a, int pieces) {
  constexpr int E = Rows<T>::kE;
  const int lane = threadIdx.x & 63;
  const int64_t w = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int64_t tile = w / pieces;
  const int64_t at = ((w - tile * pieces) * 64 + lane) * E;
  const int n = uniform(a.start + a.V);
  const int64_t p1 = (tile + 1) * a.tile;
  if (p1 >= n) return;
  const int word = (int)uniform(a.ids + uniform(a.order + p1 - 1));
  const int end = uniform(a.start + word + 1);
  if (end <= p1 || uniform(a.start + word) < p1 - a.tile) return;
  if (at >= a.D) return;
  const int64_t last = (end - 1) / a.tile;
  float acc[E];
  const float* part = a.slab + (2 * tile + 1) * a.D + at;
#pragma unroll
  for (int e = 0; e < E; ++e) acc[e] = at + e < a.D ? part[e] : 0.f;
  part += a.D;   // row 0 of the next tile
#pragma unroll 4
  for (int64_t t = tile + 1; t <= last; ++t, part += 2 * a.D) {
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = acc[e] + (at + e < a.D ? part[e] : 0.f);
  }
  write_row<T>(a, word, at, acc);
}

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

template <typename T>
hipError_t embed(const EmbedArgs& a, hipStream_t st) {
  const int pieces = (int)ceil_div(a.D, kPiece * 64 * Rows<T>::kE);
  return launch(k_embed<T>, dim3((unsigned)ceil_div(a.T * pieces, 4)), 256, 0, st, a, pieces);
}

template <typename T>
hipError_t embed_grad(const EmbedArgs& a, hipStream_t st) {
  const int pieces = (int)ceil_div(a.D, 64 * Rows<T>::kE);
  const int64_t tiles = ceil_div(a.T, a.tile);
  const size_t lds = (size_t)a.sort_waves * a.words * sizeof(int32_t);
  if (const hipError_t e = launch(k_embed_sort, dim3((unsigned)ceil_div(a.V, a.words)),
                                  64 * a.sort_waves, lds, st, a))
    return e;
  const int64_t sums = ceil_div(tiles * pieces, 4), zeros = a.add ? 0 : ceil_div(a.V, 4);
  if (sums + zeros == 0) return hipSuccess;
  if (const hipError_t e =
          launch(k_embed_sum<T>, dim3((unsigned)(sums + zeros)), 256, 0, st, a, pieces, sums))
    return e;
  return tiles > 1 ? launch(k_embed_join<T>, dim3((unsigned)sums), 256, 0, st, a, pieces)
                   : hipSuccess;
}

}  // namespace

hipError_t launch_embed(const EmbedArgs& a, hipStream_t st) {
  return a.bf16 ? embed<uint16_t>(a, st) : embed<float>(a, st);
}

hipError_t launch_embed_grad(const EmbedArgs& a, hipStream_t st) {
  return a.bf16 ? embed_grad<uint16_t>(a, st) : embed_grad<float>(a, st);
}

}  // namespace flr
