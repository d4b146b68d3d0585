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

// out[t] = scale * weight[ids[t]], one chunk to a lane, so that all that is read and
// written at a time lies together.  Outputs larger than the L2s go past them (16384 rows
// of 8 KiB, of 7 k words: 31.4 us, 6.1 TB/s; 46 through the caches, 43 with four chunks to
// a lane).
template <typename T, bool kPast>
__global__ void __launch_bounds__(256) k_embed(const EmbedArgs a, int pieces) {
  constexpr int E = Rows<T>::kE;
  const int lane = threadIdx.x & 63;
  const int64_t w = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int64_t t = w / pieces;
  if (t >= a.T) return;
  const int64_t at = ((w - t * pieces) * 64 + lane) * E;
  const int64_t id = uniform(a.ids + t);
  T* out = static_cast<T*>(a.out) + t * a.D;
  u32x4 x{0, 0, 0, 0};
  if (id >= 0 && id < a.V) x = load_chunk(static_cast<const T*>(a.in) + id * a.ld, at, a.D);
  float f[E];
  Rows<T>::floats(x, f);
#pragma unroll
  for (int e = 0; e < E; ++e)
    f[e] = id < 0 ? 0.f : id >= a.V ? __builtin_nanf("") : f[e] * a.scale;
  store_chunk<kPast>(out, at, a.D, f);
}

// The tokens by word.  A workgroup finds those of a.words words, and where they begin
// among all, by reading every id: each wave counts its share of the tokens (a section of
// them, in order) for each word, and the tokens of all lower words; from the sums of
// these counts it knows where its next token of each word goes.  So one launch sorts,
// stably, and nothing depends on which wave comes first.  A wave lists the tokens that it
// finds (few, as all workgroups read all tokens) and handles 64 of its list at a time;
// one that finds more than the list holds reads the ids of its share again instead.
//
// 32768 tokens take 23 us, 6.5 of them reading the ids, which all waves do alike; the rest
// is the workgroup of a word that 30 % of the tokens are.  4096 tokens take 9.  The reading
// grows as the tokens times the workgroups (256, or the words over 512).
//
// The workgroups behind those that sort fill the gradient with zeros meanwhile; the rows
// of the words that occur are written by the next launch.

constexpr int kIds = 16;   // ids that a lane holds at a time

// Ids that are no words (< 0, or past 32 bits) as 2^32 - 1; those from V on are no
// workgroup's.
__device__ __forceinline__ unsigned word_of(int2 id) { return id.y != 0 ? ~0u : (unsigned)id.x; }

// One chunk to a thread, so that all that is written at a time lies together (128 k rows of
// 8 KiB beside the sort: 165 to 172 us; 2 chunks 180, 4 chunks 184), and past the caches.
template <typename T>
__device__ __forceinline__ void fill_zero(void* out, int64_t n, int64_t block) {
  constexpr int E = Rows<T>::kE;
  const float zero[E] = {};
  store_chunk<true>(static_cast<T*>(out), (block * blockDim.x + threadIdx.x) * E, n, zero);
}

// What the sort's launch has no threads for.
template <typename T>
__global__ void __launch_bounds__(256) k_embed_zeros(void* out, int64_t n) {
  fill_zero<T>(out, n, blockIdx.x);
}

template <typename T>
__global__ void __launch_bounds__(64 * kEmbedMaxWaves) k_embed_sort(const EmbedArgs a,
                                                                    int sort_blocks) {
  extern __shared__ int32_t lds[];   // next place [wave][word], then the waves' lists
  __shared__ int32_t sums[kEmbedMaxWaves], belows[kEmbedMaxWaves];
  if ((int)blockIdx.x >= sort_blocks) {
    fill_zero<T>(a.out, a.zeros, (int)blockIdx.x - sort_blocks);
    return;
  }
  const int waves = blockDim.x / 64, lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const unsigned v0 = blockIdx.x * a.words;
  const unsigned nv = (unsigned)(a.V - v0 < a.words ? a.V - v0 : a.words);
  const int share = (int)((a.T + waves * 64 - 1) / (waves * 64)) * 64;
  const int t0 = wave * share, t1 = t0 + share < (int)a.T ? t0 + share : (int)a.T;
  int32_t* next = lds;
  volatile int32_t* mine = next + wave * a.words;   // (its lanes write for each other)
  volatile uint32_t* list = reinterpret_cast<uint32_t*>(next + waves * a.words) + wave * a.list;
  for (int i = lane; i < a.words; i += 64) mine[i] = 0;
  const uint64_t lower = (1ull << lane) - 1;
  const int2* ids = reinterpret_cast<const int2*>(a.ids);
  // f(token, its word or 2^32 - 1) for 64 tokens of the share at a time
  auto every = [&](auto f) {
    for (int t = t0; t < t1; t += 64 * kIds) {
      int2 id[kIds];
#pragma unroll
      for (int k = 0; k < kIds; ++k) {
        const int at = t + 64 * k + lane;
        id[k] = at < t1 ? ids[at] : make_int2(-1, -1);
      }
#pragma unroll
      for (int k = 0; k < kIds; ++k) f(t + 64 * k + lane, word_of(id[k]));
    }
  };
  // f(token, its word less v0 or -1) for 64 tokens that are this workgroup's, or fewer
  int below = 0, found = 0;
  auto own = [&](auto f) {
    if (found <= a.list) {
      for (int i = 0; i < found; i += 64) {
        const uint32_t x = i + lane < found ? list[i + lane] : 0;
        f(t0 + (int)(x & 0xFFFF), i + lane < found ? (int)(x >> 16) : -1);
      }
    } else {
      every([&](int token, unsigned word) {
        const bool here = word - v0 < nv;
        if (__ballot(here)) f(token, here ? (int)(word - v0) : -1);
      });
    }
  };
  // How many of the lanes below this one have its word, and how many lanes in all.
  auto alike = [&](int w, int& rank, int& count) {
    uint64_t left = __ballot(w >= 0);
    rank = count = 0;
    while (left) {
      const int x = __builtin_amdgcn_readlane(w, __builtin_ctzll(left));
      const uint64_t same = __ballot(w == x);
      if (w == x) rank = __popcll(same & lower), count = __popcll(same);
      left &= ~same;
    }
  };
  every([&](int token, unsigned word) {
    below += word < v0 ? 1 : 0;
    const bool here = word - v0 < nv;
    const uint64_t at = __ballot(here);
    if (at) {
      const int place = found + __popcll(at & lower);
      if (here && place < a.list) list[place] = (word - v0) << 16 | (uint32_t)(token - t0);
      found += __popcll(at);
    }
  });
  own([&](int, int w) {
    int rank, count;
    alike(w, rank, count);
    if (w >= 0 && rank == 0) mine[w] = mine[w] + count;
  });
  for (int d = 32; d > 0; d /= 2) below += __shfl_xor(below, d);
  if (lane == 0) belows[wave] = below;
  __syncthreads();
  // where each word begins: thread j sums words j * per .. + per - 1
  const int per = (nv + blockDim.x - 1) / blockDim.x;
  const int w0 = threadIdx.x * per, w1 = w0 + per < (int)nv ? w0 + per : (int)nv;
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
  int at = upto - total, all = 0;
  for (int k = 0; k < waves; ++k) {
    if (k < wave) at += sums[k];
    at += belows[k];
    all += sums[k] + belows[k];
  }
  for (int w = w0; w < w1; ++w) {
    a.start[v0 + w] = at;
    for (int k = 0; k < waves; ++k) {
      const int c = next[k * a.words + w];
      next[k * a.words + w] = at;
      at += c;
    }
  }
  if (v0 + (int64_t)nv == a.V && threadIdx.x == 0) a.start[a.V] = all;
  __syncthreads();
  own([&](int token, int w) {
    const int first = w >= 0 ? mine[w] : 0;
    int rank, count;
    alike(w, rank, count);
    if (w >= 0) a.order[first + rank] = make_int2(token, (int)v0 + w);
    if (w >= 0 && rank == 0) mine[w] = first + count;
  });
}

// scale * sum, beside what stands there, into the gradient's row (from column `at` on).
template <typename T, bool kAdd, bool kPast = false>
__device__ __forceinline__ void write_row(const EmbedArgs& a, int64_t word, int64_t at,
                                          const float acc[Rows<T>::kE], u32x4 there) {
  constexpr int E = Rows<T>::kE;
  float f[E], old[E];
  Rows<T>::floats(there, old);
#pragma unroll
  for (int e = 0; e < E; ++e) f[e] = kAdd ? old[e] + acc[e] * a.scale : acc[e] * a.scale;
  store_chunk<kPast>(static_cast<T*>(a.out) + word * a.D, at, a.D, f);
}

constexpr int kJoinWaves = 8;

// Sums of the sorted tokens' rows.  A wave sums a tile of tokens, one chunk per lane:
// words that lie in the tile are done, those that begin before it or go on beyond it
// leave their part in the slab (rows 0 and 1 of the tile's).  What it reads of dout, and
// of the gradient where it adds to it, is asked for kAhead tokens ahead, in a loop: 16
// tokens at a time without one are code that is slower to fetch than the rows (32768
// tokens added to 32000 x 2048: 82 us for the gradient, 92 without the loop).  More rows
// than the L2s hold are read past them: 73.
template <typename T, bool kAdd, bool kPastIn, bool kPastOut>
__global__ void __launch_bounds__(256) k_embed_sum(const EmbedArgs a, int pieces) {
  constexpr int E = Rows<T>::kE, kAhead = 4;
  const int lane = threadIdx.x & 63;
  const int64_t w = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int64_t tile = w / pieces;
  const int64_t at = ((w - tile * pieces) * 64 + lane) * E;
  const int64_t p0 = tile * a.tile, p1 = p0 + a.tile;
  if (p0 >= a.T) return;
  // the tile's tokens with their words, one to a lane, and the words beside it
  const int2 mine = a.order[p0 + lane < a.T ? p0 + lane : a.T - 1];
  const int before = p0 > 0 ? uniform(&a.order[p0 - 1].y) : -1;
  const int behind = p1 < a.T ? uniform(&a.order[p1].y) : -1;
  const int n = uniform(a.start + a.V);
  if (p0 >= n) return;
  const int count = (int)(n < p1 ? n - p0 : a.tile);
  const int after = p1 < n ? behind : -1;   // the word that follows the tile's last
  const T* in = static_cast<const T*>(a.in);
  const T* out = static_cast<const T*>(a.out);
  float* slab = a.slab + 2 * tile * a.ld_slab + at;
  float acc[E] = {};
  bool whole = __builtin_amdgcn_readlane(mine.y, 0) != before;   // it begins in this tile
  u32x4 x[kAhead], old[kAhead];
  auto ask = [&](int i0) {
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      if (i0 + i >= count) continue;
      const int t = __builtin_amdgcn_readlane(mine.x, i0 + i);
      x[i] = load_chunk<kPastIn>(in + t * a.ld, at, a.D);
      if constexpr (kAdd) {
        const int64_t word = __builtin_amdgcn_readlane(mine.y, i0 + i);
        const int next = i0 + i + 1 < count ? __builtin_amdgcn_readlane(mine.y, i0 + i + 1) : after;
        if (word != next) old[i] = load_chunk(out + word * a.D, at, a.D);
      }
    }
  };
  ask(0);
#pragma unroll 1
  for (int i0 = 0; i0 < count; i0 += kAhead) {
    u32x4 now[kAhead], there[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      now[i] = x[i];
      there[i] = kAdd ? old[i] : u32x4{0, 0, 0, 0};
    }
    ask(i0 + kAhead);
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      if (i0 + i >= count) continue;
      float f[E];
      Rows<T>::floats(now[i], f);
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] = acc[e] + f[e];
      const bool last = i0 + i + 1 == count;
      const int word = __builtin_amdgcn_readlane(mine.y, i0 + i);
      const int next = last ? after : __builtin_amdgcn_readlane(mine.y, i0 + i + 1);
      if (word == next && !last) continue;
      if (at < a.D) {
        if (whole && word != next) {
          write_row<T, kAdd, kPastOut>(a, word, at, acc, there[i]);
        } else {
          f32x4* p = reinterpret_cast<f32x4*>(slab + (whole ? a.ld_slab : 0));
#pragma unroll
          for (int e = 0; e < E; e += 4)
            p[e / 4] = f32x4{acc[e], acc[e + 1], acc[e + 2], acc[e + 3]};
        }
      }
      whole = true;
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] = 0.f;
    }
  }
}

// A word that begins in a tile and goes on beyond it: every eighth of its parts in
// ascending order by each wave, then the waves' sums (a word of 9800 tokens x 2048: 7 us;
// 136 by one wave for each 512 columns).
template <typename T, bool kAdd>
__global__ void __launch_bounds__(64 * kJoinWaves) k_embed_join(const EmbedArgs a, int pieces) {
  constexpr int E = Rows<T>::kE;
  __shared__ float red[kJoinWaves][E][64];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int64_t tile = blockIdx.x / pieces;
  const int64_t at = ((blockIdx.x - tile * pieces) * 64 + lane) * E;
  const int64_t p0 = tile * a.tile, p1 = p0 + a.tile;
  if (p1 >= a.T) return;
  const int word = uniform(&a.order[p1 - 1].y), behind = uniform(&a.order[p1].y);
  const int before = p0 > 0 ? uniform(&a.order[p0 - 1].y) : -1;
  const int n = uniform(a.start + a.V);
  if (p1 >= n || behind != word || before == word) return;
  const int end = uniform(a.start + word + 1);
  u32x4 old{0, 0, 0, 0};
  if (kAdd && wave == 0) old = load_chunk(static_cast<const T*>(a.out) + word * a.D, at, a.D);
  const int parts = (int)((end - 1) / a.tile - tile) + 1;
  // part 0: row 1 of this tile's; part i: row 0 of tile + i
  const float* slab = a.slab + 2 * tile * a.ld_slab + at;
  float acc[E] = {};
  if (at < a.D) {
#pragma unroll 8
    for (int i = wave; i < parts; i += kJoinWaves) {
      const f32x4* p = reinterpret_cast<const f32x4*>(slab + (i == 0 ? 1 : 2 * (int64_t)i) * a.ld_slab);
#pragma unroll
      for (int e = 0; e < E; e += 4) {
        const f32x4 x = p[e / 4];
        acc[e] = acc[e] + x.x, acc[e + 1] = acc[e + 1] + x.y;
        acc[e + 2] = acc[e + 2] + x.z, acc[e + 3] = acc[e + 3] + x.w;
      }
    }
  }
#pragma unroll
  for (int e = 0; e < E; ++e) red[wave][e][lane] = acc[e];
  __syncthreads();
  if (wave > 0 || at >= a.D) return;
#pragma unroll
  for (int k = 1; k < kJoinWaves; ++k)
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = acc[e] + red[k][e][lane];
  write_row<T, kAdd>(a, word, at, acc, old);
}

// Few tokens need no sort: one launch does all of it.  A workgroup for a token and 64
// chunks of its row looks for the tokens of the same word by reading all ids; that of the
// word's first token sums their rows, every eighth of them in ascending order in each
// wave, then the waves' sums.  The workgroups behind these write zeros to the rows of
// some words each, but for those that occur.
// (333 tokens into 5003 x 321 fp32: 7.9 us, 14.4 by the sort and its two launches.)
constexpr int kFewIds = kEmbedFew / 64;   // ids that a lane holds
constexpr int kFewWaves = 8, kFewThreads = 64 * kFewWaves;
constexpr int kFewRows = 4;               // rows that a wave has asked for at a time
constexpr int kFewFill = 1024;            // words of a workgroup of zeros, at most

template <typename T, bool kAdd>
__global__ void __launch_bounds__(kFewThreads) k_embed_few(const EmbedArgs a, int pieces, int sum_blocks,
                                                   int fill_words) {
  constexpr int E = Rows<T>::kE;
  __shared__ float red[kFewWaves][E][64];
  __shared__ bool used[kFewFill];
  __shared__ int tokens_of[kEmbedFew];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int tokens = (int)a.T;
  if ((int)blockIdx.x >= sum_blocks) {
    const int64_t v0 = (int64_t)((int)blockIdx.x - sum_blocks) * fill_words;
    const int n = (int)(a.V - v0 < fill_words ? a.V - v0 : fill_words);
    for (int i = threadIdx.x; i < n; i += kFewThreads) used[i] = false;
    __syncthreads();
    for (int t = threadIdx.x; t < tokens; t += kFewThreads) {
      const int64_t id = a.ids[t];
      if (id >= v0 && id < v0 + n) used[id - v0] = true;
    }
    __syncthreads();
    const float zero[E] = {};
    const unsigned chunks = (unsigned)((a.D + E - 1) / E);
    for (unsigned c = threadIdx.x; c < n * chunks; c += kFewThreads) {
      const unsigned row = c / chunks;
      if (used[row]) continue;
      T* to = static_cast<T*>(a.out) + (v0 + row) * a.D;
      const int64_t k = (int64_t)(c - row * chunks) * E;
      store_chunk<true>(to, k, a.D, zero);
    }
    return;
  }
  const int t = blockIdx.x / pieces;
  const int64_t at = ((blockIdx.x - t * pieces) * 64 + lane) * E;
  int64_t id[kFewIds];
#pragma unroll
  for (int k = 0; k < kFewIds; ++k) id[k] = 64 * k + lane < tokens ? a.ids[64 * k + lane] : -1;
  const int64_t word = uniform(a.ids + t);
  if (word < 0 || word >= a.V) return;
  uint64_t same[kFewIds];
  int count = 0, first = -1;
#pragma unroll
  for (int k = 0; k < kFewIds; ++k) {
    same[k] = __ballot(id[k] == word);
    if (first < 0 && same[k]) first = 64 * k + __builtin_ctzll(same[k]);
    count += __popcll(same[k]);
  }
  if (first != t || (count == 1 && wave > 0)) return;
  const T* in = static_cast<const T*>(a.in);
  u32x4 old{0, 0, 0, 0};
  if (kAdd && wave == 0) old = load_chunk(static_cast<const T*>(a.out) + word * a.D, at, a.D);
  if (count > 1) {   // the word's tokens in ascending order: 64 ids to a wave at a time
    int before = 0;
#pragma unroll
    for (int k = 0; k < kFewIds; ++k) {
      if (k % kFewWaves == wave && id[k] == word)
        tokens_of[before + __popcll(same[k] & ((1ull << lane) - 1))] = 64 * k + lane;
      before += __popcll(same[k]);
    }
    __syncthreads();
  }
  float acc[E] = {};
  for (int i0 = wave; i0 < count; i0 += kFewWaves * kFewRows) {
    u32x4 x[kFewRows];
#pragma unroll
    for (int i = 0; i < kFewRows; ++i) {
      const int rank = i0 + i * kFewWaves;
      x[i] = u32x4{0, 0, 0, 0};
      if (rank < count)
        x[i] = load_chunk(in + (count > 1 ? tokens_of[rank] : t) * a.ld, at, a.D);
    }
#pragma unroll
    for (int i = 0; i < kFewRows; ++i) {
      float f[E];
      Rows<T>::floats(x[i], f);
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] = acc[e] + f[e];
    }
  }
  if (count > 1) {
#pragma unroll
    for (int e = 0; e < E; ++e) red[wave][e][lane] = acc[e];
    __syncthreads();
    if (wave > 0) return;
#pragma unroll
    for (int k = 1; k < kFewWaves; ++k)
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] = acc[e] + red[k][e][lane];
  }
  if (at < a.D) write_row<T, kAdd>(a, word, at, acc, old);
}

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

template <typename T>
hipError_t embed(const EmbedArgs& a, hipStream_t st) {
  const int pieces = embed_pieces(a);
  return launch(past_l2(a.T * a.D * (int64_t)sizeof(T)) ? k_embed<T, true> : k_embed<T, false>,
                dim3((unsigned)ceil_div(a.T * pieces, 4)), 256, 0, st, a, pieces);
}

template <typename T, bool kAdd>
hipError_t embed_grad(const EmbedArgs& a, hipStream_t st) {
  const int pieces = embed_pieces(a);
  if (a.T <= kEmbedFew) {
    // zeros of 16 KiB to a workgroup
    const int64_t row = a.D * (int64_t)sizeof(T);
    const int words = (int)(row < 16 ? kFewFill : row < 16384 ? 16384 / row : 1);
    const int64_t sums = a.T * pieces, fills = kAdd ? 0 : ceil_div(a.V, words);
    return sums + fills ? launch(k_embed_few<T, kAdd>, dim3((unsigned)(sums + fills)),
                                 kFewThreads, 0, st, a, pieces, (int)sums, words)
                        : hipSuccess;
  }
  const int64_t tiles = ceil_div(a.T, a.tile);
  const unsigned threads = 64 * a.sort_waves;
  const size_t lds = (size_t)a.sort_waves * (a.words + a.list) * sizeof(int32_t);
  const int64_t sorts = ceil_div(a.V, a.words);
  const int64_t fills = ceil_div(a.zeros, (int64_t)threads * Rows<T>::kE);
  if (const hipError_t e = launch(k_embed_sort<T>, dim3((unsigned)(sorts + fills)), threads, lds, st,
                                  a, (int)sorts))
    return e;
  const dim3 grid((unsigned)ceil_div(tiles * pieces, 4));
  const bool in = past_l2(a.T * a.D * (int64_t)sizeof(T)), out = past_l2(a.V * a.D * (int64_t)sizeof(T));
  if (const hipError_t e = launch(in ? (out ? k_embed_sum<T, kAdd, true, true>
                                            : k_embed_sum<T, kAdd, true, false>)
                                     : (out ? k_embed_sum<T, kAdd, false, true>
                                            : k_embed_sum<T, kAdd, false, false>),
                                  grid, 256, 0, st, a, pieces))
    return e;
  return launch(k_embed_join<T, kAdd>, dim3((unsigned)(tiles * pieces)), 64 * kJoinWaves, 0, st, a,
                pieces);
}

}  // namespace

hipError_t launch_embed(const EmbedArgs& a, hipStream_t st) {
  return a.bf16 ? embed<uint16_t>(a, st) : embed<float>(a, st);
}

hipError_t launch_embed_zeros(void* out, int64_t n, bool bf16, hipStream_t st) {
  const dim3 grid((unsigned)ceil_div(n, 256 * (bf16 ? 8 : 4)));
  return launch(bf16 ? k_embed_zeros<uint16_t> : k_embed_zeros<float>, grid, 256, 0, st, out, n);
}

hipError_t launch_embed_grad(const EmbedArgs& a, hipStream_t st) {
  if (a.add) return a.bf16 ? embed_grad<uint16_t, true>(a, st) : embed_grad<float, true>(a, st);
  return a.bf16 ? embed_grad<uint16_t, false>(a, st) : embed_grad<float, false>(a, st);
}

}  // namespace flr
