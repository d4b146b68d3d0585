// flr_layers.h -- types shared by the C-ABI layer of the embedding and the layer
// norm (flround_layers_api.cpp) and their gfx950 kernels (flround_embed.hip,
// flround_norm.hip).  Not part of the public ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace flr {

// Whether an array is more than the eight L2s hold: what is read or written of it once goes
// past them.
inline bool past_l2(int64_t bytes) { return bytes > (int64_t)32 << 20; }

// Threads of one launch, of which HIP takes less than 2^32: what needs more takes several
// (each of them milliseconds long, so that another costs nothing).
constexpr int64_t kMaxLaunchThreads = (int64_t)1 << 31;

// The embedding and its gradient.
struct EmbedArgs {
  int64_t T, V, D, ld;     // ld: elements between rows of the input
  bool bf16;               // elements of all rows: bf16, or fp32
  const int64_t* ids;
  const void* in;          // the weight (V rows), or the gradient of the output (T rows)
  float scale;
  void* out;               // T x D, or the weight's gradient (V x D)
  int add;                 // gradient: added to what stands there
  // gradient's plan and workspace
  int64_t zeros;           // elements of the table, from its first on, zeroed beside the sort
  int words;               // words whose tokens one workgroup of the sort finds
  int sort_waves;
  int list;                // found tokens that a wave of the sort can list
  int tile;                // sorted tokens that one wave sums
  int32_t* start;          // V + 1: word v's tokens are order[start[v] .. start[v + 1])
  int2* order;             // (token, word), by word, a word's tokens in ascending order
  float* slab;             // two rows per tile: sums of words that go on beyond it
  int64_t ld_slab;
};

// Waves to a row of the input, which has a chunk of 16 bytes for each lane.
inline int embed_pieces(const EmbedArgs& a) {
  const int64_t wave = 64 * (a.bf16 ? 8 : 4);
  return (int)((a.D + wave - 1) / wave);
}

// Tokens up to which the gradient is one launch, whose workgroups all read all ids (1000
// tokens into 5000 x 1024: 12.5 us, 14.1 by the sort, but 22 and 18.6 where nine of ten are
// one word; 512 tokens into 128256 x 4096 185 us, 513 by the sort 193).  It takes no
// workspace.
constexpr int kEmbedFew = 512;
constexpr int kEmbedMaxWords = 512;
constexpr int kEmbedMaxWaves = 16;
// Found tokens that a wave of the sort lists: half of its share of 32768 tokens.  (Added to
// 32000 x 2048: 32768 tokens, 30 % of them one word, 74 us for the gradient, 91 with a list
// of 512, as the ids of a share are read again where it is full; 131072 without a frequent
// word 207 and 293.  With 90 % one word the list is full either way: 91 and 300.)
constexpr int kEmbedMaxList = 1024;

// The layer norm and its gradient.
struct NormArgs {
  int64_t T, D, ldx, ldy;  // ldy: elements between rows of dy
  bool bf16, rms;
  const void* x;
  const void* weight;      // null: ones
  const void* bias;        // null: zeros
  float eps;
  const float* mean_in;    // gradient
  const float* rstd_in;
  const void* dy;
  void* y;                 // or dx
  float* mean;             // may be null
  float* rstd;
  void* dweight;           // either may be null
  void* dbias;
  float* parts;            // n_parts rows of D for dweight, then as many for dbias
  int64_t n_parts;         // workgroups of the gradient
};

// Whether the gradient is one launch (up to 512 rows), which takes no workspace.
inline bool norm_few(int64_t rows, int64_t width, bool bf16) {
  return rows > 0 && rows <= 512 && width <= 1024 * (bf16 ? 8 : 4);
}

// Rows that a workgroup of the gradient takes at once.
int norm_rows(int64_t width, bool bf16);

hipError_t launch_norm(const NormArgs& a, hipStream_t st);
hipError_t launch_norm_grad(const NormArgs& a, hipStream_t st);

// Up to kMaxLaunchThreads.
hipError_t launch_embed(const EmbedArgs& a, hipStream_t st);
hipError_t launch_embed_grad(const EmbedArgs& a, hipStream_t st);
// Zeros to n elements, a thread to each chunk of 16 bytes.
hipError_t launch_embed_zeros(void* out, int64_t n, bool bf16, hipStream_t st);

}  // namespace flr
