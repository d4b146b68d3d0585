// flr_head.h -- types shared by the C-ABI layer of the output head's operators
// (flround_head_api.cpp) and their gfx950 kernels (flround_head.hip,
// flround_top.hip).  Not part of the public ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "flr_launch.h"

namespace flr {

constexpr int kRowPad = 256;      // compacted rows are padded to this many
constexpr int kStep = 64;         // elements of the summed axis a tile takes at a time
constexpr int kMaxTargets = 128;  // listed teacher logits per token

// The gradient of a call of up to this many tokens, whether they take part or not,
// has two rows for each: G rounded to bf16, and what that leaves, rounded too, which
// makes G's error 2^-16 of an entry instead of 2^-8.  Of 50257 words, 1024 wide, the
// gradients of 32 tokens are off by at most 1.7e-3 in the 2-norm, the results' own
// rounding; those of 33 tokens, with one row each, by 1.8e-3 to 1.9e-3 with labels and
// 2.3e-3 to 2.5e-3 with 16 listed words.  Both rows of 32 tokens fit the products'
// smallest tiles, of 64 rows (102 and 110 us; 33 tokens 97 and 105); beyond, the two
// products after G would be twice as long.  The choice is the host's, which does not
// know how many tokens take part.
constexpr int kTwiceTokens = 32;

// Written by the first kernel of a call.
struct HeadHeader {
  int32_t n_live;   // rows of the tokens that take part
  float scale;      // largest finite |dloss| among them (1 where that is 0)
  int32_t pad[2];
  uint32_t zero[4]; // what a load past an operand's end reads
};

// Arguments of the small kernels around the products.  A token that takes
// part is "live"; the q-th live token is row q of the compacted arrays (rows 2 q and
// 2 q + 1 where copies is 2).
struct HeadArgs {
  int64_t T, V, D, Dp;              // Dp: row length of hc (and of wc), a multiple of kStep
  int64_t ldh, ldw;                 // elements between rows of hidden and of weight
  const uint16_t* hidden;
  const uint16_t* weight;
  int copies;                       // compacted rows per token: 1, or 2 (kTwiceTokens)
  int K;                            // targets per token (1 for labels)
  float tau;
  const int64_t* labels;            // labels, or null:
  const int32_t* ids;               //   T x K
  const float* teacher;             //   T x K
  const float* teacher_lse;         //   T, or null
  const float* lse_in;              // gradient: T
  const float* target_in;           // gradient: T x K
  const float* dloss;               // gradient: T
  float* loss;                      // forward outputs
  float* lse;
  float* target;
  uint16_t* dhidden;                // gradient outputs
  // workspace
  HeadHeader* hdr;
  int32_t* rows;                    // live row -> token
  int32_t* pos;                     // token -> live row, or -1
  float* logp;                      // T x K (distillation), -inf where nothing is listed
  float* mass;                      // T (distillation): sum of p, NaN for an id past the vocabulary
  uint8_t* flag;                    // T (distillation): token takes part
  uint16_t* hc;                     // compacted hidden rows, Dp each
  uint16_t* wc;                     // weight rows of Dp each, or null: weight is used as it is
  float* row_lse;                   // gradient, per live row: lse
  float* row_coef;                  // gradient, per live row: dloss / scale * mass
  int32_t* row_label;               // gradient of the labels' loss, per live row: the label,
  float* row_spot;                  // and its entry of G
  const float2* parts;              // per (p tile, live row): maximum, and sum of exp over it
  int n_parts;
  int64_t rows_pad;                 // T rounded up to kRowPad
};

// One tiled product.  P supplies the four consecutive outputs of a lane, Q
// the lane's own row: out[q][p] = sum over k of P(p, k) Q(q, k).
struct TileArgs {
  const uint16_t* P;
  const uint16_t* Q;
  int64_t ldp, ldq;                 // elements between rows in memory
  int64_t np, nq;                   // valid outputs along p and q
  int64_t nk;                       // length of the summed axis
  const HeadHeader* hdr;
  int live_q;                       // nq is hdr->n_live
  int live_k;                       // nk is hdr->n_live
  const uint16_t* zero;             // 16 zero bytes
  // epilogues
  float s2;                         // logits: log2(e) / tau
  float2* parts;                    // statistics
  int64_t parts_ld;
  float inv_tau;                    // gradient of the logits: 1 / tau
  const float* row_lse;
  const float* row_coef;
  const int32_t* row_label;         // or null
  const float* row_spot;
  int64_t p_first;                  // the word that p = 0 is
  uint16_t* G;
  int64_t ldg;                      // also the columns of G to write
  int copies;                       // 2: odd rows hold what rounding left of the even ones
  float* slab;                      // fp32 sums: slab[split][live row][ld_slab]
  int64_t ld_slab;
  int add;                          // add to the slab
  int max_splits;
  uint16_t* out;                    // bf16 output, scaled by hdr->scale * out_scale
  int64_t ld_out;
  int vec_out;                      // rows of out are 16-byte aligned and whole eights long
  float out_scale;
};

enum TileShape { kTile256 = 0, kTile128 = 1, kTile64 = 2, kTile16 = 3 };
inline int tile_p(int s) { return s == kTile256 ? 256 : 128; }
inline int tile_q(int s) { return s == kTile256 ? 256 : s == kTile128 ? 128 : s == kTile64 ? 64 : 16; }

inline int tile_fit(int s) {   // tiles that the chip holds at a time, by LDS
  return 256 * (s == kTile256 ? 1 : s == kTile128 ? 2 : s == kTile64 ? 3 : 4);
}
// How many ways the summed axis is split: as many as fill the chip where the
// live rows make few tiles.
__host__ __device__ inline int splits_of(int fit, int tiles, int max_splits) {
  const int s = tiles > 0 ? fit / tiles : 1;
  return s < 1 ? 1 : s < max_splits ? s : max_splits;
}

hipError_t launch_head_teacher(const HeadArgs& a, hipStream_t st);
// The live tokens and their rows.
hipError_t launch_head_pack(const HeadArgs& a, bool grad, hipStream_t st);
hipError_t launch_head_pack_weight(const HeadArgs& a, hipStream_t st);
hipError_t launch_head_finish(const HeadArgs& a, hipStream_t st);
hipError_t launch_head_fix(const HeadArgs& a, uint16_t* G, int64_t ldg, int64_t v0, int64_t v1,
                           hipStream_t st);
hipError_t launch_head_dh(const HeadArgs& a, const float* slab, int64_t ld_slab, int shape,
                          int max_splits, float out_scale, hipStream_t st);
hipError_t launch_logits_stats(const TileArgs& a, int shape, hipStream_t st);
hipError_t launch_logits_grad(const TileArgs& a, int shape, hipStream_t st);
// The sums for the hidden state's gradient (nothing if it has no rows), and the
// weight's gradient.
hipError_t launch_grads(const TileArgs& h, int h_shape, const TileArgs& w, int w_shape,
                        hipStream_t st);

// Top logits.
constexpr int kTopThreads = 512;
constexpr int kTopMaxChunks = 8;        // 16-byte chunks per thread
constexpr int64_t kTopMaxEntries = 8192; // of a row's segment lists where shorter segments are chosen (65 x 128 at most)

struct TopArgs {
  const void* logits;
  int64_t rows, vocab, stride;      // stride: elements between rows
  int bf16;
  int k;
  float tau, s2;                    // s2: log2(e) / tau
  float* values;
  int32_t* ids;
  float* lse;                       // may be null
  int chunks, segs;                 // chunks per thread of a segment, segments per row
  uint64_t* lists;                  // rows x segs x k, sorted; 0: nothing
  float2* parts;                    // rows x segs
};
hipError_t launch_top(const TopArgs& a, hipStream_t st);

}  // namespace flr
