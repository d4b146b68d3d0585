// flround_head.hip -- gfx950 kernels of the output head: the cross entropy over
// the vocabulary, the distillation from a teacher's top logits, and their
// gradients.
//
// With z = h W^T (T tokens, V words, D wide), lse_t = log sum_v exp(z_tv / tau)
// and a target distribution p of mass M listed by a few words per token:
//     forward:   lse, and z at the listed words
//     gradient:  G_tv = dloss_t tau (M_t exp(z_tv / tau - lse_t) - p_tv),
//                dh = G W,  dW = G^T h
// z is never stored: the forward pass keeps a running maximum and sum per row,
// the gradient makes z again for a piece of the vocabulary and stores G of that
// piece in bf16.  Everything large is a matrix product on the matrix cores, so
// the file is one tiled product with four epilogues and the small kernels
// around it.
//
// Tokens that take no part are dropped first: the rest are copied to
// consecutive rows, so that no product spends time on them, and nothing that
// stands in their rows (infinities, NaN) reaches a sum.
#include "flr_head.h"

namespace flr {
namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 u32x4_at2 __attribute__((aligned(2)));   // on an element's boundary only

#define LDS_SPACE __attribute__((address_space(3)))
#define GLOBAL_SPACE __attribute__((address_space(1)))

constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{lo, hi}, bf16x2));
}
__device__ __forceinline__ uint16_t to_bf16(float x) { return (uint16_t)pack2(x, 0.f); }
// What rounding to bf16 leaves of x.
__device__ __forceinline__ float rest_of(float x) {
  return x - __uint_as_float((uint32_t)to_bf16(x) << 16);
}
__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

// (m, s) stands for s exp(m / tau), s2 being log2(e) / tau; a part of nothing is
// (-inf, 0).  Infinities have no difference: a maximum of +inf has an s > 0, here
// +inf, whose logarithm changes nothing.
__device__ __forceinline__ void join(float& m, float& s, float pm, float ps, float s2) {
  const float top = fmaxf(m, pm), ref = fabsf(top) == INFINITY ? 0.f : top;
  s = s * exp2_((m - ref) * s2) + ps * exp2_((pm - ref) * s2);
  m = top;
}

// ---- the tiled product ------------------------------------------------------
//
// A workgroup makes BP x BQ outputs, kStep of the summed axis at a time, from
// two stages of LDS: while the waves multiply one, the other is filled by loads
// that go from memory to LDS directly.  An operand comes in either order:
//
//   rows along the summed axis (TR = false): the stage holds B rows of 64
//   elements (128 B).  A fragment is one 16-byte read per lane (row l % 16,
//   elements 8 (l / 16) .. + 7).  The 16-byte chunk c of row r lies at place
//   c ^ (r & 7), so that the rows' equal chunks fall on different banks.
//
//   rows across it (TR = true): the stage holds 64 rows of B elements.  A
//   fragment is two transposing reads of 8 bytes: 16 lanes read 4 rows of 16
//   elements, and lane i gets column i.  A wave reads 32 bytes of each of 16
//   rows at a time, 8 (l / 16) + 0..3.  So that these fall on different banks,
//   what a wave loads at once (1024 B: 2 or 4 rows) is a block of its own, 64 B
//   on from where the last one ends (and 128 B more after every 8 rows where a
//   block has 2), and in a block the pairs of chunks of row r lie at place
//   c ^ r.
//
// The loads write LDS in lane order, so the places are permuted by permuting
// which global chunk a lane asks for.

// The same value, of which the compiler keeps nothing derived: it is to hold few
// registers across the loop below rather than save an addition in it.
__device__ __forceinline__ uint32_t pinned(uint32_t x) {
  asm volatile("" : "+v"(x));
  return x;
}

template <int B, int NT, bool TR>
struct Operand {
  static constexpr int kLoads = (B * 8 + NT - 1) / NT;   // 16-byte loads per thread and step
  static constexpr int kChunks = TR ? B / 8 : 8;         // 16-byte chunks per row
  static constexpr int kBlockRows = 64 / kChunks;        // rows per block (TR)
  static constexpr int kPitch = TR ? 1024 + 64 : 1024;   // bytes from block to block
  static constexpr int kSkip = TR && B == 256 ? 128 : 0; // and after every 8 rows
  static constexpr int kBytes = (B / 8 * kPitch + 8 * kSkip + 127) / 128 * 128;
  static_assert(B * 8 % NT == 0 || B * 8 < NT, "whole loads, or the first waves' alone");
  static_assert(!TR || B == 128 || B == 256, "blocks of whole rows");

  const char* base;       // of the tile
  uint32_t at[kLoads];    // byte offset of each load
  int64_t step;           // bytes per step

  __device__ __forceinline__ static int row(int tid, int c) { return (tid + c * NT) / kChunks; }
  __device__ __forceinline__ static int chunk(int tid, int c) {
    const int place = (tid + c * NT) % kChunks, r = row(tid, c);
    return TR ? place ^ (r % kBlockRows) << 1 : place ^ (r & 7);
  }
  // Where load c of a wave goes.
  __device__ __forceinline__ static char* place(char* lds, int wave, int c) {
    const int m = c * (NT / 64) + wave;
    return lds + m * kPitch + (m / 4) * kSkip;
  }

  // src: row 0 of the tile (TR = false: row b0, column 0; TR = true: row 0,
  // column b0); n: rows (TR = false) or columns (TR = true) from there on.
  // Those beyond n are replaced by ones that exist, their products are not
  // used.
  __device__ __forceinline__ void init(const uint16_t* src, int64_t ld, int64_t n, int tid) {
    base = reinterpret_cast<const char*>(src);
    step = TR ? (int64_t)kStep * ld * 2 : (int64_t)kStep * 2;
#pragma unroll
    for (int c = 0; c < kLoads; ++c) {
      const int r = row(tid, c), ch = chunk(tid, c);
      if (TR)
        at[c] = (uint32_t)((r * ld + (ch * 8 < n ? ch * 8 : 0)) * 2);
      else
        at[c] = (uint32_t)(((r < n ? r : (int)n - 1) * ld + ch * 8) * 2);
    }
  }

  // Loads [c0, c1) of step s.
  __device__ __forceinline__ void load(char* lds, int s, int wave, int c0, int c1) const {
    const char* b = base + s * step;
#pragma unroll
    for (int c = c0; c < c1; ++c)
      if (B * 8 % NT == 0 || wave * 64 < B * 8) {
        __builtin_amdgcn_global_load_lds((const GLOBAL_SPACE void*)(b + pinned(at[c])),
                                         (LDS_SPACE void*)place(lds, wave, c), 16, 0, 0);
      }
  }

  // The step that the summed axis ends inside: `left` elements of it remain (in
  // whole chunks where TR = false), the others are zero.
  __device__ __forceinline__ void load_tail(char* lds, int s, int wave, int c0, int c1, int tid,
                                            int left, const uint16_t* zero) const {
    const char* b = base + s * step;
#pragma unroll
    for (int c = c0; c < c1; ++c) {
      if (B * 8 % NT != 0 && wave * 64 >= B * 8) continue;
      const bool in = TR ? row(tid, c) < left : chunk(tid, c) * 8 < left;
      const char* p = in ? b + pinned(at[c]) : reinterpret_cast<const char*>(zero);
      __builtin_amdgcn_global_load_lds((const GLOBAL_SPACE void*)p,
                                       (LDS_SPACE void*)place(lds, wave, c), 16, 0, 0);
    }
  }

  // Place of this lane's part of the fragment at rows (columns) b0 of the tile.
  __device__ __forceinline__ static uint32_t lane_place(int b0, int l) {
    if (!TR) return (uint32_t)((b0 + (l & 15)) * 128 + (((l >> 4) ^ (l & 7)) * 16));
    const int g = l >> 4, r = (l & 15) >> 2;   // row 8 g + r, and 4 on
    const int x = r % kBlockRows;
    return (uint32_t)((g * 8 / kBlockRows + r / kBlockRows) * kPitch + g * kSkip + x * (B * 2) +
                      (l & 3) * 8 + ((b0 / 16) ^ x) * 32);
  }
  // Fragment 16 i rows (columns) on from 16 f0, lane_place()'s b0, in half ks of
  // the step.
  __device__ __forceinline__ static bf16x8 frag(const char* lds, uint32_t lane, int f0, int i, int ks,
                                                int l) {
    if (!TR)
      return *reinterpret_cast<const bf16x8*>(lds + (ks ? lane ^ 64 : lane) + i * 16 * 128);
    // (f0 + i) ^ x is f0 ^ x and the difference: where f0 is a multiple of
    // kBlockRows it depends on i's low bits alone
    const int x = ((l & 15) >> 2) % kBlockRows, low = i % kBlockRows;
    const int on = f0 % kBlockRows ? ((f0 + i) ^ x) - (f0 ^ x) : i - low + ((low ^ x) - x);
    const char* p = lds + lane + on * 32 + ks * (32 / kBlockRows * kPitch + 4 * kSkip);
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_SPACE s16x4*)p);
    const s16x4 hi =
        __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_SPACE s16x4*)(p + 4 / kBlockRows * kPitch));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  }
};

// All of this wave's loads to LDS and reads from it are done, and all other
// waves' too.  (A volatile statement that touches memory: neither the reads nor
// the loads on either side cross it.)
__device__ __forceinline__ void wait_and_meet() {
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// Two 16 x 16 results of a wave, each lane's four (along p) as bf16: a lane gets
// eight in a row, lanes 16 k .. 16 k + 15 those from 8 k of the 32 on.
__device__ __forceinline__ u32x4 eight(u32x2 a, u32x2 b) {
  u32x4 o;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    // rows of 16 lanes: a0 a1 a2 a3, b0 b1 b2 b3 -> a0 a1 b0 b1, a2 a3 b2 b3
    // -> a0 a2 b0 b2, a1 a3 b1 b3
    const auto x = __builtin_amdgcn_permlane32_swap(a[h], b[h], false, false);
    const auto y = __builtin_amdgcn_permlane16_swap(x[0], x[1], false, false);
    o[h] = y[0];
    o[2 + h] = y[1];
  }
  return o;
}

enum Epilogue { kStats, kGrad, kSlab, kOut };

// What bounds it: the matrix cores, at the clock that the power leaves them.
// They are busy in 78 % of the cycles of the loss's product and 66 to 68 % of
// the gradient's, no read of LDS meets a bank conflict, and a step of 256 x 256
// outputs takes 1.43 us.  4096 live rows, 128256 words, 4096 wide, in PFLOP/s:
// 1.37 for the statistics, 1.24 for G (0.87 ms a piece of 32256 words), 1.26 for
// dW (0.86 ms), 1.37 for dh (0.79 ms); the library's plain products of these
// sizes run at 1.43, 1.48 and 1.60.  What G and dW lose is the ends of their
// tiles: without the stores dW takes 0.77 ms, with all on a few lines 0.80, as a
// CU's 128 KiB go out at once and the next tile's first step waits for them.  2048
// and fewer rows lose 10 to 15 % where the weight comes from HBM in every round of
// tiles, a step's loads being one step ahead.
//
// The 256 x 256 tiles take all 256 registers of a lane and spill some: 15 of the
// statistics', 17 of G's, 4 of dW's, 8 of the sums', to 20 to 72 bytes of scratch.
// All of it is in a tile's last two steps and its epilogue, where the next tile's
// addresses are alive beside this one's; the loop over the steps has none.
//
// Why these tiles: eight waves of 128 x 64 outputs read 96 KiB of LDS a step of
// 64, a third of what LDS can give in that time, and keep their sums in 128
// registers; four waves of 128 x 128 read a third less, but ran at 1.02 against
// 1.27 (a plain product of 16384 x 4096 x 4096), alone on their SIMDs.  Reading
// fragments half a step ahead, with the loads between the products, took that
// product from 1.20 to 1.27, and to 1.50 without its fp32 output.
//
// Workgroups stay and take one tile after another, so that the loads of the next
// tile's first steps run under the last products and the epilogue of this one.
// Tiles are dealt so that the workgroups of an XCD, which share an L2, share
// rows: workgroups go to the XCDs in turn, and each XCD takes a contiguous range
// of an order that runs over q within bands of kBand p tiles.  (The gradient of
// 4096 tokens takes 10.40 ms with bands of 2, 9.99 of 4, 10.09 of 8.)
constexpr int kBand = 4;
constexpr int kXcds = 8;

template <int WP_, int WQ_, int FP_, int FQ_, bool PTR_, bool QTR_, int EPI_, int FIT_>
struct Tile {
  static constexpr int WP = WP_, WQ = WQ_;      // waves along p and q
  static constexpr int FP = FP_, FQ = FQ_;      // 16 x 16 outputs of a wave along p and q
  static constexpr bool PTR = PTR_, QTR = QTR_; // orders of the operands
  static constexpr int EPI = EPI_;
  static constexpr int FIT = FIT_;              // workgroups that the chip holds
  static constexpr int NT = WP * WQ * 64, BP = WP * FP * 16, BQ = WQ * FQ * 16;
  using OpP = Operand<BP, NT, PTR>;
  using OpQ = Operand<BQ, NT, QTR>;
  static constexpr int kBytes = OpP::kBytes + OpQ::kBytes;   // of a stage
};

// Workgroup `block` of `blocks` of a tiled product.  sm0, sm1: the stages.
template <typename S>
__device__ __forceinline__ void tile_work(const TileArgs& a, int block, int blocks, char* sm0,
                                          char* sm1) {
  constexpr int WP = S::WP, FP = S::FP, FQ = S::FQ, EPI = S::EPI, FIT = S::FIT;
  constexpr bool PTR = S::PTR, QTR = S::QTR;
  constexpr int BP = S::BP, BQ = S::BQ;
  using OpP = typename S::OpP;
  using OpQ = typename S::OpQ;
  __shared__ float2 folded[EPI == kStats ? WP : 1][EPI == kStats ? BQ : 1];
  __shared__ float row_lse[EPI == kGrad ? BQ : 1], row_coef[EPI == kGrad ? BQ : 1];
  __shared__ int row_label[EPI == kGrad ? BQ : 1];

  const int tid = threadIdx.x, l = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wp = w % WP, wq = w / WP;
  const int n_live = a.hdr->n_live;
  const float out_factor = EPI == kOut ? a.hdr->scale * a.out_scale : 0.f;
  const int64_t nq = a.live_q ? n_live : a.nq;
  const int64_t nk = a.live_k ? n_live : a.nk;
  const int tiles_p = (int)((a.np + BP - 1) / BP), tiles_q = (int)((nq + BQ - 1) / BQ);
  const int tiles = tiles_p * tiles_q;
  const int splits = EPI == kSlab ? splits_of(FIT, tiles, a.max_splits) : 1;
  const int steps_all = (int)((nk + kStep - 1) / kStep);
  const int left = (int)(nk - (int64_t)(steps_all - 1) * kStep);

  // this workgroup's tiles: id, id + stride, ... below end
  int id, end;
  const int stride = blocks / kXcds;
  {
    const int all = tiles * splits, x = block % kXcds;
    const int per = all / kXcds, rem = all % kXcds;
    const int start = x * per + (x < rem ? x : rem);
    id = start + block / kXcds;
    end = start + per + (x < rem);
  }
  if (id >= end) return;

  // A tile's steps, made an even number by a step of zeros.  The step that the
  // summed axis ends inside and the one of zeros come first, so that the loop
  // has whole ones only.  (An operand with rows of zeros makes it whole by
  // itself.)
  OpP op;
  OpQ oq;
  int tp, tq, split, n, shift, first, first_left, second_left;
  auto aim = [&](int id) {
    const int t = (int)pinned(tid);
    split = EPI == kSlab ? id / tiles : 0;
    const int in_split = id - split * tiles;
    const int band = in_split / (kBand * tiles_q), in = in_split % (kBand * tiles_q);
    const int width = tiles_p - band * kBand < kBand ? tiles_p - band * kBand : kBand;
    tp = band * kBand + in % width;
    tq = in / width;
    const int64_t p0 = (int64_t)tp * BP, q0 = (int64_t)tq * BQ;
    op.init(PTR ? a.P + p0 : a.P + p0 * a.ldp, a.ldp, a.np - p0, t);
    // the rows of q are padded to whole tiles
    oq.init(QTR ? a.Q + q0 : a.Q + q0 * a.ldq, a.ldq, BQ, t);
    const int s0 = (int)((int64_t)steps_all * split / splits);
    const int s1 = (int)((int64_t)steps_all * (split + 1) / splits);
    const int ragged = EPI != kOut && s1 == steps_all && left < kStep;
    const int zeros = s1 == s0 ? 2 : (s1 - s0) & 1;
    n = s1 - s0 + zeros;
    shift = s0 - ragged - (zeros & 1);   // step i of the tile is i + shift, for i > 1
    first = ragged ? steps_all - 1 : s0;
    first_left = zeros == 2 ? 0 : ragged ? left : kStep;
    second_left = zeros ? 0 : kStep;     // and its second is s0 + 1 - ragged
    n = __builtin_amdgcn_readfirstlane(n);
    shift = __builtin_amdgcn_readfirstlane(shift);
    first = __builtin_amdgcn_readfirstlane(first);
    first_left = __builtin_amdgcn_readfirstlane(first_left);
    second_left = __builtin_amdgcn_readfirstlane(second_left);
  };
  // Part i of n of the loads of a tile's first and second step.
  auto load_first = [&](char* to, int i, int n) {
    const int t = (int)pinned(tid);
    op.load_tail(to, first, w, i * OpP::kLoads / n, (i + 1) * OpP::kLoads / n, t, first_left, a.zero);
    oq.load_tail(to + OpP::kBytes, first, w, i * OpQ::kLoads / n, (i + 1) * OpQ::kLoads / n, t,
                 first_left ? kStep : 0, a.zero);
  };
  auto load_second = [&](char* to, int i, int n) {
    const int t = (int)pinned(tid);
    op.load_tail(to, 1 + shift, w, i * OpP::kLoads / n, (i + 1) * OpP::kLoads / n, t, second_left,
                 a.zero);
    oq.load_tail(to + OpP::kBytes, 1 + shift, w, i * OpQ::kLoads / n, (i + 1) * OpQ::kLoads / n, t,
                 second_left, a.zero);
  };

  f32x4 acc[FP][FQ];
  bf16x8 fp[FP], qa[FQ], qb[FQ];
  // Half a step: the products of one set of fragments and, as each of P's is
  // done with, the read of the next; Q's, which all products use, have two
  // places.
  const uint32_t lane_p = OpP::lane_place(wp * FP * 16, l), lane_q = OpQ::lane_place(wq * FQ * 16, l);
  auto half = [&](const bf16x8(&q)[FQ], bf16x8(&qn)[FQ], const char* from, int ks, bool meet,
                  auto fill) {
    const uint32_t lp = pinned(lane_p), lq = pinned(lane_q);
#pragma unroll
    for (int i = 0; i < FP; ++i) {
#pragma unroll
      for (int j = 0; j < FQ; ++j)
        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fp[i], q[j], acc[i][j], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
      if (meet && i == 0) wait_and_meet();
      fp[i] = OpP::frag(from, lp, wp * FP, i, ks, l);
#pragma unroll
      for (int j = i * FQ / FP; j < (i + 1) * FQ / FP; ++j)
        qn[j] = OpQ::frag(from + OpP::kBytes, lq, wq * FQ, j, ks, l);
      fill(i);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  // A step in stage `in`, whose successor is in stage `next`; fill(i), part i of
  // FP, loads what comes after that to `in`.  At the meeting every wave has read
  // `in`, and `next` is filled.
  auto step = [&](char* in, char* next, auto fill) {
    half(qa, qb, in, 1, false, [](int) {});
    half(qb, qa, next, 0, true, fill);
  };

  aim(id);
  load_first(sm0, 0, 1);
  load_second(sm1, 0, 1);
  wait_and_meet();
#pragma unroll
  for (int j = 0; j < FQ; ++j) qa[j] = OpQ::frag(sm0 + OpP::kBytes, lane_q, wq * FQ, j, 0, l);
#pragma unroll
  for (int i = 0; i < FP; ++i) fp[i] = OpP::frag(sm0, lane_p, wp * FP, i, 0, l);

#pragma unroll 1
  for (;;) {
#pragma unroll
    for (int i = 0; i < FP; ++i)
#pragma unroll
      for (int j = 0; j < FQ; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
    for (int s = 2; s < n; s += 2) {
      auto fill = [&](char* to, int s, int i) {
        op.load(to, s, w, i * OpP::kLoads / FP, (i + 1) * OpP::kLoads / FP);
        oq.load(to + OpP::kBytes, s, w, i * OpQ::kLoads / FP, (i + 1) * OpQ::kLoads / FP);
      };
      step(sm0, sm1, [&](int i) { fill(sm0, s + shift, i); });
      step(sm1, sm0, [&](int i) { fill(sm1, s + 1 + shift, i); });
    }
    const int my_split = split;
    const int64_t p0 = (int64_t)tp * BP, q0 = (int64_t)tq * BQ;
    const int my_tp = tp;
    // after the last tile: its own first steps again, which nothing reads
    const bool more = id + stride < end;
    aim(more ? id + stride : id);
    // What the epilogue wants of its rows is asked for before the last steps and
    // passed through LDS between them, behind whose meeting it is there.
    float lse_in = 0.f, coef_in = 0.f;
    int label_in = -1;
    if (EPI == kGrad && tid < BQ && q0 + tid < n_live) {
      lse_in = a.row_lse[q0 + tid];
      coef_in = a.row_coef[q0 + tid];
      if (a.row_label) label_in = a.row_label[q0 + tid];
    }
    step(sm0, sm1, [&](int i) { load_first(sm0, i, FP); });
    if (EPI == kGrad && tid < BQ) {
      row_lse[tid] = lse_in;
      row_coef[tid] = coef_in;
      row_label[tid] = label_in;
    }
    step(sm1, sm0, [&](int i) { load_second(sm1, i, FP); });

    // lane l holds, of the 16 x 16 outputs (i, j), q = l % 16 and
    // p = 4 (l / 16) .. + 3
    const int l = (int)pinned(tid) & 63;
    const int64_t pw = p0 + wp * FP * 16 + (l >> 4) * 4;
    const int64_t qw = q0 + wq * FQ * 16 + (l & 15);

    if constexpr (EPI == kStats) {
      if (p0 + BP > a.np) {
#pragma unroll
        for (int i = 0; i < FP; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (pw + i * 16 + e >= a.np)
#pragma unroll
              for (int j = 0; j < FQ; ++j) acc[i][j][e] = -INFINITY;
      }
#pragma unroll
      for (int j = 0; j < FQ; ++j) {
        float m = -INFINITY;
#pragma unroll
        for (int i = 0; i < FP; ++i)
          m = fmaxf(fmaxf(fmaxf(m, acc[i][j][0]), fmaxf(acc[i][j][1], acc[i][j][2])), acc[i][j][3]);
        m = fmaxf(m, __shfl_xor(m, 16));
        m = fmaxf(m, __shfl_xor(m, 32));
        // A row of which nothing is there, or only -inf, sums to 0.  The difference
        // is taken before it is scaled: the scaled maximum's rounding is more than an
        // exponent holds from 2^32 on.
        const float ref = fabsf(m) == INFINITY ? 0.f : m;
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < FP; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) sum += exp2_((acc[i][j][e] - ref) * a.s2);
        sum += __shfl_xor(sum, 16);
        sum += __shfl_xor(sum, 32);
        if (m == INFINITY && sum > 0.f) sum = 1.f;   // (a NaN stays)
        if (l < 16) folded[wp][(wq * FQ + j) * 16 + l] = make_float2(m, sum);
      }
      __syncthreads();
      // (The next write here is a tile's steps and their meetings away.)
      if (tid < BQ) {
        float2 p = folded[0][tid];
#pragma unroll
        for (int i = 1; i < WP; ++i) join(p.x, p.y, folded[i][tid].x, folded[i][tid].y, a.s2);
        a.parts[(int64_t)my_tp * a.parts_ld + q0 + tid] = p;
      }
    } else if constexpr (EPI == kGrad) {
      // G is rounded to bf16, what the matrix cores multiply with bf16 hidden states
      // and weights: its entries' error, up to 2^-8, takes the gradients' in the
      // 2-norm from the results' own rounding, 1.7e-3, to 1.8e-3 to 2.5e-3.  With a
      // second row for what that leaves (copies) the two products that follow would
      // be twice as long; up to kTwiceTokens tokens have it.
      const bool inside = p0 + BP <= a.np && q0 + BQ <= n_live;
      uint16_t* g = a.G + qw * a.ldg + p0 + wp * FP * 16 + (l >> 4) * 8;
#pragma unroll
      for (int j = 0; j < FQ; ++j, g += 16 * a.ldg) {
        const int r = (wq * FQ + j) * 16 + (l & 15);
        const float lse = row_lse[r], coef = row_coef[r];
        // the label's place among this lane's, where one of the wave's rows has
        // it among the wave's
        const int64_t y = row_label[r] - a.p_first - pw;
        const bool here = y >= 0 && y < FP * 16 && (y & 12) == 0;
        const bool labels = __any(here);
        const float spot = here ? a.row_spot[qw + j * 16] : 0.f;
#pragma unroll
        for (int i = 0; i < FP; i += 2) {
          u32x2 d[2];
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            float v[4];
            // (lse is taken off before the scaling to base 2: of a large lse the
            // scaled value's rounding would be a factor of the softmax)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              v[e] = coef * exp2_(__builtin_fmaf(acc[i + h][j][e], a.inv_tau, -lse) * kLog2e);
            if (!inside)
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if (qw + j * 16 >= n_live || pw + (i + h) * 16 + e >= a.np) v[e] = 0.f;
            if (labels)
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if (here && y == (i + h) * 16 + e) v[e] = spot;
            if constexpr (BQ == 64)   // rows of up to kTwiceTokens tokens are one such tile's
              if (a.copies == 2 && (l & 1))
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = rest_of(v[e]);
            d[h] = u32x2{pack2(v[0], v[1]), pack2(v[2], v[3])};
          }
          *reinterpret_cast<u32x4*>(g + i * 16) = eight(d[0], d[1]);
        }
      }
    } else if constexpr (EPI == kSlab) {
#pragma unroll
      for (int j = 0; j < FQ; ++j) {
        const int64_t q = qw + j * 16;
        if (q >= nq) continue;
        float* o = a.slab + (my_split * nq + q) * a.ld_slab;
#pragma unroll
        for (int i = 0; i < FP; ++i) {
          const int64_t p = pw + i * 16;
          if (p < a.ld_slab) {
            f32x4* d = reinterpret_cast<f32x4*>(o + p);
            *d = a.add ? *d + acc[i][j] : acc[i][j];
          }
        }
      }
    } else {
      const bool inside = a.vec_out && p0 + BP <= a.np && q0 + BQ <= nq;
      uint16_t* o = a.out + qw * a.ld_out + p0 + wp * FP * 16 + (l >> 4) * 8;
      auto result = [&](int i, int j) {
        const f32x4 x = acc[i][j] * out_factor, y = acc[i + 1][j] * out_factor;
        return eight(u32x2{pack2(x[0], x[1]), pack2(x[2], x[3])},
                     u32x2{pack2(y[0], y[1]), pack2(y[2], y[3])});
      };
      if (inside) {
#pragma unroll
        for (int j = 0; j < FQ; ++j, o += 16 * a.ld_out)
#pragma unroll
          for (int i = 0; i < FP; i += 2) *reinterpret_cast<u32x4*>(o + i * 16) = result(i, j);
      } else {
#pragma unroll
        for (int j = 0; j < FQ; ++j, o += 16 * a.ld_out)
#pragma unroll
          for (int i = 0; i < FP; i += 2) {
            const u32x4 x = result(i, j);
            const int64_t p = p0 + (wp * FP + i) * 16 + (l >> 4) * 8;
            if (qw + j * 16 >= nq || p >= a.np) continue;
            if (a.vec_out) {
              *reinterpret_cast<u32x4*>(o + i * 16) = x;
            } else {
#pragma unroll
              for (int e = 0; e < 8; ++e)
                if (p + e < a.np) o[i * 16 + e] = (uint16_t)(x[e >> 1] >> (e & 1) * 16);
            }
          }
      }
    }
    if (!more) break;
    id += stride;
  }
  // no load to LDS outlives the workgroup that owns it
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
}

template <typename S>
__global__ __launch_bounds__(S::NT) __attribute__((amdgpu_waves_per_eu(2))) void k_tile(
    const TileArgs a) {
  // Two arrays, and two steps to a turn of the loop, so that the compiler sees
  // that reads of one stage need not wait for the loads to the other.
  __shared__ __attribute__((aligned(128))) char sm0[S::kBytes];
  __shared__ __attribute__((aligned(128))) char sm1[S::kBytes];
  tile_work<S>(a, blockIdx.x, gridDim.x, sm0, sm1);
}

// Two products at a time, the first by the first `blocks` workgroups: the
// gradient's last two read the same G, and where they are short neither fills the
// chip.
template <typename S, typename R>
__global__ __launch_bounds__(S::NT) __attribute__((amdgpu_waves_per_eu(2))) void k_tiles(
    const TileArgs a, const int blocks, const TileArgs b) {
  static_assert(S::NT == R::NT, "one size of workgroup");
  constexpr int kBytes = S::kBytes > R::kBytes ? S::kBytes : R::kBytes;
  __shared__ __attribute__((aligned(128))) char sm0[kBytes];
  __shared__ __attribute__((aligned(128))) char sm1[kBytes];
  if ((int)blockIdx.x < blocks)
    tile_work<S>(a, blockIdx.x, blocks, sm0, sm1);
  else
    tile_work<R>(b, blockIdx.x - blocks, gridDim.x - blocks, sm0, sm1);
}

template <bool PTR, bool QTR, int EPI>
struct Tiles {
  using T256 = Tile<2, 4, 8, 4, PTR, QTR, EPI, 256>;
  using T128 = Tile<2, 2, 4, 4, PTR, QTR, EPI, 512>;
  using T64 = Tile<4, 1, 2, 4, PTR, QTR, EPI, 768>;
  using T16 = Tile<4, 1, 2, 1, PTR, QTR, EPI, 1024>;
};
using StatsTiles = Tiles<false, false, kStats>;
using GradTiles = Tiles<false, false, kGrad>;
using SlabTiles = Tiles<true, false, kSlab>;
using OutTiles = Tiles<true, true, kOut>;

// Workgroups of a product, 0 if it has no tiles.
int blocks_of(const TileArgs& a, int shape, bool splits) {
  const int64_t tp = (a.np + tile_p(shape) - 1) / tile_p(shape);
  const int64_t tq = (a.nq + tile_q(shape) - 1) / tile_q(shape);
  int64_t tiles = tp * tq;
  if (tiles <= 0) return 0;
  const int64_t fit = tile_fit(shape);
  if (splits || tiles > fit) tiles = fit;   // fewer live rows, more splits
  return (int)((tiles + kXcds - 1) / kXcds * kXcds);
}

template <typename S>
hipError_t launch_tile(const TileArgs& a, int shape, hipStream_t st) {
  const int n = blocks_of(a, shape, S::EPI == kSlab);
  return n > 0 ? launch(k_tile<S>, dim3((unsigned)n), S::NT, 0, st, a) : hipSuccess;
}

// ---- small kernels ------------------------------------------------------------

__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
  for (int d = 32; d; d >>= 1) x += __shfl_xor(x, d);
  return x;
}
__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
  for (int d = 32; d; d >>= 1) x = fmaxf(x, __shfl_xor(x, d));
  return x;
}

// None of these takes more than 27 us at 4096 tokens, but k_pack where many words
// are listed.

// The teacher's log probabilities of the listed words, one wave per token.  NaN,
// or an id past the vocabulary, makes the token's loss NaN, by its mass.  An entry
// with a negative id, or of a teacher logit of -inf, has probability 0; a token
// without any other takes no part.
__global__ __launch_bounds__(256) void k_teacher(const HeadArgs a) {
  const int64_t t = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int l = threadIdx.x & 63;
  if (t >= a.T) return;
  float x[2];
  bool bad = false;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int k = l + 64 * h;
    x[h] = -INFINITY;
    if (k < a.K) {
      const int32_t id = a.ids[t * a.K + k];
      if (id >= 0) x[h] = a.teacher[t * a.K + k];
      bad |= id >= a.V || x[h] != x[h];
    }
  }
  bad = __any(bad);
  const bool any = __any(!(x[0] == -INFINITY) || !(x[1] == -INFINITY));
  // log p = (x - ref) / tau - rest: in this order no digits of a small log p are
  // lost, and a logit at fp32's lowest value, finite as it is, does not overflow
  float ref = 0.f, rest = 0.f;
  if (a.teacher_lse) {
    rest = a.teacher_lse[t];
  } else if (any) {
    ref = wave_max(fmaxf(x[0], x[1]));
    rest = logf(wave_sum(expf((x[0] - ref) / a.tau) + expf((x[1] - ref) / a.tau)));
  }
  float mass = 0.f;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const float lp = x[h] == -INFINITY ? -INFINITY : (x[h] - ref) / a.tau - rest;
    mass += expf(lp);
    const int k = l + 64 * h;
    if (k < a.K) a.logp[t * a.K + k] = lp;
  }
  mass = wave_sum(mass);
  if (l == 0) {
    a.mass[t] = bad ? NAN : mass;
    a.flag[t] = any || bad;
  }
}

// Which tokens take part, in order, and (gradient) the largest finite |dloss|
// among them.  One workgroup.
__global__ __launch_bounds__(1024) void k_live(const HeadArgs a) {
  __shared__ int counts[2][16];
  __shared__ float tops[16];
  const int tid = threadIdx.x, l = tid & 63, w = tid >> 6;
  int base = 0, par = 0;
  float top = 0.f;
  for (int64_t t0 = 0; t0 < a.T; t0 += 1024, par ^= 1) {
    const int64_t t = t0 + tid;
    bool on = false;
    if (t < a.T) on = a.labels ? a.labels[t] >= 0 : a.flag[t] != 0;
    const uint64_t mask = __ballot(on);
    if (l == 0) counts[par][w] = __popcll(mask);
    __syncthreads();
    int before = base, all = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int c = counts[par][i];
      before += i < w ? c : 0;
      all += c;
    }
    base += all;
    const int q = before + __popcll(mask & (((uint64_t)1 << l) - 1));
    if (t < a.T) a.pos[t] = on ? q : -1;
    if (on) {
      a.rows[q] = (int32_t)t;
      if (a.dloss) {
        const float d = fabsf(a.dloss[t]);
        if (d < INFINITY) top = fmaxf(top, d);
      }
    }
  }
  top = wave_max(top);
  if (l == 0) tops[w] = top;
  __syncthreads();
  if (tid == 0) {
    for (int i = 0; i < 16; ++i) top = fmaxf(top, tops[i]);
    a.hdr->n_live = base;
    a.hdr->scale = top > 0.f ? top : 1.f;
    for (int i = 0; i < 4; ++i) a.hdr->zero[i] = 0;
  }
}

// Eight elements of a row of D from d on, those past its end 0.
__device__ __forceinline__ u32x4 row_chunk(const uint16_t* row, int64_t d, int64_t D) {
  if (d + 8 <= D) return *reinterpret_cast<const u32x4_at2*>(row + d);
  u32x4 o;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint32_t lo = d + 2 * e < D ? row[d + 2 * e] : 0;
    const uint32_t hi = d + 2 * e + 1 < D ? row[d + 2 * e + 1] : 0;
    o[e] = lo | hi << 16;
  }
  return o;
}
__device__ __forceinline__ bool is_live(const HeadArgs& a, int64_t t) {
  return a.labels ? a.labels[t] >= 0 : a.flag[t] != 0;
}

// Copies the live tokens' rows to consecutive ones, padded with zeros to Dp
// and, past the last, to whole tiles of rows.  Forward: also the products with
// the listed words' rows of the weight (a wave per listed word), and zeros as
// the results of the other tokens.  Gradient: also the coefficients of the
// rows, and zeros as the other tokens' gradient.  SCAN: of up to kScan tokens
// every workgroup finds by itself what k_live finds of more, which saves a launch
// (7 tokens x 1000 x 96: 18.5 us for 21.6).
//
// The listed words' rows are what takes time: 1000 tokens of 64 words are 0.52 GB
// of the weight, 91 us (5.8 TB/s; 130 with one word at a time), a tenth of the
// call.  The product's tiles hold these logits too, but looking for them there took
// as long and cost the loss of labels registers.
constexpr int kScan = 1024;
constexpr int kPackWords = 16;   // listed words of a workgroup

template <bool GRAD, bool SCAN>
__global__ __launch_bounds__(256) void k_pack(const HeadArgs a) {
  __shared__ int before_[4], all_[4];
  __shared__ float top_[4];
  const int tid = threadIdx.x, l = tid & 63, w = tid >> 6;
  const int64_t t = blockIdx.x;
  const u32x4 zero = {0, 0, 0, 0};
  int n;
  int64_t q;
  float scale;
  if (SCAN) {
    int before = 0, all = 0;
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < kScan / 256; ++i) {
      const int64_t u = i * 256 + tid;
      const bool on = u < a.T && is_live(a, u);
      all += __popcll(__ballot(on));
      before += __popcll(__ballot(on && u < t));
      if (GRAD && on) {
        const float d = fabsf(a.dloss[u]);
        if (d < INFINITY) top = fmaxf(top, d);
      }
    }
    if (GRAD) top = wave_max(top);
    if (l == 0) before_[w] = before, all_[w] = all, top_[w] = top;
    __syncthreads();
    n = all_[0] + all_[1] + all_[2] + all_[3];
    top = fmaxf(fmaxf(top_[0], top_[1]), fmaxf(top_[2], top_[3]));
    scale = top > 0.f ? top : 1.f;
    q = t < a.T && is_live(a, t) ? before_[0] + before_[1] + before_[2] + before_[3] : -1;
    if (tid == 0 && q >= 0) a.rows[q] = (int32_t)t;
    if (tid == 0 && t == a.T && blockIdx.y == 0) {
      a.hdr->n_live = n * a.copies;
      a.hdr->scale = scale;
      for (int i = 0; i < 4; ++i) a.hdr->zero[i] = 0;
    }
  } else {
    n = a.hdr->n_live;
    scale = a.hdr->scale;
    q = t < a.T ? a.pos[t] : -1;
  }
  // (a workgroup of each token's words; the first has the rest to do, too)
  const bool words_only = !GRAD && blockIdx.y > 0;
  if (t >= a.T) {
    const int64_t rows = (int64_t)n * (SCAN ? a.copies : 1), r = rows + (t - a.T);
    if (words_only || r >= (rows + kRowPad - 1) / kRowPad * kRowPad) return;
    for (int64_t d = tid * 8; d < a.Dp; d += 2048) *reinterpret_cast<u32x4*>(a.hc + r * a.Dp + d) = zero;
    return;
  }
  if (q < 0) {
    if (words_only) return;
    if (GRAD) {
      for (int64_t d = tid; d < a.D; d += 256) a.dhidden[t * a.D + d] = 0;
    } else {
      if (tid == 0) a.loss[t] = a.lse[t] = 0.f;
      if (tid < a.K) a.target[t * a.K + tid] = 0.f;
    }
    return;
  }
  const uint16_t* h = a.hidden + t * a.ldh;
  const int copies = GRAD && SCAN ? a.copies : 1;
  uint16_t* hc = a.hc + q * copies * a.Dp;
  if (!words_only)
    for (int64_t d = tid * 8; d < a.Dp; d += 2048) {
      const u32x4 x = row_chunk(h, d, a.D);
      *reinterpret_cast<u32x4*>(hc + d) = x;
      if (copies == 2) *reinterpret_cast<u32x4*>(hc + a.Dp + d) = x;
    }
  if (GRAD) {
    if (tid < copies) {
      q = q * copies + tid;
      const float ratio = a.dloss[t] / scale, lse = a.lse_in[t];
      a.row_lse[q] = lse;
      if (a.labels) {
        const int64_t y = a.labels[t];
        a.row_coef[q] = y < a.V ? ratio : NAN;
        a.row_label[q] = y < a.V ? (int32_t)y : -1;
        a.row_spot[q] = ratio * (exp2_((a.target_in[t] - lse) * kLog2e) - 1.f);
      } else {
        a.row_coef[q] = ratio * a.mass[t];
      }
    }
    return;
  }
  // four listed words to a wave, so that enough loads are out
  const int k0 = blockIdx.y * kPackWords + w * 4;
  if (k0 < a.K) {
    int64_t id[4];
    const uint16_t* r[4];
    float s[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      id[i] = k0 + i < a.K ? (a.labels ? a.labels[t] : a.ids[t * a.K + k0 + i]) : -1;
      s[i] = 0.f;
      // the others' products, with row 0, are not used
      r[i] = a.weight + (id[i] >= 0 && id[i] < a.V ? id[i] : 0) * a.ldw;
    }
    const int n = a.K - k0 < 4 ? a.K - k0 : 4;
    for (int64_t d = l * 8; d < a.D; d += 512) {
      const u32x4 x = row_chunk(h, d, a.D);
      u32x4 y[4];
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (i < n) y[i] = row_chunk(r[i], d, a.D);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (i >= n) break;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          s[i] = __builtin_fmaf(__uint_as_float(x[e] << 16), __uint_as_float(y[i][e] << 16), s[i]);
          s[i] = __builtin_fmaf(__uint_as_float(x[e] & 0xFFFF0000u),
                                __uint_as_float(y[i][e] & 0xFFFF0000u), s[i]);
        }
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (i >= n) break;
      const float z = wave_sum(s[i]);
      if (l == 0) a.target[t * a.K + k0 + i] = id[i] >= a.V ? NAN : id[i] >= 0 ? z : 0.f;
    }
  }
}

// Weight rows whose length or place the 16-byte loads cannot take, copied to
// rows of Dp.
__global__ __launch_bounds__(256) void k_pack_weight(const HeadArgs a) {
  const int64_t n = a.V * a.Dp;
  for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8; i < n;
       i += (int64_t)gridDim.x * 2048) {
    const int64_t v = i / a.Dp, d = i % a.Dp;
    *reinterpret_cast<u32x4*>(a.wc + i) = row_chunk(a.weight + v * a.ldw, d, a.D);
  }
}

// lse and loss of C live rows: 1024 / C threads fold a row's parts, then a wave
// sums over its listed words.
template <int C>
__global__ __launch_bounds__(1024) void k_finish(const HeadArgs a) {
  __shared__ float ms[C][17], ss[C][17];
  const int tid = threadIdx.x, l = tid & 63, w = tid >> 6;
  const int n = a.hdr->n_live;
  const int64_t q0 = (int64_t)blockIdx.x * C;
  if (q0 >= n) return;
  const int c = tid % C;
  float m = -INFINITY, s = 0.f;
  const float s2 = kLog2e / a.tau;
  if (q0 + c < n) {
    const float2* p = a.parts + q0 + c;
    int i = tid / C;
    for (; i + 3 * (1024 / C) < a.n_parts; i += 4 * (1024 / C)) {
      float2 x[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) x[k] = p[(int64_t)(i + k * (1024 / C)) * a.rows_pad];
#pragma unroll
      for (int k = 0; k < 4; ++k) join(m, s, x[k].x, x[k].y, s2);
    }
    for (; i < a.n_parts; i += 1024 / C) {
      const float2 x = p[(int64_t)i * a.rows_pad];
      join(m, s, x.x, x.y, s2);
    }
  }
#pragma unroll
  for (int d = C; d < 64; d <<= 1) join(m, s, __shfl_xor(m, d), __shfl_xor(s, d), s2);
  if (l < C) ms[l][w] = m, ss[l][w] = s;
  __syncthreads();
  if (w >= C || q0 + w >= n) return;
  m = l < 16 ? ms[w][l] : -INFINITY;
  s = l < 16 ? ss[w][l] : 0.f;
#pragma unroll
  for (int d = 8; d; d >>= 1) join(m, s, __shfl_xor(m, d), __shfl_xor(s, d), s2);
  m = __shfl(m, 0);
  s = __shfl(s, 0);
  // A loss is a small difference of these: a row's last steps are in 64 bits.
  const double lse = (double)m / (double)a.tau + log((double)s);
  const int64_t t = a.rows[q0 + w];
  if (a.labels) {
    if (l == 0) {
      a.lse[t] = (float)lse;
      a.loss[t] = (float)(lse - (double)a.target[t]);
    }
    return;
  }
  double sum = 0.0;
  for (int k = l; k < a.K; k += 64) {
    const float lp = a.logp[t * a.K + k];
    if (lp != -INFINITY)
      sum += (double)expf(lp) * ((double)lp - (double)a.target[t * a.K + k] / (double)a.tau + lse);
  }
#pragma unroll
  for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
  if (l == 0) {
    a.lse[t] = (float)lse;
    // (an id past the vocabulary is one also where the teacher rules the word out)
    a.loss[t] = a.mass[t] != a.mass[t] ? NAN : (float)((double)a.tau * (double)a.tau * sum);
  }
}

// Distillation: G at the listed words [v0, v1), a wave per live row: the tile's epilogue left
// the softmax's share there in bf16; this replaces it by the whole difference,
// rounded once.  A word that a token lists more than once gets the sum of its
// probabilities.
__global__ __launch_bounds__(256) void k_fix(const HeadArgs a, uint16_t* G, int64_t ldg, int64_t v0,
                                             int64_t v1) {
  const int64_t q = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int l = threadIdx.x & 63;
  if (q >= a.hdr->n_live / a.copies) return;
  const int64_t t = a.rows[q];
  const float ratio = a.dloss[t] / a.hdr->scale;
  const float mass = a.mass[t], lse = a.lse_in[t];
  for (int k0 = 0; k0 < a.K; k0 += 64) {
    const int k = k0 + l;
    const int32_t id = k < a.K ? a.ids[t * a.K + k] : -1;
    float p = 0.f;
    for (int j0 = 0; j0 < a.K; j0 += 64) {
      const int j = j0 + l;
      const int32_t jd = j < a.K ? a.ids[t * a.K + j] : -1;
      const float jp = j < a.K ? expf(a.logp[t * a.K + j]) : 0.f;
      const int n = a.K - j0 < 64 ? a.K - j0 : 64;
      for (int i = 0; i < n; ++i) {
        const int32_t other = __shfl(jd, i);
        const float op = __shfl(jp, i);
        if (other == id) p += op;
      }
    }
    if (id >= v0 && id < v1) {
      const float z = a.target_in[t * a.K + k];
      const float g = ratio * (mass * exp2_((z / a.tau - lse) * kLog2e) - p);
      uint16_t* to = G + q * a.copies * ldg + (id - v0);
      *to = to_bf16(g);
      if (a.copies == 2) to[ldg] = to_bf16(rest_of(g));
    }
  }
}

// The gradient of the hidden state from the splits' fp32 sums, added in order
// (bound by memory: 4096 x 4096 of one split, 101 MB, in 26 us).
__global__ __launch_bounds__(256) void k_dh(const HeadArgs a, const float* slab, int64_t ld_slab,
                                            int bp, int bq, int fit, int max_splits,
                                            float out_scale) {
  // at most 2^20 rows of 2^15 elements: 2^25 chunks
  const int64_t n = a.hdr->n_live;
  const unsigned chunks = (unsigned)((a.D + 1023) / 1024), all = (unsigned)(n / a.copies) * chunks;
  const int splits =
      splits_of(fit, (int)((a.D + bp - 1) / bp) * (int)((n + bq - 1) / bq), max_splits);
  const float f = a.hdr->scale * out_scale;
  const bool vec = ((a.D & 3) | (reinterpret_cast<uintptr_t>(a.dhidden) & 7)) == 0;
  for (unsigned b = blockIdx.x; b < all; b += gridDim.x) {
    const int64_t q = b / chunks, d = (b % chunks * 256 + threadIdx.x) * 4;
    if (d >= a.D) continue;
    const float* p = slab + q * a.copies * ld_slab + d;
    f32x4 s = *reinterpret_cast<const f32x4*>(p);
#pragma unroll 4
    for (int i = 1; i < splits; ++i) s += *reinterpret_cast<const f32x4*>(p + i * (n * ld_slab));
    if (a.copies == 2) {
      f32x4 r = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
      for (int i = 0; i < splits; ++i)
        r += *reinterpret_cast<const f32x4*>(p + ld_slab + i * (n * ld_slab));
      s += r;
    }
    s *= f;
    uint16_t* o = a.dhidden + (int64_t)a.rows[q] * a.D + d;
    if (vec) {
      *reinterpret_cast<u32x2*>(o) = u32x2{pack2(s[0], s[1]), pack2(s[2], s[3])};
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (d + e < a.D) o[e] = to_bf16(s[e]);
    }
  }
}

}  // namespace

hipError_t launch_head_teacher(const HeadArgs& a, hipStream_t st) {
  return launch(k_teacher, dim3((unsigned)((a.T + 3) / 4)), 256, 0, st, a);
}
hipError_t launch_head_pack(const HeadArgs& a, bool grad, hipStream_t st) {
  const dim3 grid((unsigned)(a.T + kRowPad), grad ? 1 : (a.K + kPackWords - 1) / kPackWords);
  if (a.T <= kScan)
    return grad ? launch(k_pack<true, true>, grid, 256, 0, st, a)
                : launch(k_pack<false, true>, grid, 256, 0, st, a);
  if (const hipError_t e = launch(k_live, dim3(1), 1024, 0, st, a)) return e;
  return grad ? launch(k_pack<true, false>, grid, 256, 0, st, a)
              : launch(k_pack<false, false>, grid, 256, 0, st, a);
}
hipError_t launch_head_pack_weight(const HeadArgs& a, hipStream_t st) {
  const int64_t blocks = (a.V * a.Dp / 8 + 255) / 256;
  return launch(k_pack_weight, dim3((unsigned)(blocks < 8192 ? blocks : 8192)), 256, 0, st, a);
}
hipError_t launch_head_finish(const HeadArgs& a, hipStream_t st) {
  if (a.T == 1) return launch(k_finish<1>, dim3(1), 1024, 0, st, a);
  if (a.T <= 4) return launch(k_finish<4>, dim3(1), 1024, 0, st, a);
  return launch(k_finish<16>, dim3((unsigned)((a.T + 15) / 16)), 1024, 0, st, a);
}
hipError_t launch_head_fix(const HeadArgs& a, uint16_t* G, int64_t ldg, int64_t v0, int64_t v1,
                           hipStream_t st) {
  return launch(k_fix, dim3((unsigned)((a.T + 3) / 4)), 256, 0, st, a, G, ldg, v0, v1);
}
hipError_t launch_head_dh(const HeadArgs& a, const float* slab, int64_t ld_slab, int shape,
                          int max_splits, float out_scale, hipStream_t st) {
  const int64_t blocks = (a.D + 1023) / 1024 * a.T;
  return launch(k_dh, dim3((unsigned)(blocks < 65536 ? blocks : 65536)), 256, 0, st, a, slab, ld_slab,
                tile_p(shape), tile_q(shape), tile_fit(shape), max_splits, out_scale);
}
hipError_t launch_logits_stats(const TileArgs& a, int shape, hipStream_t st) {
  switch (shape) {
    case kTile256: return launch_tile<StatsTiles::T256>(a, shape, st);
    case kTile128: return launch_tile<StatsTiles::T128>(a, shape, st);
    case kTile64: return launch_tile<StatsTiles::T64>(a, shape, st);
    default: return launch_tile<StatsTiles::T16>(a, shape, st);
  }
}
hipError_t launch_logits_grad(const TileArgs& a, int shape, hipStream_t st) {
  switch (shape) {
    case kTile256: return launch_tile<GradTiles::T256>(a, shape, st);
    case kTile128: return launch_tile<GradTiles::T128>(a, shape, st);
    default: return launch_tile<GradTiles::T64>(a, shape, st);
  }
}
hipError_t launch_grads(const TileArgs& h, int h_shape, const TileArgs& w, int w_shape,
                        hipStream_t st) {
  // One launch for both where they are short: the gradients of 333 tokens x 5003 x
  // 321 in 46 us for 49, of 64 x 50257 x 1024 in 104 for 110, but of 64 x 128256 x
  // 4096 in 813 for 801.
  if (w_shape == kTile128 && h_shape != kTile256 && w.np * w.nq <= (int64_t)1 << 26) {
    const int nh = blocks_of(h, h_shape, true), nw = blocks_of(w, w_shape, false);
    const dim3 grid((unsigned)(nh + nw));
    return h_shape == kTile64
               ? launch(k_tiles<SlabTiles::T64, OutTiles::T128>, grid, 256, 0, st, h, nh, w)
               : launch(k_tiles<SlabTiles::T128, OutTiles::T128>, grid, 256, 0, st, h, nh, w);
  }
  const hipError_t e = w_shape == kTile256 ? launch_tile<OutTiles::T256>(w, w_shape, st)
                                           : launch_tile<OutTiles::T128>(w, w_shape, st);
  if (e != hipSuccess) return e;
  switch (h_shape) {
    case kTile256: return launch_tile<SlabTiles::T256>(h, h_shape, st);
    case kTile128: return launch_tile<SlabTiles::T128>(h, h_shape, st);
    default: return launch_tile<SlabTiles::T64>(h, h_shape, st);
  }
}

}  // namespace flr
