// flround_head_api.cpp -- the C ABI of the output head's operators (declared in
// include/flround.h): arguments are checked, a call's workspace is laid out,
// the vocabulary is cut into pieces, and the kernels are enqueued.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "flr_head.h"
#include "flround.h"

using namespace flr;

namespace {

constexpr int64_t kMaxTokens = (int64_t)1 << 20;
constexpr int64_t kMaxWidth = (int64_t)1 << 15;
constexpr int64_t kMaxHiddenStride = (int64_t)1 << 40;   // all rows within 62 bits of bytes
constexpr int64_t kMaxWeightStride = (int64_t)1 << 22;   // 256 rows of it within 32
constexpr int64_t kMaxVocab = (int64_t)1 << 21;
constexpr int64_t kMaxTopVocab = (int64_t)1 << 20;
constexpr int64_t kMaxTiles = (int64_t)1 << 22;
constexpr int kCus = 256;

// G of a piece of the vocabulary: at most this many bytes, or kMinPiece words.
constexpr int64_t kPieceBytes = (int64_t)256 << 20;
constexpr int64_t kMinPiece = 8192;

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
int64_t round_up(int64_t a, int64_t b) { return ceil_div(a, b) * b; }

int64_t tiles_of(int shape, int64_t np, int64_t nq) {
  return ceil_div(np, tile_p(shape)) * ceil_div(nq, tile_q(shape));
}

// Tiles of 256 x 256 once they fill the chip; smaller ones where rows or words
// are few.  (The loss of 128 tokens x 128256 x 4096 takes 207 us in tiles of 128
// x 128 and 266 in large ones, that of 256 tokens 338 and 272; their gradient,
// with the hidden state's alike, 883 and 977 us.)
int shape_for(int64_t np, int64_t nq, bool few_rows) {
  if (few_rows && nq <= 16) return kTile16;
  if (few_rows && nq <= 64) return kTile64;
  if (few_rows && nq <= 128) return kTile128;
  return tiles_of(kTile256, np, nq) >= kCus ? kTile256 : kTile128;
}

struct Plan {
  int64_t T, V, D, Dp, rows, rows_pad;   // rows: compacted ones, of all tokens
  int copies, K;
  bool grad, distill, pack_w;
  int logits_shape, dh_shape, dw_shape;
  int n_parts, max_splits;
  int64_t slab_rows;
  int64_t piece, n_pieces;
  // byte offsets into the workspace
  size_t hdr, live, pos, logp, mass, flag, hc, wc, parts, row_lse, row_coef, row_label, row_spot, G, slab, bytes;
};

// The tiles' loads take 16 bytes; rows of another length are copied first, from any
// element's boundary.
bool copies_weight(const fl_head_shape& s) {
  return (((s.weight_stride ? s.weight_stride : s.width) | s.width) & 7) != 0;
}

Plan plan_for(const fl_head_shape& s, int K, bool grad) {
  Plan p{};
  const bool pack_w = copies_weight(s);
  p.T = s.tokens, p.V = s.vocab, p.D = s.width;
  p.K = K > 0 ? K : 1;
  p.grad = grad, p.distill = K > 0, p.pack_w = pack_w;
  p.Dp = round_up(p.D, kStep);
  p.copies = grad && p.T <= kTwiceTokens ? 2 : 1;
  p.rows = p.T * p.copies;
  p.rows_pad = round_up(p.rows, kRowPad);
  p.piece = p.V;
  p.n_pieces = 1;
  if (grad && p.T > 0) {
    const int64_t words = std::max(kMinPiece, kPieceBytes / (2 * p.rows_pad));
    p.n_pieces = ceil_div(p.V, words);
    p.piece = round_up(ceil_div(p.V, p.n_pieces), 256);
    p.n_pieces = ceil_div(p.V, p.piece);
  }
  p.logits_shape = shape_for(p.piece, p.rows, true);
  if (grad && p.logits_shape == kTile16) p.logits_shape = kTile64;   // G is read 64 rows at a time
  p.n_parts = (int)ceil_div(p.V, tile_p(p.logits_shape));
  // Large tiles where there are enough of them, with eight steps each.
  p.dh_shape = p.T <= 64 ? kTile64 : p.T <= 128 ? kTile128
               : tiles_of(kTile256, p.D, p.T) * (p.piece / (8 * kStep)) >= kCus ? kTile256 : kTile128;
  // The weight's gradient of few tokens is bound by its stores, which two small
  // tiles to a CU overlap: 64 tokens x 128256 x 4096 in 765 us, 814 with large
  // ones; 128 tokens in 981 and 965, 512 in 1884 and 1751.
  p.dw_shape = p.T <= 64 ? kTile128 : shape_for(p.D, p.piece, false);
  // The sum over a piece is split where the outputs are too few tiles to fill
  // the chip, four steps at least to a split.  How many tiles there are depends
  // on the live rows, and the rows of all splits are at most the chip's share.
  p.max_splits = (int)std::max<int64_t>(1, std::min<int64_t>(ceil_div(p.piece, kStep) / 4, 64));
  p.slab_rows = std::max(p.rows, tile_fit(p.dh_shape) * tile_q(p.dh_shape) /
                                  ceil_div(p.D, tile_p(p.dh_shape)));
  p.slab_rows = std::min(p.slab_rows, p.rows * p.max_splits);

  size_t at = 0;
  auto take = [&](int64_t bytes) {
    const size_t o = at;
    at += (size_t)round_up(std::max<int64_t>(bytes, 1), 256);
    return o;
  };
  p.hdr = take(sizeof(HeadHeader));
  p.live = take(4 * p.T);
  p.pos = take(4 * p.T);
  if (p.distill) {
    p.logp = take(4 * p.T * p.K);
    p.mass = take(4 * p.T);
    p.flag = take(p.T);
  }
  p.hc = take(2 * p.rows_pad * p.Dp);
  if (pack_w) p.wc = take(2 * p.V * p.Dp);
  if (grad) {
    p.row_lse = take(4 * p.rows_pad);
    p.row_coef = take(4 * p.rows_pad);
    p.row_label = take(4 * p.rows_pad);
    p.row_spot = take(4 * p.rows_pad);
    p.G = take(2 * p.rows_pad * round_up(p.piece, 256));
    p.slab = take(4 * p.slab_rows * p.Dp);
  } else {
    p.parts = take(8 * (int64_t)p.n_parts * p.rows_pad);
  }
  p.bytes = at + 256;   // for a workspace that does not start on 256 bytes
  return p;
}

bool shape_ok(const fl_head_shape* s) {
  if (!s || s->tokens < 0 || s->tokens > kMaxTokens || s->vocab < 1 || s->vocab > kMaxVocab ||
      s->width < 1 || s->width > kMaxWidth)
    return false;
  const int64_t ldh = s->hidden_stride, ldw = s->weight_stride;
  if (ldh != 0 && (ldh < s->width || ldh > kMaxHiddenStride)) return false;
  if (ldw != 0 && (ldw < s->width || ldw > kMaxWeightStride)) return false;
  return ceil_div(s->tokens, 128) * ceil_div(s->vocab, 128) <= kMaxTiles;
}

// A device pointer argument, aligned to its elements; may be null when the
// array is empty.
int elem_ptr(const void* p, int64_t n, size_t align) {
  if (n == 0) return FL_OK;
  if (!p) return FL_ERR_INVALID;
  return reinterpret_cast<uintptr_t>(p) & (align - 1) ? FL_ERR_ALIGN : FL_OK;
}

int status_of(hipError_t e) {
  return e == hipSuccess ? FL_OK : e == hipErrorOutOfMemory ? FL_ERR_NOMEM : FL_ERR_HIP;
}

// log2(e) / tau, by which the kernels scale, has to be finite in 32 bits.
bool tau_ok(float tau) {
  return std::isfinite(tau) && tau > 0.f && std::isfinite((float)(1.4426950408889634 / (double)tau));
}

struct Targets {
  const int64_t* labels;
  const int32_t* ids;
  const float* teacher;
  const float* teacher_lse;
  int K;      // 0: labels
  float tau;
};

int check_targets(const fl_head_shape& s, const Targets& t) {
  int rc;
  if (t.K == 0) return elem_ptr(t.labels, s.tokens, 8);
  if (t.K < 1 || t.K > kMaxTargets || !tau_ok(t.tau)) return FL_ERR_INVALID;
  if ((rc = elem_ptr(t.ids, s.tokens, 4)) != FL_OK) return rc;
  if ((rc = elem_ptr(t.teacher, s.tokens, 4)) != FL_OK) return rc;
  return t.teacher_lse ? elem_ptr(t.teacher_lse, s.tokens, 4) : FL_OK;
}

struct Call {
  Plan p;
  HeadArgs a{};
  char* ws = nullptr;
  hipStream_t st = nullptr;

  template <typename T>
  T* at(size_t off) const {
    return reinterpret_cast<T*>(ws + off);
  }

  int begin(const fl_head_shape& s, const uint16_t* hidden, const uint16_t* weight,
            const Targets& t, bool grad, void* workspace, size_t bytes, void* stream) {
    const int64_t ldh = s.hidden_stride ? s.hidden_stride : s.width;
    const int64_t ldw = s.weight_stride ? s.weight_stride : s.width;
    p = plan_for(s, t.K, grad);
    if (!workspace) return FL_ERR_INVALID;
    if (bytes < p.bytes) return FL_ERR_SCRATCH;
    ws = reinterpret_cast<char*>((reinterpret_cast<uintptr_t>(workspace) + 255) & ~(uintptr_t)255);
    st = static_cast<hipStream_t>(stream);
    a.T = p.T, a.V = p.V, a.D = p.D, a.Dp = p.Dp;
    a.ldh = ldh, a.ldw = ldw;
    a.hidden = hidden, a.weight = weight;
    a.copies = p.copies, a.K = p.K, a.tau = t.K ? t.tau : 1.f;
    a.labels = t.K ? nullptr : t.labels;
    a.ids = t.ids, a.teacher = t.teacher, a.teacher_lse = t.teacher_lse;
    a.hdr = at<HeadHeader>(p.hdr);
    a.rows = at<int32_t>(p.live), a.pos = at<int32_t>(p.pos);
    if (p.distill) {
      a.logp = at<float>(p.logp), a.mass = at<float>(p.mass), a.flag = at<uint8_t>(p.flag);
    }
    a.hc = at<uint16_t>(p.hc);
    a.wc = p.pack_w ? at<uint16_t>(p.wc) : nullptr;
    if (grad) {
      a.row_lse = at<float>(p.row_lse), a.row_coef = at<float>(p.row_coef);
      a.row_label = at<int32_t>(p.row_label), a.row_spot = at<float>(p.row_spot);
    }
    a.n_parts = p.n_parts;
    a.rows_pad = p.rows_pad;
    return FL_OK;
  }

  // The live tokens, their rows, and the weight's where they are copied.
  int prepare() {
    if (p.distill && p.T > 0)
      if (const hipError_t e = launch_head_teacher(a, st)) return status_of(e);
    if (const hipError_t e = launch_head_pack(a, p.grad, st)) return status_of(e);
    if (p.pack_w)
      if (const hipError_t e = launch_head_pack_weight(a, st)) return status_of(e);
    return FL_OK;
  }

  const uint16_t* weight_rows(int64_t v0) const {
    return a.wc ? a.wc + v0 * p.Dp : a.weight + v0 * a.ldw;
  }
  int64_t weight_ld() const { return a.wc ? p.Dp : a.ldw; }

  TileArgs logits(int64_t v0, int64_t v1) const {
    TileArgs g{};
    g.P = weight_rows(v0), g.ldp = weight_ld();
    g.Q = a.hc, g.ldq = p.Dp;
    g.np = v1 - v0, g.nq = p.rows, g.nk = a.wc ? p.Dp : p.D;
    g.hdr = a.hdr, g.live_q = 1, g.zero = reinterpret_cast<const uint16_t*>(a.hdr->zero);
    g.s2 = (float)(1.4426950408889634 / (double)a.tau);
    return g;
  }
};

int forward(const fl_head_shape* s, const uint16_t* hidden, const uint16_t* weight,
            const Targets& t, float* loss, float* lse, float* target, void* workspace,
            size_t bytes, void* stream) {
  int rc;
  if (!shape_ok(s)) return FL_ERR_INVALID;
  if ((rc = check_targets(*s, t)) != FL_OK) return rc;
  if ((rc = elem_ptr(hidden, s->tokens, 2)) != FL_OK) return rc;
  if ((rc = elem_ptr(weight, 1, copies_weight(*s) ? 2 : 16)) != FL_OK) return rc;
  for (const void* o : {(const void*)loss, (const void*)lse, (const void*)target})
    if ((rc = elem_ptr(o, s->tokens, 4)) != FL_OK) return rc;
  Call c;
  if ((rc = c.begin(*s, hidden, weight, t, false, workspace, bytes, stream)) != FL_OK) return rc;
  if (s->tokens == 0) return FL_OK;
  c.a.loss = loss, c.a.lse = lse, c.a.target = target;
  c.a.parts = c.at<float2>(c.p.parts);
  if ((rc = c.prepare()) != FL_OK) return rc;
  TileArgs g = c.logits(0, c.p.V);
  g.parts = c.at<float2>(c.p.parts);
  g.parts_ld = c.p.rows_pad;
  if ((rc = status_of(launch_logits_stats(g, c.p.logits_shape, c.st))) != FL_OK) return rc;
  return status_of(launch_head_finish(c.a, c.st));
}

int backward(const fl_head_shape* s, const uint16_t* hidden, const uint16_t* weight,
             const Targets& t, const float* lse, const float* target, const float* dloss,
             uint16_t* dhidden, uint16_t* dweight, void* workspace, size_t bytes, void* stream) {
  int rc;
  if (!shape_ok(s)) return FL_ERR_INVALID;
  if ((rc = check_targets(*s, t)) != FL_OK) return rc;
  if ((rc = elem_ptr(hidden, s->tokens, 2)) != FL_OK) return rc;
  if ((rc = elem_ptr(weight, 1, copies_weight(*s) ? 2 : 16)) != FL_OK) return rc;
  for (const void* i : {(const void*)lse, (const void*)target, (const void*)dloss})
    if ((rc = elem_ptr(i, s->tokens, 4)) != FL_OK) return rc;
  if ((rc = elem_ptr(dhidden, s->tokens, 2)) != FL_OK) return rc;
  if ((rc = elem_ptr(dweight, 1, 2)) != FL_OK) return rc;
  if (dweight == weight || dweight == hidden || (dhidden && (dhidden == hidden || dhidden == weight ||
                                                             dhidden == dweight)))
    return FL_ERR_INVALID;
  Call c;
  if ((rc = c.begin(*s, hidden, weight, t, true, workspace, bytes, stream)) != FL_OK) return rc;
  const Plan& p = c.p;
  c.a.lse_in = lse, c.a.target_in = target, c.a.dloss = dloss;
  c.a.dhidden = dhidden;
  if ((rc = c.prepare()) != FL_OK) return rc;
  uint16_t* G = c.at<uint16_t>(p.G);
  float* slab = c.at<float>(p.slab);
  const int64_t ldg = round_up(p.piece, 256);
  const float out_scale = c.a.tau;   // d(tau^2 loss') / d(z / tau) / tau
  for (int64_t v0 = 0; v0 < p.V; v0 += p.piece) {
    const int64_t v1 = std::min(v0 + p.piece, p.V);
    if (p.T > 0) {
      TileArgs g = c.logits(v0, v1);
      g.inv_tau = (float)(1.0 / (double)c.a.tau);
      g.row_lse = c.a.row_lse, g.row_coef = c.a.row_coef;
      g.row_label = p.distill ? nullptr : c.a.row_label, g.row_spot = c.a.row_spot;
      g.p_first = v0;
      g.G = G, g.ldg = ldg, g.copies = p.copies;
      if ((rc = status_of(launch_logits_grad(g, p.logits_shape, c.st))) != FL_OK) return rc;
      if (p.distill && (rc = status_of(launch_head_fix(c.a, G, ldg, v0, v1, c.st))) != FL_OK)
        return rc;
    }
    TileArgs w{};
    w.P = c.a.hc, w.ldp = p.Dp;
    w.Q = G, w.ldq = ldg;
    w.np = p.D, w.nq = v1 - v0, w.live_k = 1;
    w.hdr = c.a.hdr, w.zero = reinterpret_cast<const uint16_t*>(c.a.hdr->zero);
    w.out = dweight + v0 * p.D, w.ld_out = p.D;
    w.vec_out = (p.D & 7) == 0 && (reinterpret_cast<uintptr_t>(dweight) & 15) == 0;
    w.out_scale = out_scale;
    TileArgs h{};
    h.hdr = c.a.hdr;
    if (p.T > 0) {
      h.P = c.weight_rows(v0), h.ldp = c.weight_ld();
      h.Q = G, h.ldq = ldg;
      h.np = p.D, h.nq = p.rows, h.live_q = 1, h.nk = v1 - v0;
      h.hdr = c.a.hdr, h.zero = reinterpret_cast<const uint16_t*>(c.a.hdr->zero);
      h.slab = slab, h.ld_slab = p.Dp;
      h.add = v0 > 0, h.max_splits = p.max_splits;
    }
    if ((rc = status_of(launch_grads(h, p.dh_shape, w, p.dw_shape, c.st))) != FL_OK) return rc;
  }
  if (p.T == 0) return FL_OK;
  return status_of(launch_head_dh(c.a, slab, p.Dp, p.dh_shape, p.max_splits, out_scale, c.st));
}

// Segments of a row of top logits: the whole row, or as much of it as keeps
// few rows from leaving the chip idle.
struct TopPlan {
  int chunks, segs;
  size_t parts, bytes;
};
TopPlan top_plan(int64_t rows, int64_t vocab, int k, bool bf16) {
  const int64_t e = bf16 ? 8 : 4;
  TopPlan p{kTopMaxChunks, 1, 0, 0};
  // a row may start inside a chunk
  auto segs = [&](int chunks) { return ceil_div(vocab + e - 1, kTopThreads * chunks * e); };
  while (p.chunks > 1 &&
         (rows * segs(p.chunks) < 2 * kCus || segs(p.chunks / 2) == 1) &&
         segs(p.chunks / 2) * k <= kTopMaxEntries)
    p.chunks /= 2;
  p.segs = (int)segs(p.chunks);
  const size_t lists = (size_t)round_up(8 * rows * p.segs * k, 256);
  p.parts = lists;
  p.bytes = p.segs == 1 ? 0 : lists + (size_t)(8 * rows * p.segs) + 256;
  return p;
}

bool top_ok(int64_t rows, int64_t vocab, int dtype, int k) {
  return rows >= 0 && rows <= kMaxTokens && vocab >= 1 && vocab <= kMaxTopVocab && k >= 1 &&
         k <= kMaxTargets && k <= vocab && (dtype == FL_BF16 || dtype == FL_F32);
}

}  // namespace

extern "C" {

size_t fl_head_workspace_bytes(const fl_head_shape* shape, int k, int grad) {
  if (!shape_ok(shape) || k < 0 || k > kMaxTargets) return 0;
  return plan_for(*shape, k, grad != 0).bytes;
}

int fl_head_loss(const fl_head_shape* shape, const uint16_t* hidden, const uint16_t* weight,
                 const int64_t* labels, float* loss, float* lse, float* target, void* workspace,
                 size_t workspace_bytes, void* stream) {
  return forward(shape, hidden, weight, {labels, nullptr, nullptr, nullptr, 0, 1.f}, loss, lse,
                 target, workspace, workspace_bytes, stream);
}

int fl_head_loss_grad(const fl_head_shape* shape, const uint16_t* hidden, const uint16_t* weight,
                      const int64_t* labels, const float* lse, const float* target,
                      const float* dloss, uint16_t* dhidden, uint16_t* dweight, void* workspace,
                      size_t workspace_bytes, void* stream) {
  return backward(shape, hidden, weight, {labels, nullptr, nullptr, nullptr, 0, 1.f}, lse, target,
                  dloss, dhidden, dweight, workspace, workspace_bytes, stream);
}

int fl_head_distill(const fl_head_shape* shape, const uint16_t* hidden, const uint16_t* weight,
                    int k, const int32_t* ids, const float* teacher, const float* teacher_lse,
                    float tau, float* loss, float* lse, float* target, void* workspace,
                    size_t workspace_bytes, void* stream) {
  if (k < 1) return FL_ERR_INVALID;
  return forward(shape, hidden, weight, {nullptr, ids, teacher, teacher_lse, k, tau}, loss, lse,
                 target, workspace, workspace_bytes, stream);
}

int fl_head_distill_grad(const fl_head_shape* shape, const uint16_t* hidden,
                         const uint16_t* weight, int k, const int32_t* ids, const float* teacher,
                         const float* teacher_lse, float tau, const float* lse,
                         const float* target, const float* dloss, uint16_t* dhidden,
                         uint16_t* dweight, void* workspace, size_t workspace_bytes,
                         void* stream) {
  if (k < 1) return FL_ERR_INVALID;
  return backward(shape, hidden, weight, {nullptr, ids, teacher, teacher_lse, k, tau}, lse, target,
                  dloss, dhidden, dweight, workspace, workspace_bytes, stream);
}

size_t fl_top_workspace_bytes(int64_t rows, int64_t vocab, int dtype, int k) {
  return top_ok(rows, vocab, dtype, k) ? top_plan(rows, vocab, k, dtype == FL_BF16).bytes : 0;
}

int fl_top_logits(int64_t rows, int64_t vocab, int64_t stride, int dtype, const void* logits, int k,
                  float tau, float* values, int32_t* ids, float* lse, void* workspace,
                  size_t workspace_bytes, void* stream) {
  int rc;
  if (!top_ok(rows, vocab, dtype, k) || !tau_ok(tau)) return FL_ERR_INVALID;
  if (stride != 0 && stride < vocab) return FL_ERR_INVALID;
  if (rows == 0) return FL_OK;
  if ((rc = elem_ptr(logits, rows, dtype == FL_BF16 ? 2 : 4)) != FL_OK) return rc;
  if ((rc = elem_ptr(values, rows, 4)) != FL_OK) return rc;
  if ((rc = elem_ptr(ids, rows, 4)) != FL_OK) return rc;
  if (lse && (rc = elem_ptr(lse, rows, 4)) != FL_OK) return rc;
  const TopPlan p = top_plan(rows, vocab, k, dtype == FL_BF16);
  if (p.bytes && !workspace) return FL_ERR_INVALID;
  if (workspace_bytes < p.bytes) return FL_ERR_SCRATCH;
  char* ws = reinterpret_cast<char*>((reinterpret_cast<uintptr_t>(workspace) + 255) & ~(uintptr_t)255);
  TopArgs a{};
  a.logits = logits;
  a.rows = rows, a.vocab = vocab, a.stride = stride ? stride : vocab;
  a.bf16 = dtype == FL_BF16;
  a.k = k;
  a.tau = tau;
  a.s2 = (float)(1.4426950408889634 / (double)tau);
  a.values = values, a.ids = ids, a.lse = lse;
  a.chunks = p.chunks, a.segs = p.segs;
  if (p.segs > 1) {
    a.lists = reinterpret_cast<uint64_t*>(ws);
    a.parts = reinterpret_cast<float2*>(ws + p.parts);
  }
  return status_of(launch_top(a, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
