// flround_layers_api.cpp -- the C ABI of the embedding and the layer norm (declared in
// include/flround.h): arguments are checked, a call's workspace is laid out, and the
// kernels are enqueued.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "flr_layers.h"
#include "flround.h"

using namespace flr;

namespace {

constexpr int64_t kMaxRows = (int64_t)1 << 20;
constexpr int64_t kMaxWidth = (int64_t)1 << 15;
constexpr int64_t kMaxVocab = (int64_t)1 << 21;
constexpr int64_t kMaxStride = (int64_t)1 << 40;
constexpr int kCus = 256;

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
int64_t round_up(int64_t a, int64_t b) { return ceil_div(a, b) * b; }

int status_of(hipError_t e) {
  return e == hipSuccess ? FL_OK : e == hipErrorOutOfMemory ? FL_ERR_NOMEM : FL_ERR_HIP;
}

// A device pointer argument, aligned to its elements; may be null when the array is
// empty.
int elem_ptr(const void* p, int64_t n, size_t align) {
  if (n == 0) return FL_OK;
  if (!p) return FL_ERR_INVALID;
  return reinterpret_cast<uintptr_t>(p) & (align - 1) ? FL_ERR_ALIGN : FL_OK;
}

// One that may be left out.
int may_ptr(const void* p, size_t align) { return p ? elem_ptr(p, 1, align) : FL_OK; }

bool stride_ok(int64_t stride, int64_t width) {
  return stride == 0 || (stride >= width && stride <= kMaxStride);
}

size_t elem(int dtype) { return dtype == FL_BF16 ? 2 : 4; }

char* aligned(void* ws) {
  return reinterpret_cast<char*>((reinterpret_cast<uintptr_t>(ws) + 255) & ~(uintptr_t)255);
}

bool embed_ok(const fl_embed_shape* s) {
  return s && s->tokens >= 0 && s->tokens <= kMaxRows && s->vocab >= 1 && s->vocab <= kMaxVocab &&
         s->width >= 1 && s->width <= kMaxWidth && stride_ok(s->stride, s->width) &&
         (s->dtype == FL_BF16 || s->dtype == FL_F32);
}

bool norm_ok(const fl_norm_shape* s) {
  return s && s->rows >= 0 && s->rows <= kMaxRows && s->width >= 1 && s->width <= kMaxWidth &&
         stride_ok(s->x_stride, s->width) && stride_ok(s->dy_stride, s->width) &&
         (s->dtype == FL_BF16 || s->dtype == FL_F32);
}

struct EmbedPlan {
  int words, waves, list, tile;
  size_t start, order, slab, bytes;
};

// A workgroup of the sort for each CU, or more where its counts would not fit the LDS; a
// wave for every 64 tokens up to the 16 that a workgroup has.
EmbedPlan embed_plan(const fl_embed_shape& s) {
  EmbedPlan p{};
  p.bytes = 256;   // for a workspace that does not start on 256 bytes
  if (s.tokens <= kEmbedFew) return p;
  p.words = (int)std::min<int64_t>(ceil_div(s.vocab, kCus), kEmbedMaxWords);
  p.waves = (int)std::min<int64_t>(ceil_div(s.tokens, 64), kEmbedMaxWaves);
  // (the list's entries hold a token's place in the wave's share in 16 bits)
  p.list = (int)std::min<int64_t>(round_up(ceil_div(s.tokens, p.waves), 64), kEmbedMaxList);
  // Short tiles where tokens are few, as a wave takes its tokens one after the other; long
  // ones where many words' parts would have to be joined.  us for tiles of 4, 8, 16, 32 and
  // 64, added to 32000 x 2048 bf16 (513 and 1024 tokens: x 4096), no word frequent / 90 % of
  // the tokens one word:
  //     513   14.2 16.1 18.7 25.7  -   / 16.2 17.4 18.8 25.4  -
  //    1024   17.0 17.8 20.2 26.9  -   / 20.5 19.3 21.1 26.6  -
  //    1025    -   15.9 19.3 26.2 39.1 /  -   19.0 21.0 26.5 38.8
  //    2048    -   17.7 21.0 27.3 40.6 /  -   22.3 23.5 29.0 40.2
  //    4096    -   22.3 23.6 29.0 41.6 /  -   31.3 28.0 32.7 44.5
  //    8192    -   31.9 29.2 31.2 43.8 /  -   47.1 37.7 38.3 50.3
  //   16384    -   52.0 46.2 44.1 50.1 /  -   85.8 65.1 53.4 57.2
  //   32768    -   84.0 76.3 70.5 68.4 /  -  160.3 117.9 98.2 90.5
  p.tile = s.tokens <= 1024    ? 4
           : s.tokens <= 2048  ? 8
           : s.tokens <= 8192  ? 16
           : s.tokens <= 16384 ? 32
                               : 64;
  const int64_t tiles = ceil_div(s.tokens, p.tile);
  size_t at = 0;
  auto take = [&at](int64_t bytes) {
    const size_t here = at;
    at += (size_t)round_up(bytes, 256);
    return here;
  };
  p.start = take(4 * (s.vocab + 1));
  p.order = take(8 * s.tokens);
  p.slab = take(8 * tiles * round_up(s.width, 8));
  p.bytes += at;
  return p;
}

EmbedArgs embed_args(const fl_embed_shape& s, const int64_t* ids, const void* in, float scale,
                     void* out) {
  EmbedArgs a{};
  a.T = s.tokens, a.V = s.vocab, a.D = s.width;
  a.ld = s.stride ? s.stride : s.width;
  a.bf16 = s.dtype == FL_BF16;
  a.ids = ids, a.in = in, a.scale = scale, a.out = out;
  return a;
}

// Workgroups of the norm's gradient, each of which leaves a part of the weight's: one a CU
// (16384 x 4096 bf16: 74 us, 77 with two, whose parts are twice as many).
int64_t norm_parts(const fl_norm_shape& s) {
  return std::min<int64_t>(ceil_div(s.rows, norm_rows(s.width, s.dtype == FL_BF16)), kCus);
}

size_t norm_bytes(const fl_norm_shape& s) {
  const bool few = norm_few(s.rows, s.width, s.dtype == FL_BF16);
  return (few ? 0 : (size_t)(8 * norm_parts(s) * s.width)) + 256;
}

NormArgs norm_args(const fl_norm_shape& s, const void* x, const void* weight) {
  NormArgs a{};
  a.T = s.rows, a.D = s.width;
  a.ldx = s.x_stride ? s.x_stride : s.width;
  a.ldy = s.dy_stride ? s.dy_stride : s.width;
  a.bf16 = s.dtype == FL_BF16, a.rms = s.rms != 0;
  a.x = x, a.weight = weight;
  return a;
}

}  // namespace

extern "C" {

int fl_embed(const fl_embed_shape* shape, const int64_t* ids, const void* weight, float scale,
             void* out, void* stream) {
  int rc;
  if (!embed_ok(shape) || !std::isfinite(scale)) return FL_ERR_INVALID;
  const size_t es = elem(shape->dtype);
  if ((rc = elem_ptr(ids, shape->tokens, 8)) != FL_OK) return rc;
  if ((rc = elem_ptr(weight, 1, es)) != FL_OK) return rc;
  if ((rc = elem_ptr(out, shape->tokens, es)) != FL_OK) return rc;
  if (out == weight) return FL_ERR_INVALID;
  EmbedArgs a = embed_args(*shape, ids, weight, scale, out);
  const int64_t most = kMaxLaunchThreads / (64 * embed_pieces(a));   // tokens of a launch
  for (int64_t t = 0; t < shape->tokens; t += most) {
    a.T = std::min(most, shape->tokens - t);
    a.ids = ids + t;
    a.out = static_cast<char*>(out) + t * a.D * (int64_t)es;
    if ((rc = status_of(launch_embed(a, static_cast<hipStream_t>(stream)))) != FL_OK) return rc;
  }
  return FL_OK;
}

size_t fl_embed_workspace_bytes(const fl_embed_shape* shape) {
  return embed_ok(shape) ? embed_plan(*shape).bytes : 0;
}

int fl_embed_grad(const fl_embed_shape* shape, const int64_t* ids, const void* dout, float scale,
                  int add, void* dweight, void* workspace, size_t workspace_bytes, void* stream) {
  int rc;
  if (!embed_ok(shape) || !std::isfinite(scale)) return FL_ERR_INVALID;
  const size_t es = elem(shape->dtype);
  if ((rc = elem_ptr(ids, shape->tokens, 8)) != FL_OK) return rc;
  if ((rc = elem_ptr(dout, shape->tokens, es)) != FL_OK) return rc;
  if ((rc = elem_ptr(dweight, 1, es)) != FL_OK) return rc;
  if (dweight == dout || !workspace) return FL_ERR_INVALID;
  const EmbedPlan p = embed_plan(*shape);
  if (workspace_bytes < p.bytes) return FL_ERR_SCRATCH;
  EmbedArgs a = embed_args(*shape, ids, dout, scale, dweight);
  char* ws = aligned(workspace);
  a.add = add != 0;
  a.words = p.words, a.sort_waves = p.waves, a.list = p.list, a.tile = p.tile;
  a.start = reinterpret_cast<int32_t*>(ws + p.start);
  a.order = reinterpret_cast<int2*>(ws + p.order);
  a.slab = reinterpret_cast<float*>(ws + p.slab);
  a.ld_slab = round_up(shape->width, 8);
  const hipStream_t st = static_cast<hipStream_t>(stream);
  // one launch writes the zeros of few tokens' gradient, row by row; else those that the
  // sort's launch has no threads for are written before it
  const int64_t table = a.V * a.D, most = kMaxLaunchThreads * (int64_t)(16 / es);
  a.zeros = add || a.T <= kEmbedFew ? 0 : std::min(table, most);
  for (int64_t from = a.zeros; a.zeros && from < table; from += most) {
    char* at = static_cast<char*>(dweight) + from * (int64_t)es;
    rc = status_of(launch_embed_zeros(at, std::min(most, table - from), a.bf16, st));
    if (rc != FL_OK) return rc;
  }
  return status_of(launch_embed_grad(a, st));
}

int fl_layer_norm(const fl_norm_shape* shape, const void* x, const void* weight, const void* bias,
                  float eps, void* y, float* mean, float* rstd, void* stream) {
  int rc;
  if (!norm_ok(shape) || !std::isfinite(eps) || !(eps >= 0.f)) return FL_ERR_INVALID;
  const size_t es = elem(shape->dtype);
  for (const void* p : {x, (const void*)y})
    if ((rc = elem_ptr(p, shape->rows, es)) != FL_OK) return rc;
  for (const void* p : {weight, bias})
    if ((rc = may_ptr(p, es)) != FL_OK) return rc;
  if ((rc = may_ptr(mean, 4)) != FL_OK) return rc;
  if ((rc = elem_ptr(rstd, shape->rows, 4)) != FL_OK) return rc;
  if (shape->rows == 0) return FL_OK;
  if (y == x || y == weight || y == bias) return FL_ERR_INVALID;
  NormArgs a = norm_args(*shape, x, weight);
  a.bias = bias, a.eps = eps, a.y = y, a.mean = mean, a.rstd = rstd;
  return status_of(launch_norm(a, static_cast<hipStream_t>(stream)));
}

size_t fl_layer_norm_workspace_bytes(const fl_norm_shape* shape) {
  return norm_ok(shape) ? norm_bytes(*shape) : 0;
}

int fl_layer_norm_grad(const fl_norm_shape* shape, const void* x, const void* weight,
                       const float* mean, const float* rstd, const void* dy, void* dx,
                       void* dweight, void* dbias, void* workspace, size_t workspace_bytes,
                       void* stream) {
  int rc;
  if (!norm_ok(shape)) return FL_ERR_INVALID;
  const size_t es = elem(shape->dtype);
  for (const void* p : {x, dy, (const void*)dx})
    if ((rc = elem_ptr(p, shape->rows, es)) != FL_OK) return rc;
  for (const void* p : {weight, (const void*)dweight, (const void*)dbias})
    if ((rc = may_ptr(p, es)) != FL_OK) return rc;
  if ((rc = shape->rms ? may_ptr(mean, 4) : elem_ptr(mean, shape->rows, 4)) != FL_OK) return rc;
  if ((rc = elem_ptr(rstd, shape->rows, 4)) != FL_OK) return rc;
  for (const void* o : {(const void*)dx, (const void*)dweight, (const void*)dbias})
    if (o && (o == x || o == weight || o == dy)) return FL_ERR_INVALID;
  if ((dweight && (dweight == dbias || dweight == dx)) || (dbias && dbias == dx))
    return FL_ERR_INVALID;
  if (!workspace) return FL_ERR_INVALID;
  if (workspace_bytes < norm_bytes(*shape)) return FL_ERR_SCRATCH;
  NormArgs a = norm_args(*shape, x, weight);
  a.mean_in = mean, a.rstd_in = rstd, a.dy = dy, a.y = dx;
  a.dweight = dweight, a.dbias = dbias;
  a.parts = reinterpret_cast<float*>(aligned(workspace));
  a.n_parts = norm_parts(*shape);
  return status_of(launch_norm_grad(a, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
