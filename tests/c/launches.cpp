// Calls the library's entry points at sizes that need many threads, with the kernels'
// launches replaced by functions that note what each one covers: every launch is one that
// HIP takes, and together they cover the call's work once (test code; no GPU; run by
// tests/test_launches_cpu.py).
#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <vector>

#include "flr_layers.h"
#include "flr_scalars.h"
#include "flr_tensors.h"
#include "flround.h"

namespace {

constexpr int64_t kTooMany = (int64_t)1 << 32;   // threads that HIP does not take
char* const kIn = reinterpret_cast<char*>((uintptr_t)1 << 40);    // never dereferenced
char* const kWork = reinterpret_cast<char*>((uintptr_t)1 << 45);
char* const kOut = reinterpret_cast<char*>((uintptr_t)1 << 50);

struct Span {
  int64_t from, n;   // bytes of the output
};
std::vector<Span> spans;

void check(bool ok, const char* what) {
  if (ok) return;
  std::printf("wrong: %s\n", what);
  std::exit(1);
}

// The spans follow each other from 0 to n.
void check_cover(int64_t n, const char* what) {
  std::sort(spans.begin(), spans.end(), [](Span a, Span b) { return a.from < b.from; });
  int64_t at = 0;
  for (const Span& s : spans) {
    check(s.from == at && s.n > 0, what);
    at += s.n;
  }
  check(at == n, what);
  std::printf("%s: %zu launches\n", what, spans.size());
  spans.clear();
}

}  // namespace

namespace flr {

hipError_t launch_embed(const EmbedArgs& a, hipStream_t) {
  const int64_t es = a.bf16 ? 2 : 4, chunk = 16 / es;
  check((a.D + 64 * chunk - 1) / (64 * chunk) * a.T * 64 + 256 < kTooMany, "threads of the embedding");
  const int64_t from = static_cast<char*>(a.out) - kOut;
  check(reinterpret_cast<const char*>(a.ids) - kIn == from / (a.D * es) * 8, "ids of a launch");
  spans.push_back({from, a.T * a.D * es});
  return hipSuccess;
}

hipError_t launch_embed_zeros(void* out, int64_t n, bool bf16, hipStream_t) {
  check((n * (bf16 ? 2 : 4) + 15) / 16 + 256 < kTooMany, "threads of the zeros");
  spans.push_back({static_cast<char*>(out) - kOut, n * (bf16 ? 2 : 4)});
  return hipSuccess;
}

hipError_t launch_embed_grad(const EmbedArgs& a, hipStream_t) {
  const int64_t es = a.bf16 ? 2 : 4, table = a.V * a.D;
  if (a.T <= kEmbedFew) {   // zeros by rows: 512 threads for 16 KiB, or for a row, or for 1024
    const int64_t row = a.D * es, words = row < 16 ? 1024 : row < 16384 ? 16384 / row : 1;
    check((a.V / words + 1 + a.T * embed_pieces(a)) * 512 < kTooMany, "threads of few tokens");
    check(a.zeros == 0, "zeros of few tokens");
    spans.push_back({0, table * es});
    return hipSuccess;
  }
  const int64_t tiles = (a.T + a.tile - 1) / a.tile, threads = 64 * a.sort_waves;
  const int64_t sorts = (a.V + a.words - 1) / a.words;
  const int64_t fills = (a.zeros + threads * (16 / es) - 1) / (threads * (16 / es));
  check((sorts + fills) * threads < kTooMany, "threads of the sort");
  check(tiles * embed_pieces(a) * 512 < kTooMany, "threads of the sums and of the parts");
  check(static_cast<char*>(a.out) == kOut, "the gradient");
  if (a.zeros) spans.push_back({0, a.zeros * es});
  return hipSuccess;
}

hipError_t launch_norm(const NormArgs&, hipStream_t) { return hipSuccess; }
hipError_t launch_norm_grad(const NormArgs&, hipStream_t) { return hipSuccess; }
int norm_rows(int64_t, bool) { return 1; }

bool hparams_ok(const fl_adamw_hparams*) { return true; }
AdamScalars adam_scalars(const fl_adamw_hparams&, int64_t) { return {}; }

// The tensors' masters stand in kOut as their moments do in the state; gradients and
// working copies, of half the size, likewise in kIn and kWork.
hipError_t launch_tensors(const TensorsArgs& a, int64_t units, hipStream_t) {
  check(units * 64 + 256 < kTooMany, "threads of the step");
  int n = 0;
  while (n < kMaxTensors && a.first[n + 1] != INT32_MAX) ++n;
  check(n > 0 && a.first[n] == units, "units of a launch");
  for (int k = n + 1; k <= kMaxTensors; ++k) check(a.first[k] == INT32_MAX, "behind the last tensor");
  for (int k = 0; k < n; ++k) {
    const int64_t from = (a.unit0 + a.first[k]) * kUnit, its = a.first[k + 1] - a.first[k];
    check(reinterpret_cast<char*>(a.master[k]) == kOut + 4 * from, "master");
    check(static_cast<const char*>(a.grad[k]) == kIn + 2 * from, "gradient");
    check(reinterpret_cast<char*>(a.working[k]) == kWork + 2 * from, "working copy");
    check(a.numel[k] > (its - 1) * kUnit, "elements");
    check(((a.decay[k / 32] >> (k % 32)) & 1) == (from / kUnit) % 2, "decay");
    spans.push_back({from, its * kUnit});
  }
  return hipSuccess;
}

int64_t all;   // elements of a state that is converted

hipError_t launch_state_convert(const StateDev& from, const StateDev& to, int64_t units,
                                hipStream_t) {
  check(units * 64 + 256 < kTooMany, "threads of the conversion");
  const StateDev &narrow = from.bits == 8 ? from : to, &wide = from.bits == 8 ? to : from;
  check(narrow.bits == 8 && wide.bits == 32, "bits");
  const char *n = from.bits == 8 ? kIn : kOut, *w = from.bits == 8 ? kOut : kIn;
  const int64_t at = static_cast<char*>(narrow.m) - n;
  check(static_cast<char*>(narrow.v) == n + all + at, "codes of v");
  check(reinterpret_cast<char*>(narrow.m_exp) == n + 2 * all + at / 64, "exponents of m");
  check(reinterpret_cast<char*>(narrow.v_exp) == n + 2 * all + all / 64 + at / 64, "exponents of v");
  check(static_cast<char*>(wide.m) == w + 4 * at, "m");
  check(static_cast<char*>(wide.v) == w + 4 * all + 4 * at, "v");
  spans.push_back({at, units * kUnit});
  return hipSuccess;
}

}  // namespace flr

namespace {

// One step of tensors of these sizes.
void tensors(const std::vector<int64_t>& sizes) {
  std::vector<fl_tensor> t;
  std::vector<const void*> grads;
  int64_t at = 0;
  for (int64_t n : sizes) {
    t.push_back({n, reinterpret_cast<float*>(kOut + 4 * at),
                 reinterpret_cast<uint16_t*>(kWork + 2 * at), (int)(at / 512 % 2)});
    grads.push_back(kIn + 2 * at);
    at += (n + 511) / 512 * 512;
  }
  const fl_adamw_hparams h{};
  check(fl_adamw_tensors((int64_t)t.size(), t.data(), grads.data(), FL_BF16, 1.f, &h, 1, 8, kOut, 1,
                         nullptr) == FL_OK, "status");
  check_cover(at, "step");
}

}  // namespace

int main() {
  const int64_t T = 1 << 20, D = 1 << 15;
  for (int dtype : {FL_BF16, FL_F32})
    for (int64_t tokens : {(int64_t)1, (int64_t)333, T / 8, T / 2 - 1, T - 1, T})
      for (int64_t width : {(int64_t)1, (int64_t)4096, D - 511, D}) {
        const fl_embed_shape s{tokens, 1000, width, 0, dtype};
        check(fl_embed(&s, reinterpret_cast<int64_t*>(kIn), kIn, 1.f, kOut, nullptr) == FL_OK, "status");
        check_cover(tokens * width * (dtype == FL_BF16 ? 2 : 4), "embedding");
      }
  for (int dtype : {FL_BF16, FL_F32})
    for (int64_t tokens : {(int64_t)0, (int64_t)512, (int64_t)513, T})
      for (int64_t vocab : {(int64_t)1, (int64_t)32000, T, 2 * T - 1, 2 * T})
        for (int64_t width : {(int64_t)1, (int64_t)7, (int64_t)4096, D - 511, D})
          for (int add : {0, 1}) {
            const fl_embed_shape s{tokens, vocab, width, 0, dtype};
            check(fl_embed_grad(&s, reinterpret_cast<int64_t*>(kIn), kIn, 1.f, add, kOut, kIn,
                                fl_embed_workspace_bytes(&s), nullptr) == FL_OK, "status");
            if (add) check(tokens <= 512 || spans.empty(), "no zeros where the sum is added");
            if (add) spans.clear();
            else check_cover(vocab * width * (dtype == FL_BF16 ? 2 : 4), "zeros");
          }
  const int64_t most = (int64_t)1 << 32;   // elements of a launch
  tensors({1});
  tensors({most});
  tensors({most + 1});
  tensors({most - 512, 512, 513, most, 7});
  tensors({700, 3 * most + 5, 512, 1});
  tensors({((int64_t)1 << 41) - 512, 1});
  for (int64_t n : {95, 96, 97, 300}) tensors(std::vector<int64_t>(n, 777));
  for (int bits : {8, 32})
    for (int64_t n : {(int64_t)512, most, most + 512, 3 * most - 1024, (int64_t)1 << 41}) {
      flr::all = n;
      check(fl_state_convert(n, bits, kIn, kOut, nullptr) == FL_OK, "status");
      check_cover(n, "conversion");
    }
  return 0;
}
