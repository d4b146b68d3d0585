// flround_tensors_api.cpp -- the C ABI of AdamW over many tensors (declared in
// include/flround.h): arguments are checked and the tensors are spread over launches.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "flr_scalars.h"
#include "flr_tensors.h"
#include "flround.h"

using namespace flr;

namespace {

constexpr int64_t kMaxUnits = (int64_t)1 << 32;        // of all tensors: 2^41 elements
// Of one launch, whose threads, 64 to a unit, have to be fewer than 2^32: 2^32 elements,
// whose step takes ten milliseconds, so that another launch costs nothing.
constexpr int64_t kMaxLaunchUnits = (int64_t)1 << 23;

int64_t units_of(int64_t numel) { return (numel + kUnit - 1) / kUnit; }

// Units of all tensors, or -1 where a size is invalid.
int64_t all_units(int64_t count, const fl_tensor* t) {
  if (count < 0 || (count > 0 && !t)) return -1;
  int64_t units = 0;
  for (int64_t i = 0; i < count; ++i) {
    if (t[i].numel < 0 || t[i].numel > kMaxUnits * kUnit) return -1;
    units += units_of(t[i].numel);
    if (units > kMaxUnits) return -1;
  }
  return units;
}

int ptr_ok(const void* p, size_t align) {
  if (!p) return FL_ERR_INVALID;
  return reinterpret_cast<uintptr_t>(p) & (align - 1) ? FL_ERR_ALIGN : FL_OK;
}

StateDev state_at(void* state, int64_t units, int bits) {
  StateDev s{};
  s.bits = bits;
  char* at = static_cast<char*>(state);
  const int64_t n = units * kUnit, wide = bits / 8;
  s.m = at;
  s.v = at + n * wide;
  if (bits == 8) {
    s.m_exp = reinterpret_cast<uint8_t*>(at + 2 * n);
    s.v_exp = s.m_exp + n / kStateBlock;
  }
  return s;
}

// The state from a unit on.
StateDev state_from(StateDev s, int64_t unit) {
  const int64_t n = unit * kUnit, wide = s.bits / 8;
  s.m = static_cast<char*>(s.m) + n * wide;
  s.v = static_cast<char*>(s.v) + n * wide;
  if (s.bits == 8) s.m_exp += n / kStateBlock, s.v_exp += n / kStateBlock;
  return s;
}

int status_of(hipError_t e) {
  return e == hipSuccess ? FL_OK : e == hipErrorOutOfMemory ? FL_ERR_NOMEM : FL_ERR_HIP;
}

}  // namespace

extern "C" {

int64_t fl_tensors_state_numel(int64_t count, const fl_tensor* tensors) {
  const int64_t units = all_units(count, tensors);
  return units < 0 ? -1 : units * kUnit;
}

size_t fl_tensors_state_bytes(int64_t state_numel, int state_bits) {
  if (state_numel < 0 || state_numel % kUnit || state_numel > kMaxUnits * kUnit) return 0;
  if (state_bits == 32) return (size_t)state_numel * 8;
  return state_bits == 8 ? (size_t)(2 * state_numel + 2 * (state_numel / kStateBlock)) : 0;
}

int fl_adamw_tensors(int64_t count, const fl_tensor* tensors, const void* const* grads,
                     int grad_dtype, float grad_scale, const fl_adamw_hparams* h, int64_t step,
                     int state_bits, void* state, uint64_t seed, void* stream) {
  int rc;
  const int64_t units = all_units(count, tensors);
  if (units < 0 || (count > 0 && !grads) || !hparams_ok(h) || step < 1 ||
      !std::isfinite(grad_scale) || (grad_dtype != FL_BF16 && grad_dtype != FL_F32) ||
      (state_bits != 8 && state_bits != 32) || (state_bits == 32 && seed != 0))
    return FL_ERR_INVALID;
  const size_t grad_align = grad_dtype == FL_BF16 ? 2 : 4;
  for (int64_t i = 0; i < count; ++i) {
    const fl_tensor& t = tensors[i];
    if (t.numel == 0) continue;
    if ((rc = ptr_ok(t.master, 4)) != FL_OK) return rc;
    if (t.working && (rc = ptr_ok(t.working, 2)) != FL_OK) return rc;
    if (!grads[i]) continue;
    if ((rc = ptr_ok(grads[i], grad_align)) != FL_OK) return rc;
    if (grads[i] == t.master || grads[i] == t.working) return FL_ERR_INVALID;
  }
  if (units == 0) return FL_OK;
  if ((rc = ptr_ok(state, 16)) != FL_OK) return rc;
  TensorsArgs a{};
  a.s = adam_scalars(*h, step);
  a.grad_scale = grad_scale;
  a.grad_f32 = grad_dtype == FL_F32;
  a.drawn = seed != 0;
  // (odd multipliers: 2^64 over the golden ratio, and over the root of x^4 = x + 1, its
  // counterpart in three dimensions)
  const uint64_t key = seed * 0x9E3779B97F4A7C15ull + (uint64_t)step * 0xD1B54A32D192ED03ull;
  a.key_lo = (uint32_t)key, a.key_hi = (uint32_t)(key >> 32);
  a.state = state_at(state, units, state_bits);
  // tensors follow each other in a launch until it is full, one is left out, or its units
  // are many
  int n = 0;
  int64_t here = 0, before = 0;   // units of this launch, and before it
  auto flush = [&]() -> int {
    if (n == 0) return FL_OK;
    for (int k = n; k <= kMaxTensors; ++k) a.first[k] = k == n ? (int32_t)here : INT32_MAX;
    a.unit0 = before;
    const int status = status_of(launch_tensors(a, here, static_cast<hipStream_t>(stream)));
    before += here;
    n = 0, here = 0;
    for (uint32_t& w : a.decay) w = 0;
    return status;
  };
  for (int64_t i = 0; i < count; ++i) {
    const fl_tensor& t = tensors[i];
    const int64_t its = units_of(t.numel);
    if (its == 0) continue;
    if (!grads[i]) {
      if ((rc = flush()) != FL_OK) return rc;
      before += its;
      continue;
    }
    int64_t done = 0;   // a tensor of more units than a launch takes goes on in the next
    while (done < its) {
      const int64_t take = its - done < kMaxLaunchUnits - here ? its - done : kMaxLaunchUnits - here;
      a.first[n] = (int32_t)here;
      a.grad[n] = static_cast<const char*>(grads[i]) + done * kUnit * (int64_t)grad_align;
      a.master[n] = t.master + done * kUnit;
      a.working[n] = t.working ? t.working + done * kUnit : nullptr;
      a.numel[n] = t.numel - done * kUnit;
      if (t.decay) a.decay[n / 32] |= 1u << (n % 32);
      ++n;
      here += take;
      done += take;
      if ((n == kMaxTensors || here == kMaxLaunchUnits) && (rc = flush()) != FL_OK) return rc;
    }
  }
  return flush();
}

int fl_state_convert(int64_t state_numel, int from_bits, const void* from, void* to,
                     void* stream) {
  int rc;
  if (state_numel < 0 || state_numel % kUnit || state_numel > kMaxUnits * kUnit ||
      (from_bits != 8 && from_bits != 32))
    return FL_ERR_INVALID;
  if (state_numel == 0) return FL_OK;
  if ((rc = ptr_ok(from, 16)) != FL_OK || (rc = ptr_ok(to, 16)) != FL_OK) return rc;
  if (from == to) return FL_ERR_INVALID;
  const int64_t units = state_numel / kUnit;
  const StateDev src = state_at(const_cast<void*>(from), units, from_bits);
  const StateDev dst = state_at(to, units, 40 - from_bits);
  for (int64_t u = 0; u < units; u += kMaxLaunchUnits) {
    const int64_t n = units - u < kMaxLaunchUnits ? units - u : kMaxLaunchUnits;
    rc = status_of(launch_state_convert(state_from(src, u), state_from(dst, u), n,
                                        static_cast<hipStream_t>(stream)));
    if (rc != FL_OK) return rc;
  }
  return FL_OK;
}

}  // extern "C"
