// flr_tensors.h -- types shared by the C-ABI layer of AdamW over many tensors
// (flround_tensors_api.cpp) and its gfx950 kernels (flround_tensors.hip).  Not part of
// the public ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "flr_internal.h"

namespace flr {

constexpr int kStateBlock = 64;   // elements that share an exponent in states of 8 bits
constexpr int kMaxTensors = 96;   // tensors of one launch: as many as its arguments hold

// The moments: n elements of each, a tensor's from a multiple of kUnit on.
struct StateDev {
  int bits;          // 32: m and v are floats; 8: codes, with an exponent to a block
  void* m;
  void* v;
  uint8_t* m_exp;
  uint8_t* v_exp;
};

// One launch's tensors.  Unit u of the launch, of kUnit elements, is of the tensor k with
// first[k] <= u < first[k + 1].
struct TensorsArgs {
  AdamScalars s;
  float grad_scale;
  bool grad_f32, drawn;           // drawn: roundings of the states by random bits
  uint32_t key_lo, key_hi;
  StateDev state;
  int64_t unit0;                  // of the launch's first unit among all units
  uint32_t decay[kMaxTensors / 32];
  int32_t first[kMaxTensors + 1]; // INT32_MAX behind the last
  const void* grad[kMaxTensors];
  float* master[kMaxTensors];
  uint16_t* working[kMaxTensors]; // may be null
  int64_t numel[kMaxTensors];
};
static_assert(sizeof(TensorsArgs) <= 4096, "a launch's arguments");

hipError_t launch_tensors(const TensorsArgs& a, int64_t units, hipStream_t st);
// 8 to 32 bits, or (to nearest) the other way.
hipError_t launch_state_convert(const StateDev& from, const StateDev& to, int64_t units,
                                hipStream_t st);

}  // namespace flr
