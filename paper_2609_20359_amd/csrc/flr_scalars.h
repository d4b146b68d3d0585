// flr_scalars.h -- AdamW's host side (defined in flround_api.cpp): the checks of its
// hyperparameters and a step's scalars.
#pragma once

#include "flr_internal.h"
#include "flround.h"

namespace flr {

bool hparams_ok(const fl_adamw_hparams* h);

// Computed in double, each rounded once to float.
AdamScalars adam_scalars(const fl_adamw_hparams& h, int64_t step);

}  // namespace flr
