// draft.hpp -- what the entry points of drafted words (w4.hip, verify.hip)
// share with the rest of the library.  Not part of the public ABI.
#pragma once

#include "../../include/nmt.h"
#include "internal.hpp"

namespace nmt {

// The calling thread's error message (nmt_last_error), as api.hip sets it.
nmt_status entry_fail(nmt_status st, const char* msg);
nmt_status entry_hip_fail(hipError_t e, const char* what);
nmt_status entry_ok();
// NMT_EINVAL unless the model's device is the current one.
nmt_status entry_check_device(const nmt_model* m);

// A model's packed output weights and its device's compute units, and its
// device error flag (bit 0: an id out of range, bit 1: a row of logits that is
// no distribution).
struct OutputLayer {
  const Packed* W;
  int E, V, cus;
};
OutputLayer output_layer(const nmt_model* m);
int* error_flag(nmt_model* m);

}  // namespace nmt
