// What the optimizers' kernels share of the control block (see include/unettrain.h).
#pragma once

#include <hip/hip_runtime.h>

#include "unettrain.h"

namespace rotconv {
namespace {

// The factor of a step's gradients: a clip factor that a step has used, and that nobody has written over, counts no more.
__device__ __forceinline__ float factor(const train_control& c) {
  return c.clip == 2 && __float_as_uint(c.coef) == __float_as_uint(c.spent) ? 1.f : c.coef;
}

// The end of a step that has updated its tensors (skip: that has left them, for a norm that was not finite); t: its number.  One
// thread's, when no other of the step will read the block again.
__device__ __forceinline__ void end_step(train_control* ctl, int skip, int t) {
  if (skip) {
    ctl->skipped += 1, ctl->nonfinite = 0;
    ctl->coef = 1.f, ctl->clip = 0;                    // of a norm that was not finite
    return;
  }
  ctl->step = t;
  if (ctl->clip == 1) ctl->clip = 2, ctl->spent = ctl->coef;
}

}  // namespace
}  // namespace rotconv
