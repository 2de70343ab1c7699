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

// Whether a workgroup is the last of its launch to come here.  Atomics on one counter take 12 ns each, one after the other, so a workgroup
// draws from one of 64 counters, a cache line each, and the last of each from a further one.  All are 0 again afterwards.
constexpr int kFan = 64, kTicketWords = (kFan + 1) * 32;
__device__ __forceinline__ bool draw_last(uint32_t* ticket, uint32_t of) {
  const bool last = __hip_atomic_fetch_add(ticket, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == of - 1;
  if (last) __hip_atomic_store(ticket, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return last;
}
// by one thread of every workgroup of the grid, once
__device__ __forceinline__ bool last_to_come(uint32_t* tickets) {
  const uint32_t mine = blockIdx.x % kFan, of = (gridDim.x - mine + kFan - 1) / kFan;
  return draw_last(tickets + 32 * (1 + mine), of) && draw_last(tickets, min(gridDim.x, (uint32_t)kFan));
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
