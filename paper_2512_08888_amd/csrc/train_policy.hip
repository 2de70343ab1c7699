// The clipped policy loss and its gradient: the launches of train_logp.h's kernels, and the end of their sums.
#include "train_logp.h"

namespace rotconv {
namespace {

// out[k] = sum of the workgroups' k-th sums: a thread's, 16 at a time on their way, then a fixed tree over lanes and waves.  What it takes
// is the way of its loads and its launch: the fewest waves that have them all on their way at once (32 workgroups' sums by one wave 1.5 us,
// by sixteen 3.3; 711 workgroups' by four 2.1, by sixteen 3.4; 4096 workgroups' by sixteen 5.4).
constexpr int kEndThreads = 1024;
__global__ __launch_bounds__(kEndThreads) void k_policy_end(const double* __restrict__ part, uint32_t values, float* __restrict__ out) {
  constexpr int kWaves = kEndThreads / 64, kAhead = 16;
  __shared__ double red[kWaves * 4];
  double v = 0;
  for (uint32_t i = threadIdx.x; i < values; i += kAhead * blockDim.x) {
    double a[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) a[k] = part[min(i + k * blockDim.x, values - 1)];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) v += i + k * blockDim.x < values ? a[k] : 0.0;
  }
#pragma unroll
  for (int o = 32; o >= 4; o /= 2) v += __shfl_xor(v, o);
  if (blockDim.x > 64) {
    if (threadIdx.x % 64 < 4) red[threadIdx.x / 64 * 4 + threadIdx.x % 64] = v;
    __syncthreads();
    if (threadIdx.x >= 64) return;
    v = threadIdx.x / 4 < blockDim.x / 64 ? red[threadIdx.x] : 0.0;
#pragma unroll
    for (int o = 32; o >= 4; o /= 2) v += __shfl_xor(v, o);
  }
  if (threadIdx.x < 4) out[threadIdx.x] = (float)v;
}

}  // namespace

void launch_policy(const LossArgs& g, bool bf16, bool rows, float* out, hipStream_t st) {
  unsigned blocks;
  if (bf16) launch_loss<uint16_t, kPolicy>(g, rows, &blocks, st);
  else launch_loss<float, kPolicy>(g, rows, &blocks, st);
  k_policy_end<<<1, blocks <= 256 ? 64 : blocks <= 1024 ? 256 : kEndThreads, 0, st>>>(g.part, 4 * blocks, out);
}

}  // namespace rotconv
