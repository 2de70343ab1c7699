// The clipped policy loss and its gradient: the launches of train_logp.h's kernels, and the end of their sums.
#include "train_logp.h"

namespace rotconv {
namespace {

// out[k] = sum of the workgroups' k-th sums, each thread's in order and then a fixed tree
__global__ __launch_bounds__(1024) void k_policy_end(const double* __restrict__ part, int count, float* __restrict__ out) {
  __shared__ double red[16][4];
  double acc[4] = {};
  for (int i = threadIdx.x; i < count; i += 1024)
#pragma unroll
    for (int k = 0; k < 4; ++k) acc[k] += part[4 * (size_t)i + k];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
#pragma unroll
    for (int o = 32; o > 0; o /= 2) acc[k] += __shfl_xor(acc[k], o);
    if (threadIdx.x % 64 == 0) red[threadIdx.x / 64][k] = acc[k];
  }
  __syncthreads();
  if (threadIdx.x < 4) {
    double v = 0;
    for (int w = 0; w < 16; ++w) v += red[w][threadIdx.x];
    out[threadIdx.x] = (float)v;
  }
}

}  // namespace

void launch_policy(const LossArgs& g, bool bf16, bool rows, float* out, hipStream_t st) {
  unsigned blocks;
  if (bf16) launch_loss<uint16_t, kPolicy>(g, rows, &blocks, st);
  else launch_loss<float, kPolicy>(g, rows, &blocks, st);
  k_policy_end<<<1, 1024, 0, st>>>(g.part, (int)blocks, out);
}

}  // namespace rotconv
