// Group normalisation with an activation, forward and backward (see include/unettrain.h).
//
// Three launches each way: sums of every channel of every image in pieces, the groups' statistics from them, and the map.
// A piece's forward sums are its mean and its squared deviations from that mean, joined pairwise-exactly (never as
// sum x^2 - mean^2, which loses the variance of a map far from zero).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "glue_elt.h"
#include "rotconv.h"
#include "unettrain.h"

namespace rotconv {
namespace {

constexpr int kThreads = 256;

int finish() { return hipGetLastError() == hipSuccess ? ROTCONV_OK : ROTCONV_ERR_LAUNCH; }

struct Gn {
  int N, C, G, cg;
  size_t P;
  float eps;
  int act;
  int pieces;            // of a channel's pixels
  size_t step;           // pixels of a piece, the last one's are fewer
};

__device__ __forceinline__ float normalised(float x, float mean, float rstd) {
#pragma clang fp contract(off)
  return (x - mean) * rstd;
}
__device__ __forceinline__ float affine(float xh, float gamma, float beta) {
#pragma clang fp contract(off)
  return xh * gamma + beta;
}
__device__ __forceinline__ float activate(float z, int act) {
  if (act == TRAIN_ACT_RELU) return z <= 0.f ? 0.f : z;
  if (act == TRAIN_ACT_SILU) return z * (1.f / (1.f + expf(-z)));
  return z;
}
__device__ __forceinline__ float through(float dy, float z, int act) {      // dy * act'(z)
  if (act == TRAIN_ACT_RELU) return z > 0.f ? dy : 0.f;
  if (act == TRAIN_ACT_SILU) {
    const float s = 1.f / (1.f + expf(-z));
    return dy * (s * (1.f + z * (1.f - s)));
  }
  return dy;
}

struct Part {            // of a piece: forward (mean, squared deviations from it); backward (sum dz, sum dz * xh)
  float a, b;
};

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int m = 32; m > 0; m >>= 1) v += __shfl_xor(v, m);
  return v;
}

// One wave a piece of one channel of one image; pixels `stride` elements apart.
template <typename T>
__global__ __launch_bounds__(kThreads) void k_gn_fwd_parts(const T* __restrict__ x, Part* __restrict__ part, Gn q, int nhwc) {
  const size_t piece = (size_t)blockIdx.x * (kThreads / 64) + threadIdx.x / 64;
  if (piece >= (size_t)q.N * q.C * q.pieces) return;
  const size_t row = piece / q.pieces, n = row / q.C, c = row % q.C;
  const size_t p0 = piece % q.pieces * q.step, p1 = min(q.P, p0 + q.step);
  const size_t stride = nhwc ? q.C : 1;
  const T* xp = x + (nhwc ? n * q.P * q.C + c : row * q.P);
  // deviations from the first pixel keep the sums small beside a large mean
  const float first = Elt<T>::ld(xp + p0 * stride);
  float s = 0.f, s2 = 0.f;
  for (size_t p = p0 + threadIdx.x % 64; p < p1; p += 64) {
    const float d = Elt<T>::ld(xp + p * stride) - first;
    s += d;
    s2 += d * d;
  }
  s = wave_sum(s);
  s2 = wave_sum(s2);
  const float d = s / (float)(p1 - p0);
  if (threadIdx.x % 64 == 0) part[piece] = Part{first + d, s2 - s * d};
}

// One wave a group of one image
__global__ __launch_bounds__(kThreads) void k_gn_fwd_join(const Part* __restrict__ part, float* __restrict__ mean,
                                                          float* __restrict__ rstd, float2* __restrict__ stat, Gn q) {
  const size_t g = (size_t)blockIdx.x * (kThreads / 64) + threadIdx.x / 64;
  if (g >= (size_t)q.N * q.G) return;
  const int total = q.cg * q.pieces;
  const Part* p = part + g * total;
  const double M = (double)q.cg * (double)q.P;
  double s = 0, s2 = 0;
  for (int i = threadIdx.x % 64; i < total; i += 64) {
    const int k = i % q.pieces;
    s += (double)p[i].a * (double)(min(q.P, (k + 1) * q.step) - k * q.step);
  }
#pragma unroll
  for (int m = 32; m > 0; m >>= 1) s += __shfl_xor(s, m);
  const double mu = s / M;
  for (int i = threadIdx.x % 64; i < total; i += 64) {
    const int k = i % q.pieces;
    const double d = (double)p[i].a - mu;
    s2 += (double)p[i].b + d * d * (double)(min(q.P, (k + 1) * q.step) - k * q.step);
  }
#pragma unroll
  for (int m = 32; m > 0; m >>= 1) s2 += __shfl_xor(s2, m);
  if (threadIdx.x % 64) return;
  const float r = (float)(1.0 / sqrt(s2 / M + (double)q.eps));
  stat[g] = make_float2((float)mu, r);
  if (mean) mean[g] = (float)mu;
  if (rstd) rstd[g] = r;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void k_gn_fwd_map(const T* __restrict__ x, const float* __restrict__ gamma,
                                                         const float* __restrict__ beta, T* __restrict__ y,
                                                         const float2* __restrict__ stat, Gn q, int nhwc) {
  const size_t total = (size_t)q.N * q.C * q.P;
  for (size_t i = (size_t)blockIdx.x * kThreads + threadIdx.x; i < total; i += (size_t)gridDim.x * kThreads) {
    const size_t n = i / (q.C * q.P);
    const int c = nhwc ? (int)(i % q.C) : (int)(i / q.P % q.C);
    const float2 s = stat[n * q.G + c / q.cg];
    const float z = affine(normalised(Elt<T>::ld(x + i), s.x, s.y), gamma ? gamma[c] : 1.f, beta ? beta[c] : 0.f);
    Elt<T>::st(y + i, activate(z, q.act));
  }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void k_gn_bwd_parts(const T* __restrict__ x, const T* __restrict__ dy,
                                                           const float* __restrict__ gamma, const float* __restrict__ beta,
                                                           const float* __restrict__ mean, const float* __restrict__ rstd,
                                                           Part* __restrict__ part, Gn q, int nhwc) {
  const size_t piece = (size_t)blockIdx.x * (kThreads / 64) + threadIdx.x / 64;
  if (piece >= (size_t)q.N * q.C * q.pieces) return;
  const size_t row = piece / q.pieces, n = row / q.C, c = row % q.C;
  const size_t p0 = piece % q.pieces * q.step, p1 = min(q.P, p0 + q.step);
  const size_t stride = nhwc ? q.C : 1, at = nhwc ? n * q.P * q.C + c : row * q.P;
  const float mu = mean[n * q.G + c / q.cg], r = rstd[n * q.G + c / q.cg];
  const float ga = gamma ? gamma[c] : 1.f, be = beta ? beta[c] : 0.f;
  float s1 = 0.f, s2 = 0.f;
  for (size_t p = p0 + threadIdx.x % 64; p < p1; p += 64) {
    const float xh = normalised(Elt<T>::ld(x + at + p * stride), mu, r);
    const float dz = through(Elt<T>::ld(dy + at + p * stride), affine(xh, ga, be), q.act);
    s1 += dz;
    s2 += dz * xh;
  }
  s1 = wave_sum(s1);
  s2 = wave_sum(s2);
  if (threadIdx.x % 64 == 0) part[piece] = Part{s1, s2};
}

// The first N * G waves: a group's two means.  The next C waves: a channel's dbeta and dgamma.
__global__ __launch_bounds__(kThreads) void k_gn_bwd_join(const Part* __restrict__ part, const float* __restrict__ gamma,
                                                          float* __restrict__ dgamma, float* __restrict__ dbeta,
                                                          float2* __restrict__ stat, Gn q) {
  size_t w = (size_t)blockIdx.x * (kThreads / 64) + threadIdx.x / 64;
  const size_t groups = (size_t)q.N * q.G;
  double s1 = 0, s2 = 0;
  if (w < groups) {
    const int total = q.cg * q.pieces, c0 = (int)(w % q.G) * q.cg;
    const Part* p = part + w * total;
    for (int i = threadIdx.x % 64; i < total; i += 64) {
      const float ga = gamma ? gamma[c0 + i / q.pieces] : 1.f;
      s1 += (double)p[i].a * ga;
      s2 += (double)p[i].b * ga;
    }
  } else {
    w -= groups;
    if (w >= (size_t)q.C) return;
    for (int i = threadIdx.x % 64; i < q.N * q.pieces; i += 64) {
      const Part p = part[((size_t)(i / q.pieces) * q.C + w) * q.pieces + i % q.pieces];
      s1 += p.a;
      s2 += p.b;
    }
    w += groups;
  }
#pragma unroll
  for (int m = 32; m > 0; m >>= 1) {
    s1 += __shfl_xor(s1, m);
    s2 += __shfl_xor(s2, m);
  }
  if (threadIdx.x % 64) return;
  if (w < groups) {
    const double M = (double)q.cg * (double)q.P;
    stat[w] = make_float2((float)(s1 / M), (float)(s2 / M));
  } else {
    if (dbeta) dbeta[w - groups] = (float)s1;
    if (dgamma) dgamma[w - groups] = (float)s2;
  }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void k_gn_bwd_map(const T* __restrict__ x, const T* dy, const float* __restrict__ gamma,
                                                         const float* __restrict__ beta, const float* __restrict__ mean,
                                                         const float* __restrict__ rstd, T* dx,
                                                         const float2* __restrict__ stat, Gn q, int nhwc) {
  const size_t total = (size_t)q.N * q.C * q.P;
  for (size_t i = (size_t)blockIdx.x * kThreads + threadIdx.x; i < total; i += (size_t)gridDim.x * kThreads) {
    const size_t n = i / (q.C * q.P);
    const int c = nhwc ? (int)(i % q.C) : (int)(i / q.P % q.C);
    const size_t g = n * q.G + c / q.cg;
    const float ga = gamma ? gamma[c] : 1.f, r = rstd[g];
    const float xh = normalised(Elt<T>::ld(x + i), mean[g], r);
    const float t = through(Elt<T>::ld(dy + i), affine(xh, ga, beta ? beta[c] : 0.f), q.act) * ga;
    Elt<T>::st(dx + i, r * (t - stat[g].x - xh * stat[g].y));
  }
}

bool shaped(int N, int C, size_t P, int groups) {
  return N >= 1 && C >= 1 && P >= 1 && groups >= 1 && groups <= C && C % groups == 0 && P < (1ull << 40) &&
         (size_t)N * C < (1ull << 31) && (size_t)N * C * P < (1ull << 46);
}
Gn pieces_of(int N, int C, size_t P, int groups) {
  Gn q = {};
  q.N = N, q.C = C, q.G = groups, q.cg = C / groups, q.P = P;
  // a few thousand waves where the map has them, at least 1024 pixels each
  const size_t rows = (size_t)N * C;
  size_t want = std::max<size_t>(1, (8192 + rows - 1) / rows);
  want = std::min(want, std::max<size_t>(1, P / 1024));
  q.step = (P + want - 1) / want;
  q.pieces = (int)((P + q.step - 1) / q.step);
  return q;
}
size_t parts_bytes(const Gn& q) { return ((size_t)q.N * q.C * q.pieces * sizeof(Part) + 255) / 256 * 256; }
size_t need(const Gn& q) { return parts_bytes(q) + (size_t)q.N * q.G * sizeof(float2); }
unsigned waves(size_t n) { return (unsigned)((n + kThreads / 64 - 1) / (kThreads / 64)); }
unsigned map_blocks(const Gn& q) {
  return (unsigned)std::min<size_t>(((size_t)q.N * q.C * q.P + kThreads - 1) / kThreads, 1u << 16);
}
bool misaligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }
bool known(int act, int layout) {
  return (act == TRAIN_ACT_NONE || act == TRAIN_ACT_RELU || act == TRAIN_ACT_SILU) && (layout == TRAIN_NCHW || layout == TRAIN_NHWC);
}

template <typename T>
int fwd(const T* x, const float* gamma, const float* beta, T* y, float* mean, float* rstd, int N, int C, size_t P, int groups,
        float eps, int act, int layout, void* ws, size_t ws_bytes, void* stream) {
  if (!x || !y) return ROTCONV_ERR_NULL;
  if (!shaped(N, C, P, groups)) return ROTCONV_ERR_SHAPE;
  if (!known(act, layout) || !(eps >= 0.f) || misaligned(x, sizeof(T)) || misaligned(y, sizeof(T))) return ROTCONV_ERR_UNSUPPORTED;
  Gn q = pieces_of(N, C, P, groups);
  q.eps = eps, q.act = act;
  if (!ws || misaligned(ws, 16) || ws_bytes < need(q)) return ROTCONV_ERR_WORKSPACE;
  hipStream_t st = static_cast<hipStream_t>(stream);
  Part* part = static_cast<Part*>(ws);
  float2* stat = reinterpret_cast<float2*>(static_cast<char*>(ws) + parts_bytes(q));
  k_gn_fwd_parts<T><<<waves((size_t)N * C * q.pieces), kThreads, 0, st>>>(x, part, q, layout);
  k_gn_fwd_join<<<waves((size_t)N * groups), kThreads, 0, st>>>(part, mean, rstd, stat, q);
  k_gn_fwd_map<T><<<map_blocks(q), kThreads, 0, st>>>(x, gamma, beta, y, stat, q, layout);
  return finish();
}

template <typename T>
int bwd(const T* x, const T* dy, const float* gamma, const float* beta, const float* mean, const float* rstd, T* dx,
        float* dgamma, float* dbeta, int N, int C, size_t P, int groups, int act, int layout, void* ws, size_t ws_bytes,
        void* stream) {
  if (!x || !dy || !mean || !rstd || !dx) return ROTCONV_ERR_NULL;
  if (!shaped(N, C, P, groups)) return ROTCONV_ERR_SHAPE;
  if (!known(act, layout) || misaligned(x, sizeof(T)) || misaligned(dy, sizeof(T)) || misaligned(dx, sizeof(T)))
    return ROTCONV_ERR_UNSUPPORTED;
  Gn q = pieces_of(N, C, P, groups);
  q.act = act;
  if (!ws || misaligned(ws, 16) || ws_bytes < need(q)) return ROTCONV_ERR_WORKSPACE;
  hipStream_t st = static_cast<hipStream_t>(stream);
  Part* part = static_cast<Part*>(ws);
  float2* stat = reinterpret_cast<float2*>(static_cast<char*>(ws) + parts_bytes(q));
  k_gn_bwd_parts<T><<<waves((size_t)N * C * q.pieces), kThreads, 0, st>>>(x, dy, gamma, beta, mean, rstd, part, q, layout);
  k_gn_bwd_join<<<waves((size_t)N * groups + C), kThreads, 0, st>>>(part, gamma, dgamma, dbeta, stat, q);
  k_gn_bwd_map<T><<<map_blocks(q), kThreads, 0, st>>>(x, dy, gamma, beta, mean, rstd, dx, stat, q, layout);
  return finish();
}

}  // namespace
}  // namespace rotconv

extern "C" {

size_t train_groupnorm_workspace_bytes(int N, int C, size_t P, int groups) {
  if (!rotconv::shaped(N, C, P, groups)) return 0;
  return rotconv::need(rotconv::pieces_of(N, C, P, groups));
}
int train_groupnorm_fwd(const float* x, const float* gamma, const float* beta, float* y, float* mean, float* rstd, int N, int C,
                        size_t P, int groups, float eps, int act, int layout, void* ws, size_t ws_bytes, void* stream) {
  return rotconv::fwd<float>(x, gamma, beta, y, mean, rstd, N, C, P, groups, eps, act, layout, ws, ws_bytes, stream);
}
int train_groupnorm_fwd_bf16(const uint16_t* x, const float* gamma, const float* beta, uint16_t* y, float* mean, float* rstd,
                             int N, int C, size_t P, int groups, float eps, int act, int layout, void* ws, size_t ws_bytes,
                             void* stream) {
  return rotconv::fwd<uint16_t>(x, gamma, beta, y, mean, rstd, N, C, P, groups, eps, act, layout, ws, ws_bytes, stream);
}
int train_groupnorm_bwd(const float* x, const float* dy, const float* gamma, const float* beta, const float* mean,
                        const float* rstd, float* dx, float* dgamma, float* dbeta, int N, int C, size_t P, int groups, int act,
                        int layout, void* ws, size_t ws_bytes, void* stream) {
  return rotconv::bwd<float>(x, dy, gamma, beta, mean, rstd, dx, dgamma, dbeta, N, C, P, groups, act, layout, ws, ws_bytes, stream);
}
int train_groupnorm_bwd_bf16(const uint16_t* x, const uint16_t* dy, const float* gamma, const float* beta, const float* mean,
                             const float* rstd, uint16_t* dx, float* dgamma, float* dbeta, int N, int C, size_t P, int groups,
                             int act, int layout, void* ws, size_t ws_bytes, void* stream) {
  return rotconv::bwd<uint16_t>(x, dy, gamma, beta, mean, rstd, dx, dgamma, dbeta, N, C, P, groups, act, layout, ws, ws_bytes, stream);
}

}  // extern "C"
