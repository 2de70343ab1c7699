// Log-probabilities of labels, forward and backward, and the clipped policy loss with its gradient (see
// include/unettrain.h).
//
// A row is the K logits of a pixel or token.  With t its largest, y_j = z_j - t, s = sum exp(y_j) and h = sum exp(y_j) y_j,
//     l = ln s      logp = y_label - l      entropy = l - h / s      p_j = exp(y_j) / s
// and every gradient here has the form dz_j = c1 1[j = label] - p_j (base + c2 y_j), with base = c1 + c2 (entropy - l): c1 is the
// gradient of the log-probability, c2 that of the entropy.  All of it is bound by memory, but only just: a row is read once, held in
// registers (packed as it came) while its sums are formed, and its gradient written from there.
// Exponentials are the instruction's, of base 2, of x_j = y_j log2 e.
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstdint>

#include "glue_elt.h"
#include "rotconv.h"
#include "unettrain.h"

namespace rotconv {

enum Mode { kFwd, kBwd, kPolicy };
constexpr int kMostBlocks = 8192;      // of a launch whose workgroups have four sums each in the workspace; others: kMostOthers
constexpr int kMostOthers = 65536;

struct LossArgs {
  const void* z;
  const int32_t* labels;
  const float *stat, *ent, *dlogp, *dent;                    // backward
  const float *adv, *old, *ref, *w;                          // policy
  float *logp, *ent_out, *stat_out;
  void* dz;                                                  // may be z
  double* part;
  size_t rows, P;
  int K, per_image;
  int alike;                                                 // rows: dz's vectors start where z's do
  int past;                                                  // rows of many classes: past the caches, 1: gradients, 2: logits too
  float4* shares;                                            // few long rows: t, s, h of every part of a row ..
  float* taken;                                              // .. and the label's logit of every row
  float low, high, kl, entc, unit;                           // the clipping range's ends; unit: the weight where there are none
};

// The loss and its gradient (train_policy.hip): kernels of their own, since they are many.
void launch_policy(const LossArgs& g, bool bf16, bool rows, float* out, hipStream_t st);

namespace {

struct RowIn {                         // what a row brings beside its logits
  int label;
  float a, b, c, d;                    // backward: t, l, dlogp, dentropy; policy: advantage, logp_old, logp_ref, weight
  float ent;                           // backward
};
struct RowGrad {
  float t, inv, c1, base, c2;          // p_j = exp2(x_j) inv, dz_j = c1 1[j = label] - p_j (base + c2 x_j)
  bool live;                           // false: the row's gradient is 0
};

constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.693147180559945309f;

// what a row's logits are taken from: the largest, or 0 where that is -infinity
__device__ __forceinline__ float origin(float t) { return t == -INFINITY ? 0.f : t; }
__device__ __forceinline__ float exponent(float z, float from) { return (z - from) * kLog2e; }
__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }
// x as a factor: what lies 10^30 below a row's largest (-infinity too) counts as that, so that 0 times it stays 0; a NaN's exponential is a
// factor beside it
__device__ __forceinline__ float bounded(float x) { return fmaxf(x, -1e30f); }

template <int MODE>
__device__ __forceinline__ RowIn row_in(const LossArgs& g, size_t row) {
  RowIn r = {};
  // (nothing writes labels here: constant memory, which a scalar load reads where a workgroup has one row, and no wait for vectors with it)
  r.label = reinterpret_cast<const __attribute__((address_space(4))) int*>(reinterpret_cast<uintptr_t>(g.labels))[row];
  if constexpr (MODE == kBwd) {
    r.a = g.stat[2 * row], r.b = g.stat[2 * row + 1];
    r.c = g.dlogp[row];
    if (g.dent) r.d = g.dent[row], r.ent = g.ent[row];
  } else if constexpr (MODE == kPolicy) {
    r.a = g.adv[g.per_image ? (uint32_t)row / (uint32_t)g.P : row];
    if (g.old) r.b = g.old[row];
    if (g.ref) r.c = g.ref[row];
    r.d = g.w ? g.w[row] : g.unit;
  }
  return r;
}
__device__ __forceinline__ bool has_label(const LossArgs& g, const RowIn& r) { return r.label >= 0 && r.label < g.K; }

// exp(q) - 1 and exp(q) - q - 1: by series near 0, where the differences would lose their digits
__device__ __forceinline__ void distance(float q, float* e1, float* d) {
  if (fabsf(q) < 0.25f) {
    float s = 1.f / 40320;
    s = fmaf(s, q, 1.f / 5040), s = fmaf(s, q, 1.f / 720), s = fmaf(s, q, 1.f / 120);
    s = fmaf(s, q, 1.f / 24), s = fmaf(s, q, 1.f / 6), s = fmaf(s, q, 0.5f);
    *d = s * q * q;
    *e1 = q + *d;
  } else {
    *e1 = exp2_of(q * kLog2e) - 1.f;
    *d = *e1 == INFINITY ? INFINITY : *e1 - q;
  }
}

__device__ __forceinline__ void add_element(float z, float from, float& s, float& h) {
  const float x = exponent(z, from), e = exp2_of(x);
  s += e;
  h = fmaf(e, bounded(x), h);
}

struct RowOut {
  float logp, ent, t, l;
};

// A row's results from its sums (s, h: over exp2(x) and exp2(x) x), for memory (out) and for the gradient; adds: its part of the sums
// over rows goes to acc.
template <int MODE, typename A>
__device__ __forceinline__ RowGrad row_end(const LossArgs& g, const RowIn& r, float t, float s, float h, float za, RowOut* out, bool adds, A* acc) {
  RowGrad o = {};
  if constexpr (MODE == kBwd) {
    o.t = r.a;
    o.inv = exp2_of(-r.b * kLog2e);
    o.c1 = r.c, o.c2 = r.d * kLn2;
    o.base = r.d == 0.f ? r.c : r.c + r.d * (r.ent - r.b);
    // (a row of NaN, or of NaN beside -infinity, has t at -infinity too, but l is NaN there)
    o.live = has_label(g, r) && !(r.a == -INFINITY && r.b == 0.f) && !(r.c == 0.f && r.d == 0.f);
  } else {
    const bool none = t == -INFINITY && s == 0.f;
    bool live = has_label(g, r) && !none;
    if constexpr (MODE == kPolicy) live = live && r.d != 0.f;
    const float l = __logf(s), inv = __builtin_amdgcn_rcpf(s), logp = za - t - l, ent = l - kLn2 * (h * inv);
    *out = RowOut{live ? logp : 0.f, live ? ent : 0.f, has_label(g, r) ? t : 0.f, live ? l : 0.f};
    if constexpr (MODE == kPolicy) {
      const float a = r.a, w = r.d;
      const float ratio = g.old ? exp2_of((logp - r.b) * kLog2e) : 1.f;
      const bool cut = (a > 0.f && ratio > g.high) || (a < 0.f && ratio < g.low);
      // (a = 0 counts as no advantage whatever the ratio; a NaN goes through)
      const float kept = a == 0.f ? 0.f : ratio * a, gain = cut ? (a > 0.f ? g.high : g.low) * a : kept;
      float loss = -gain, G = cut ? 0.f : -kept, d = 0.f, H = 0.f;
      if (g.kl != 0.f && g.ref) {
        float e1;
        distance(r.c - logp, &e1, &d);
        loss += g.kl * d;
        G -= g.kl * e1;
      }
      if (g.entc != 0.f) {
        H = ent;
        loss -= g.entc * H;
      }
      if (adds && live) {
        const A term[4] = {(A)w * loss, (A)w * d, (A)w * H, cut ? (A)w : (A)0};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          acc[i] += term[i];
          asm volatile("" ::: "memory");               // (one after another: in LDS, four at once would cost a row's thread 16 registers)
        }
      }
      o.t = t;
      o.inv = inv;
      o.c1 = w * G;
      const float c2 = -g.entc * w;
      o.c2 = c2 * kLn2;
      o.base = g.entc != 0.f ? o.c1 + c2 * (ent - l) : o.c1;
      o.live = live;
    }
  }
  return o;
}
template <int MODE>
__device__ __forceinline__ void write_row(const LossArgs& g, size_t row, const RowOut& out) {
  if (MODE != kBwd && g.logp) g.logp[row] = out.logp;
  if (MODE == kFwd && g.ent_out) g.ent_out[row] = out.ent;
  if (MODE == kFwd && g.stat_out) g.stat_out[2 * row] = out.t, g.stat_out[2 * row + 1] = out.l;
}
__device__ __forceinline__ float element(const RowGrad& o, float z, bool label) {
  const float x = exponent(z, o.t), p = exp2_of(x) * o.inv;
  return (label ? o.c1 : 0.f) - p * fmaf(o.c2, bounded(x), o.base);
}

// Waits for a loaded value.  Where gradients take the logits' place, other waves store behind the next barrier, and a barrier alone
// does not wait for loads under way.
template <typename T>
__device__ __forceinline__ void arrived(T v) { asm volatile("" ::"v"(v)); }

// Sums that were formed below the maximum t, for the larger of t and top.  (Sums of nothing, at -infinity, stay 0; a NaN stays.)
__device__ __forceinline__ void moved_to(float top, float& t, float& s, float& h) {
  top = fmaxf(t, top);
  const float by = bounded(exponent(t, top)), f = exp2_of(by);
  h = f * fmaf(by, s, h);
  s = f * s;
  t = top;
}
// A vector's elements are taken from it anew, one vector after the other: the compiler would keep them all, in twice the registers for bf16.
__device__ __forceinline__ void packed(u4& v) {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("" : "+v"(v));
}

// max and sum over G neighbouring lanes
template <int G> __device__ __forceinline__ float lanes_max(float v) {
#pragma unroll
  for (int k = G / 2; k > 0; k /= 2) v = fmaxf(v, __shfl_xor(v, k));
  return v;
}
template <int G> __device__ __forceinline__ float lanes_sum(float v) {
#pragma unroll
  for (int k = G / 2; k > 0; k /= 2) v += __shfl_xor(v, k);
  return v;
}
// The four sums of a workgroup, to its place in the workspace.  Half of a wave's lanes take two of the sums, half of these one: 7 exchanges
// instead of 24.
__device__ __forceinline__ void write_sums(const LossArgs& g, const double* acc) {
  __shared__ double red[16][4];
  const int lane = threadIdx.x % 64, waves = (blockDim.x + 63) / 64;
  const bool upper = lane & 32, odd = lane & 16;
  const double a = (upper ? acc[2] : acc[0]) + __shfl_xor(upper ? acc[0] : acc[2], 32);
  const double b = (upper ? acc[3] : acc[1]) + __shfl_xor(upper ? acc[1] : acc[3], 32);
  double v = (odd ? b : a) + __shfl_xor(odd ? a : b, 16);
#pragma unroll
  for (int o = 8; o > 0; o /= 2) v += __shfl_xor(v, o);
  if (lane % 16 == 0) red[threadIdx.x / 64][lane / 16] = v;
  __syncthreads();
  if (threadIdx.x < 4) {
    v = 0;
    for (int w = 0; w < waves; ++w) v += red[w][threadIdx.x];
    g.part[4 * (size_t)blockIdx.x + threadIdx.x] = v;
  }
}

// Rows of few classes: G lanes to a row, up to E elements a lane, an element to a load (neighbouring rows lie side by side).
template <typename T, int G, int E, int MODE>
__global__ __launch_bounds__(256) void k_rows_small(LossArgs g) {
  const int sub = threadIdx.x % G;
  const size_t apart = (size_t)gridDim.x * (256 / G);
  double acc[4] = {};
  for (size_t row = (size_t)blockIdx.x * (256 / G) + threadIdx.x / G; row < g.rows; row += apart) {
    const T* z = static_cast<const T*>(g.z) + row * g.K;
    const RowIn r = row_in<MODE>(g, row);
    float v[E], t = -INFINITY, s = 0.f, h = 0.f, za = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = sub + G * e < g.K ? Elt<T>::ld(z + sub + G * e) : -INFINITY;
    if constexpr (MODE != kBwd) {
      if (has_label(g, r)) za = Elt<T>::ld(z + r.label);
#pragma unroll
      for (int e = 0; e < E; ++e) t = fmaxf(t, v[e]);
      t = lanes_max<G>(t);
      const float from = origin(t);
#pragma unroll
      for (int e = 0; e < E; ++e) add_element(v[e], from, s, h);
      s = lanes_sum<G>(s), h = lanes_sum<G>(h);
    }
    RowOut out;
    const RowGrad o = row_end<MODE>(g, r, t, s, h, za, &out, sub == 0, acc);
    if (sub == 0) write_row<MODE>(g, row, out);
    if (MODE != kFwd && g.dz) {
      T* d = static_cast<T*>(g.dz) + row * g.K;
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (sub + G * e < g.K) Elt<T>::st(d + sub + G * e, o.live ? element(o, v[e], sub + G * e == r.label) : 0.f);
    }
  }
  if constexpr (MODE == kPolicy) write_sums(g, acc);
}

// two values rounded to nearest even by the instruction
__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {
  typedef __bf16 b2 __attribute__((ext_vector_type(2)));
  typedef float f2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f2{a, b}, b2));
}

// A vector of 16 bytes as it lies in memory.  Rows start anywhere: vectors are those of the address space, and the first
// and the last of a row may hold elements of its neighbours, which are neither read nor written.
template <typename T> struct Vec;
template <> struct Vec<float> {
  static constexpr int V = 4;
  static constexpr uint32_t kLowest = 0xff800000u;
  static __device__ __forceinline__ float get(const u4& a, int k) { return __uint_as_float(a[k]); }
  static __device__ __forceinline__ void put(u4& a, int k, float v) { a[k] = __float_as_uint(v); }
  static __device__ __forceinline__ u4 pack(const float* v) {
    return u4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
  }
};
template <> struct Vec<uint16_t> {
  static constexpr int V = 8;
  static constexpr uint32_t kLowest = 0xff80ff80u;
  static __device__ __forceinline__ float get(const u4& a, int k) {
    return __uint_as_float(k % 2 ? a[k / 2] & 0xffff0000u : a[k / 2] << 16);
  }
  static __device__ __forceinline__ void put(u4& a, int k, float v) {        // (a value that a bf16 number holds)
    const uint32_t b = __float_as_uint(v);
    a[k / 2] = k % 2 ? (a[k / 2] & 0xffffu) | (b & 0xffff0000u) : (a[k / 2] & 0xffff0000u) | b >> 16;
  }
  static __device__ __forceinline__ u4 pack(const float* v) {
    return u4{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7])};
  }
};
// The vector of a row at `border` (the same for all lanes, so that addresses take no registers) + `off` elements; its first element is the
// row's number `first`.  -infinity outside the row.
template <typename T>
__device__ __forceinline__ u4 load_part(const T* border, uint32_t off, int first, int K) {
  constexpr int V = Vec<T>::V;
  if (first >= 0 && first + V <= K) return *reinterpret_cast<const u4*>(border + off);
  u4 a;
#pragma unroll
  for (int k = 0; k < 4; ++k) a[k] = Vec<T>::kLowest;
  if (first + V <= 0 || first >= K) return a;
  const T* row = border + off - first;
  float v[V];                          // all of them under way at once, from inside the row
#pragma unroll
  for (int k = 0; k < V; ++k) v[k] = Elt<T>::ld(row + min(max(first + k, 0), K - 1));
#pragma unroll
  for (int k = 0; k < V; ++k) Vec<T>::put(a, k, first + k >= 0 && first + k < K ? v[k] : -INFINITY);
  return a;
}
template <typename T, bool EVEN = false>       // EVEN: as in k_rows
__device__ __forceinline__ void store_part(T* border, uint32_t off, const u4& a, int first, int K, bool alike, bool past = false) {
  constexpr int V = Vec<T>::V;
  if (EVEN ? first < K : alike && first >= 0 && first + V <= K) {
    u4* to = reinterpret_cast<u4*>(border + off);
    if (past) {
      asm volatile("");                                // (before and behind: else the compiler makes one store of the two, through the caches)
      __builtin_nontemporal_store(a, to);
      asm volatile("");
    } else {
      *to = a;
    }
    return;
  }
  if constexpr (EVEN) return;
  T* row = border + off - first;
#pragma unroll
  for (int k = 0; k < V; ++k)
    if (first + k >= 0 && first + k < K) Elt<T>::st(row + first + k, Vec<T>::get(a, k));
}

// over the workgroup's B threads, the same in all of them; red: a float a wave
template <int B, bool MAX>
__device__ __forceinline__ float block_join(float v, float* red) {
  v = MAX ? lanes_max<64>(v) : lanes_sum<64>(v);
  if constexpr (B == 64) return v;
  __syncthreads();
  if (threadIdx.x % 64 == 0) red[threadIdx.x / 64] = v;
  __syncthreads();
  v = red[threadIdx.x % (B / 64)];
  return MAX ? lanes_max<B / 64>(v) : lanes_sum<B / 64>(v);
}

// ENT: the gradient has a part of the entropy's.  The label's own part is added where it lies.
template <typename T, bool ENT>
__device__ __forceinline__ u4 gradient(const RowGrad& o, const u4& a, int first, int label) {
  constexpr int V = Vec<T>::V;
  float d[V];
  const float factor = -o.inv * o.base;
#pragma unroll
  for (int k = 0; k < V; ++k) {
    const float x = exponent(Vec<T>::get(a, k), o.t), e = exp2_of(x);
    d[k] = ENT ? -(e * o.inv) * fmaf(o.c2, bounded(x), o.base) : e * factor;
  }
  if (label >= first && label < first + V) {
#pragma unroll
    for (int k = 0; k < V; ++k) d[k] += first + k == label ? o.c1 : 0.f;
  }
  return Vec<T>::pack(d);
}

// A value that a wave's lanes have alike, in a scalar register.
__device__ __forceinline__ float wave_wide(float v) { return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(v))); }
__device__ __forceinline__ RowGrad row_wide(const RowGrad& o) {
  return RowGrad{wave_wide(o.t), wave_wide(o.inv), wave_wide(o.c1), wave_wide(o.base), wave_wide(o.c2), __builtin_amdgcn_readfirstlane(o.live) != 0};
}

// Rows of many classes: B threads to a row, up to E vectors a thread in registers (those that no thread has are passed over).  64
// threads: four rows to a workgroup.  E = 0: rows of any length, read twice (their sums are then formed with a running maximum).
// ENT: somebody wants the entropy or its gradient.  EVEN: rows start on 16-byte borders and are whole vectors; nothing is asked of an end
// then, and no registers are kept for it (4096 x 65536 bf16 logits, loss, through the caches: 201 us, and 240 with the ends' code beside).
template <typename T, int B, int E, int MODE, bool ENT, bool EVEN>
__global__ __launch_bounds__(B == 64 ? 256 : B) __attribute__((amdgpu_waves_per_eu(E == 16 ? 4 : 8))) void k_rows(LossArgs g) {
  constexpr int V = Vec<T>::V, kRows = B == 64 ? 4 : 1;
  const int tid = threadIdx.x % B, which = kRows == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / B);
  __shared__ float red[16];
  __shared__ double sums[kRows][4];    // the rows' first threads'
  double* acc = sums[which];
  if (MODE == kPolicy && tid == 0) acc[0] = acc[1] = acc[2] = acc[3] = 0;
  for (size_t row = (size_t)blockIdx.x * kRows + which; row < g.rows; row += (size_t)gridDim.x * kRows) {
    const T* z = static_cast<const T*>(g.z) + row * g.K;
    T* dz = static_cast<T*>(g.dz) + row * g.K;
    // elements between the last 16-byte border and the row's start
    const int shift = EVEN ? 0 : (int)(reinterpret_cast<uintptr_t>(z) % 16 / sizeof(T));
    const RowIn r = row_in<MODE>(g, row);
    float t = -INFINITY, s = 0.f, h = 0.f, za = 0.f;
    // (as it is stored, and some class's without a label: a conversion or a branch would wait for it before the row's loads)
    T taken = {};
    if constexpr (MODE != kBwd) taken = z[has_label(g, r) ? r.label : 0];
    const u4 zero = {};
    if constexpr (E > 0) {
      int lane = tid;                  // (opaque: places are formed anew where they are asked for, and kept in no registers between)
      asm volatile("" : "+v"(lane));
      u4 v[E];
      if constexpr (EVEN) {
        const auto at = [&](int e) { return reinterpret_cast<const u4*>(z + min((uint32_t)(lane + e * B) * V, (uint32_t)g.K - V)); };
        if (g.past == 2) {
          asm volatile("");                            // (as in store_part)
#pragma unroll
          for (int e = 0; e < E; ++e) v[e] = __builtin_nontemporal_load(at(e));
          asm volatile("");
        } else {
#pragma unroll
          for (int e = 0; e < E; ++e) v[e] = *at(e);
        }
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (e * B * V < g.K + V - 1) v[e] = load_part(z - shift + e * B * V, lane * V, (lane + e * B) * V - shift, g.K);
      }
      if constexpr (MODE != kBwd) {
        arrived(taken);
        za = has_label(g, r) ? Elt<T>::ld(&taken) : 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) {
          if constexpr (EVEN) {
            asm volatile("" : "+v"(lane));
#pragma unroll
            for (int k = 0; k < 4; ++k) v[e][k] = (lane + e * B) * V < g.K ? v[e][k] : (uint32_t)Vec<T>::kLowest;
          } else if (e * B * V >= g.K + V - 1) continue;
#pragma unroll
          for (int k = 0; k < V; ++k) t = fmaxf(t, Vec<T>::get(v[e], k));
        }
        t = block_join<B, true>(t, red);
        const float from = wave_wide(origin(t));
#pragma unroll
        for (int e = 0; e < E; ++e) {
          if (e * B * V >= g.K + V - 1) continue;
          packed(v[e]);
#pragma unroll
          for (int k = 0; k < V; ++k) {
            if constexpr (ENT) add_element(Vec<T>::get(v[e], k), from, s, h);
            else s += exp2_of(exponent(Vec<T>::get(v[e], k), from));
          }
          asm volatile("" : "+v"(s), "+v"(h));         // (both sums now: the compiler would put one off, and keep its terms)
        }
        s = block_join<B, false>(s, red);
        if constexpr (ENT) h = block_join<B, false>(h, red);
      }
      RowOut out;
      const RowGrad o = row_wide(row_end<MODE>(g, r, t, s, h, za, &out, tid == 0, acc));
      if (tid == 0) write_row<MODE>(g, row, out);
      if (MODE != kFwd && g.dz) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
          if (e * B * V >= g.K + V - 1) continue;
          asm volatile("" : "+v"(lane));
          const int first = (lane + e * B) * V - shift;
          packed(v[e]);
          store_part<T, EVEN>(dz - shift + e * B * V, lane * V, o.live ? gradient<T, ENT>(o, v[e], first, r.label) : zero, first, g.K, g.alike,
                              g.past != 0);
        }
      }
    } else {
      if constexpr (MODE != kBwd) {
        arrived(taken);
        za = has_label(g, r) ? Elt<T>::ld(&taken) : 0.f;
        for (int first = tid * V - shift; first < g.K; first += B * V) {
          const u4 v = load_part(z - shift, first + shift, first, g.K);
          float top = t;
#pragma unroll
          for (int k = 0; k < V; ++k) top = fmaxf(top, Vec<T>::get(v, k));
          moved_to(top, t, s, h);
#pragma unroll
          for (int k = 0; k < V; ++k) add_element(Vec<T>::get(v, k), origin(t), s, h);
        }
        moved_to(block_join<B, true>(t, red), t, s, h);
        s = block_join<B, false>(s, red), h = block_join<B, false>(h, red);
      }
      RowOut out;
      const RowGrad o = row_end<MODE>(g, r, t, s, h, za, &out, tid == 0, acc);
      if (tid == 0) write_row<MODE>(g, row, out);
      if (MODE != kFwd && g.dz)
        for (int first = tid * V - shift; first < g.K; first += B * V)
          store_part(dz - shift, first + shift, o.live ? gradient<T, ENT>(o, load_part(z - shift, first + shift, first, g.K), first, r.label) : zero, first, g.K, g.alike);
    }
  }
  if constexpr (MODE == kPolicy) {
    __syncthreads();
    if (threadIdx.x < 4) {
      double v = sums[0][threadIdx.x];
      for (int r = 1; r < kRows; ++r) v += sums[r][threadIdx.x];
      g.part[4 * (size_t)blockIdx.x + threadIdx.x] = v;
    }
  }
}

// Few long rows: a row's parts of kPart vectors go to workgroups of their own, since one CU forms 16 exponentials a clock (one row of 131072
// bf16 logits: 10.8 us by one workgroup, 9.6 so).  k_share forms the parts' sums; k_rest, a launch behind it, joins a row's, each workgroup for
// itself, and writes the part's gradient.  The label's logit is passed on, since a gradient may take its place.
constexpr int kPartThreads = 256, kPartVecs = 4, kPart = kPartThreads * kPartVecs;

template <typename T>
__global__ __launch_bounds__(kPartThreads) void k_share(LossArgs g) {
  constexpr int V = Vec<T>::V;
  __shared__ float red[16];
  const size_t row = blockIdx.y;
  const T* z = static_cast<const T*>(g.z) + row * g.K;
  const int shift = (int)(reinterpret_cast<uintptr_t>(z) % 16 / sizeof(T)), from = ((int)blockIdx.x * kPart + (int)threadIdx.x) * V - shift;
  u4 v[kPartVecs];
#pragma unroll
  for (int e = 0; e < kPartVecs; ++e) v[e] = load_part(z - shift, from + shift + e * kPartThreads * V, from + e * kPartThreads * V, g.K);
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    const int label = g.labels[row];
    if (label >= 0 && label < g.K) g.taken[row] = Elt<T>::ld(z + label);
  }
  float t = -INFINITY, s = 0.f, h = 0.f;
#pragma unroll
  for (int e = 0; e < kPartVecs; ++e)
#pragma unroll
    for (int k = 0; k < V; ++k) t = fmaxf(t, Vec<T>::get(v[e], k));
  t = block_join<kPartThreads, true>(t, red);
#pragma unroll
  for (int e = 0; e < kPartVecs; ++e)
#pragma unroll
    for (int k = 0; k < V; ++k) add_element(Vec<T>::get(v[e], k), origin(t), s, h);
  s = block_join<kPartThreads, false>(s, red), h = block_join<kPartThreads, false>(h, red);
  if (threadIdx.x == 0) g.shares[row * gridDim.x + blockIdx.x] = make_float4(t, s, h, 0.f);
}

// parts: of a row; the grid has one workgroup for each, or (without a gradient) for each row
template <typename T, int MODE>
__global__ __launch_bounds__(kPartThreads) void k_rest(LossArgs g, int parts) {
  constexpr int V = Vec<T>::V;
  const size_t row = blockIdx.y;
  const T* z = static_cast<const T*>(g.z) + row * g.K;
  T* dz = static_cast<T*>(g.dz) + row * g.K;
  const bool writes = blockIdx.x == 0 && threadIdx.x == 0;
  const RowIn r = row_in<MODE>(g, row);
  float t = -INFINITY, s = 0.f, h = 0.f, za = 0.f;
  if constexpr (MODE != kBwd) {
    if (has_label(g, r)) za = g.taken[row];
    for (int c = threadIdx.x % 64; c < parts; c += 64) t = fmaxf(t, g.shares[row * parts + c].x);
    t = lanes_max<64>(t);
    for (int c = threadIdx.x % 64; c < parts; c += 64) {
      const float4 p = g.shares[row * parts + c];
      float pt = p.x, ps = p.y, ph = p.z;
      moved_to(t, pt, ps, ph);
      s += ps, h += ph;
    }
    s = lanes_sum<64>(s), h = lanes_sum<64>(h);
  }
  RowOut out;
  double acc[4] = {};
  const RowGrad o = row_end<MODE>(g, r, t, s, h, za, &out, writes, acc);
  if (writes) {
    write_row<MODE>(g, row, out);
    if constexpr (MODE == kPolicy) {
#pragma unroll
      for (int k = 0; k < 4; ++k) g.part[4 * row + k] = acc[k];
    }
  }
  if (MODE != kFwd && g.dz) {
    const int shift = (int)(reinterpret_cast<uintptr_t>(z) % 16 / sizeof(T)), from = ((int)blockIdx.x * kPart + (int)threadIdx.x) * V - shift;
    const u4 zero = {};
#pragma unroll
    for (int e = 0; e < kPartVecs; ++e) {
      const int first = from + e * kPartThreads * V;
      store_part(dz - shift, first + shift, o.live ? gradient<T, true>(o, load_part(z - shift, first + shift, first, g.K), first, r.label) : zero, first, g.K,
                 g.alike);
    }
  }
}

// Classes in planes: a lane holds V neighbouring pixels.  KM > 0: all K <= KM classes in registers; KM = 0: any number, read
// twice, and blockDim.y waves share the classes of 64 lanes' pixels.
template <typename T, int V>
__device__ __forceinline__ void load_pixels(const T* p, float* v) {
  if constexpr (V == 1) v[0] = Elt<T>::ld(p);
  else if constexpr (sizeof(T) == 4) Elt<T>::ldv(p, v);
  else Elt<T>::ldh(p, v);
}
template <typename T, int V>
__device__ __forceinline__ void store_pixels(T* p, const float* v) {
  if constexpr (V == 1) Elt<T>::st(p, v[0]);
  else if constexpr (sizeof(T) == 4) Elt<T>::stv(p, v);
  else *reinterpret_cast<uint2*>(p) = make_uint2(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]));
}

// V rows' values at a time: the caller has checked that vectors of them lie on their borders
template <int V>
__device__ __forceinline__ void load_rows(const float* p, size_t row, float* v) {
  if constexpr (V == 1) v[0] = p[row];
  else Elt<float>::ldv(p + row, v);
}
template <int MODE, int V>
__device__ __forceinline__ void rows_in(const LossArgs& g, size_t row, RowIn* r) {
  if constexpr (V == 1) {
    r[0] = row_in<MODE>(g, row);
  } else {
    float v[5][V] = {}, second[V] = {};
    load_rows<V>(reinterpret_cast<const float*>(g.labels), row, v[0]);
    if constexpr (MODE == kBwd) {
      load_rows<V>(g.stat, 2 * row, v[1]), load_rows<V>(g.stat, 2 * row + V, second);
      load_rows<V>(g.dlogp, row, v[2]);
      if (g.dent) load_rows<V>(g.dent, row, v[3]), load_rows<V>(g.ent, row, v[4]);
    } else if constexpr (MODE == kPolicy) {
      if (g.per_image) {
#pragma unroll
        for (int i = 0; i < V; ++i) v[1][i] = g.adv[(uint32_t)row / (uint32_t)g.P];      // (P is a multiple of V)
      } else {
        load_rows<V>(g.adv, row, v[1]);
      }
      if (g.old) load_rows<V>(g.old, row, v[2]);
      if (g.ref) load_rows<V>(g.ref, row, v[3]);
      if (g.w) load_rows<V>(g.w, row, v[4]);
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
      r[i].label = __float_as_int(v[0][i]);
      if constexpr (MODE == kBwd) {
        r[i].a = i < V / 2 ? v[1][2 * i] : second[2 * i - V], r[i].b = i < V / 2 ? v[1][2 * i + 1] : second[2 * i + 1 - V];
        r[i].c = v[2][i], r[i].d = v[3][i], r[i].ent = v[4][i];
      } else {
        r[i].a = v[1][i], r[i].b = v[2][i], r[i].c = v[3][i], r[i].d = g.w ? v[4][i] : g.unit, r[i].ent = 0.f;
      }
    }
  }
}

template <int V>
__device__ __forceinline__ void store_rows(float* p, size_t row, const float* v) {
  if constexpr (V == 1) p[row] = v[0];
  else Elt<float>::stv(p + row, v);
}
// Classes behind the last are -infinity, so that nothing but their loads and stores asks for K; x and its exponential are kept from the
// sums for the gradient (the 4 x 6 x 512 x 512 logits of a stack, bf16, with a reference and weights: 19.3 us where both were formed again and every
// class asked, bound by instructions; 13.9 so).
template <typename T, int V, int KM, int MODE>
__global__ __launch_bounds__(256) void k_planes(LossArgs g) {
  double acc[4] = {};
  const size_t apart = (size_t)gridDim.x * 256 * V;
  for (size_t row = ((size_t)blockIdx.x * 256 + threadIdx.x) * V; row < g.rows; row += apart) {
    const size_t n = (uint32_t)row / (uint32_t)g.P, at = n * g.K * g.P + (row - n * g.P);      // (fewer than 2^31 rows)
    float v[KM][V], p[KM][V];
    const T* z = static_cast<const T*>(g.z) + at;
#pragma unroll
    for (int k = 0; k < KM; ++k, z += g.P) {
      if (k < g.K) {
        load_pixels<T, V>(z, v[k]);
      } else {
#pragma unroll
        for (int i = 0; i < V; ++i) v[k][i] = -INFINITY;
      }
    }
    RowGrad o[V];
    RowIn r[V];
    RowOut out[V];
    float part[4] = {};
    rows_in<MODE, V>(g, row, r);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      float t = -INFINITY, s = 0.f, h = 0.f, za = 0.f;
      if constexpr (MODE != kBwd) {
#pragma unroll
        for (int k = 0; k < KM; ++k) t = fmaxf(t, v[k][i]);
#pragma unroll
        for (int k = 0; k < KM; ++k) za = k == r[i].label ? v[k][i] : za;
        asm volatile("" : "+v"(r[i].label));           // (opaque: the gradient asks again, rather than that every answer is kept)
      } else {
        t = r[i].a;
      }
      const float from = origin(t);
#pragma unroll
      for (int k = 0; k < KM; ++k) {
        const float x = exponent(v[k][i], from), e = exp2_of(x);
        v[k][i] = bounded(x), p[k][i] = e;
        s += e;
        h = fmaf(e, v[k][i], h);
      }
      o[i] = row_end<MODE>(g, r[i], t, s, h, za, &out[i], true, part);
    }
    if constexpr (MODE == kPolicy) {
#pragma unroll
      for (int k = 0; k < 4; ++k) acc[k] += part[k];
    }
    if constexpr (MODE != kBwd) {
      float w[2 * V];
      if (g.logp) {
#pragma unroll
        for (int i = 0; i < V; ++i) w[i] = out[i].logp;
        store_rows<V>(g.logp, row, w);
      }
      if (MODE == kFwd && g.ent_out) {
#pragma unroll
        for (int i = 0; i < V; ++i) w[i] = out[i].ent;
        store_rows<V>(g.ent_out, row, w);
      }
      if (MODE == kFwd && g.stat_out) {
#pragma unroll
        for (int i = 0; i < V; ++i) w[2 * i] = out[i].t, w[2 * i + 1] = out[i].l;
        store_rows<V>(g.stat_out, 2 * row, w);
        store_rows<V>(g.stat_out, 2 * row + V, w + V);
      }
    }
    if (MODE != kFwd && g.dz) {
      T* dz = static_cast<T*>(g.dz) + at;
#pragma unroll
      for (int k = 0; k < KM; ++k, dz += g.P)
        if (k < g.K) {
          float d[V];
#pragma unroll
          for (int i = 0; i < V; ++i) {
            const float c1 = k == r[i].label ? o[i].c1 : 0.f;
            d[i] = o[i].live ? c1 - p[k][i] * o[i].inv * fmaf(o[i].c2, v[k][i], o[i].base) : 0.f;
          }
          store_pixels<T, V>(dz, d);
        }
    }
  }
  if constexpr (MODE == kPolicy) write_sums(g, acc);
}

template <typename T, int V, int MODE>
__global__ __launch_bounds__(1024) void k_planes_long(LossArgs g) {
  extern __shared__ float joined[];    // of several waves: t, s, h of each
  auto shared = [&](int wave, int what, int at) -> float& { return joined[(wave * 3 + what) * 64 * V + at]; };
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, waves = blockDim.x / 64;
  double acc[4] = {};
  const size_t apart = (size_t)gridDim.x * 64 * V;
  for (size_t first = (size_t)blockIdx.x * 64 * V; first < g.rows; first += apart) {
    const size_t row = first + (size_t)lane * V;
    const bool inside = row < g.rows;
    const size_t n = (uint32_t)row / (uint32_t)g.P, at = n * g.K * g.P + (row - n * g.P);
    const T* z = static_cast<const T*>(g.z) + at;
    float t[V], s[V], h[V], za[V];
#pragma unroll
    for (int i = 0; i < V; ++i) t[i] = -INFINITY, s[i] = h[i] = za[i] = 0.f;
    if constexpr (MODE != kBwd) {
      if (inside) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const int label = g.labels[row + i];
          if (label >= 0 && label < g.K) za[i] = Elt<T>::ld(z + (size_t)label * g.P + i);
          arrived(za[i]);
        }
        // eight classes at a time: their largest first, so that the sums move to it once
        constexpr int U = 8;
        for (int k = wave; k < g.K; k += U * waves) {
          float v[U][V];
#pragma unroll
          for (int u = 0; u < U; ++u) {
            if (k + u * waves < g.K) {
              load_pixels<T, V>(z + (size_t)(k + u * waves) * g.P, v[u]);
            } else {
#pragma unroll
              for (int i = 0; i < V; ++i) v[u][i] = -INFINITY;
            }
          }
#pragma unroll
          for (int i = 0; i < V; ++i) {
            float top = v[0][i];
#pragma unroll
            for (int u = 1; u < U; ++u) top = fmaxf(top, v[u][i]);
            moved_to(top, t[i], s[i], h[i]);
            const float from = origin(t[i]);
#pragma unroll
            for (int u = 0; u < U; ++u) add_element(v[u][i], from, s[i], h[i]);
          }
        }
      }
      if (waves > 1) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < V; ++i) shared(wave, 0, lane * V + i) = t[i], shared(wave, 1, lane * V + i) = s[i], shared(wave, 2, lane * V + i) = h[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < V; ++i) {
          float top = -INFINITY;
          for (int w = 0; w < waves; ++w) top = fmaxf(top, shared(w, 0, lane * V + i));
          s[i] = h[i] = 0.f, t[i] = top;
          for (int w = 0; w < waves; ++w) {
            float tw = shared(w, 0, lane * V + i), sw = shared(w, 1, lane * V + i), hw = shared(w, 2, lane * V + i);
            moved_to(top, tw, sw, hw);
            s[i] += sw, h[i] += hw;
          }
        }
      }
    }
    if (!inside) continue;             // (every wave of the workgroup has the same lanes inside, and no barrier follows within the pass)
    RowGrad o[V];
    RowIn r[V];
    rows_in<MODE, V>(g, row, r);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      RowOut out;
      o[i] = row_end<MODE>(g, r[i], t[i], s[i], h[i], za[i], &out, wave == 0, acc);
      if (wave == 0) write_row<MODE>(g, row + i, out);
    }
    if (MODE != kFwd && g.dz) {
      T* dz = static_cast<T*>(g.dz) + at;
      constexpr int U = 4;
      for (int k = wave; k < g.K; k += U * waves) {
        float v[U][V];
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (k + u * waves < g.K) load_pixels<T, V>(z + (size_t)(k + u * waves) * g.P, v[u]);
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int at = k + u * waves;
          if (at >= g.K) continue;
#pragma unroll
          for (int i = 0; i < V; ++i) v[u][i] = o[i].live ? element(o[i], v[u][i], at == r[i].label) : 0.f;
          store_pixels<T, V>(dz + (size_t)at * g.P, v[u]);
        }
      }
    }
  }
  if constexpr (MODE == kPolicy) write_sums(g, acc);
}

bool misaligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }
template <int MODE> unsigned blocks_for(size_t n) { return (unsigned)std::min<size_t>(n, MODE == kPolicy ? kMostBlocks : kMostOthers); }

// What is larger than the caches' share of it passes them by, lest it drives out what the next calls read.  Made by a pass before, then the
// call, then its gradient read by a pass behind; all through the caches, gradients past them, logits too: loss of bf16 8192 x 4096 (64 MiB)
// 68.5, 71 and 71 us, of fp32 1237 x 20011 (94 MiB) 109.5, 105 and 106, of bf16 16384 x 4096 (128 MiB) 141, 134 and 135, of 4096 x 32768
// (256 MiB) 285, 298 and 274, 4096 x 65536 546, 549 and 520; forward of the last three 63, 63 and 63, 147, 147 and 122, 272, 272 and 250;
// forward of bf16 16384 x 4096 made longer ago 26.8 and 23.7.  Rows that are no whole vectors share lines: those are read through the caches.
constexpr size_t kPastGradients = (size_t)80 << 20, kPastLogits = (size_t)128 << 20;

template <typename T, int B, int E, int MODE>
void launch_rows(LossArgs g, unsigned* blocks, hipStream_t st) {
  constexpr int kRows = B == 64 ? 4 : 1;
  *blocks = blocks_for<MODE>((g.rows + kRows - 1) / kRows);
  const size_t bytes = g.rows * g.K * sizeof(T);
  g.past = bytes >= kPastLogits ? 2 : bytes >= kPastGradients;
  const bool entropy = MODE == kFwd ? g.ent_out != nullptr : MODE == kBwd ? g.dent != nullptr : g.entc != 0.f;
  auto kernel = entropy ? k_rows<T, B, E, MODE, true, false> : k_rows<T, B, E, MODE, false, false>;
  if constexpr (E > 0) {
    // gradients have to lie as the logits do, then
    if (!misaligned(g.z, 16) && g.K % Vec<T>::V == 0 && (MODE == kFwd || !g.dz || g.alike))
      kernel = entropy ? k_rows<T, B, E, MODE, true, true> : k_rows<T, B, E, MODE, false, true>;
  }
  kernel<<<*blocks, B * kRows, 0, st>>>(g);
}
template <typename T, int G, int E, int MODE>
void launch_small(const LossArgs& g, unsigned* blocks, hipStream_t st) {
  *blocks = blocks_for<MODE>((g.rows + 256 / G - 1) / (256 / G));
  k_rows_small<T, G, E, MODE><<<*blocks, 256, 0, st>>>(g);
}

// Parts of a row where few long ones are shared, 1 otherwise.  Calls one after the other, shared and by a workgroup to a row: 131072 bf16
// logits forward 9.6 and 10.8 us (1 row), 9.7 and 11.5 (128), loss 13.3 and 21.6, 24.3 and 27.8; fp32 9.5 and 15.4, 15.1 and 20.9, 13.3 and
// 31.4, 38.0 and 45.4.  With more rows every CU has one, and up to 8192 vectors a row (65536 bf16 logits) a second launch costs more than
// it gives: 32768 bf16 logits forward 9.5 and 7.0, loss 13.3 and 10.8.
constexpr size_t kFewRows = 128;
int parts_of(size_t rows, int vecs) { return rows <= kFewRows && vecs > 8 * kPart ? (vecs + kPart - 1) / kPart : 1; }

template <typename T, int MODE>
void launch_loss(const LossArgs& g, bool rows, unsigned* blocks, hipStream_t st) {
  constexpr int V = Vec<T>::V;
  if (rows) {
    // vectors of a row, counted as if it started one element past a border unless all of them start on one
    const bool even = !misaligned(g.z, 16) && g.K % V == 0;
    const int vecs = even ? g.K / V : (g.K + V - 2) / V + 1;
    if (const int parts = parts_of(g.rows, vecs); parts > 1) {
      *blocks = (unsigned)g.rows;
      if (MODE != kBwd) k_share<T><<<dim3(parts, *blocks), kPartThreads, 0, st>>>(g);
      k_rest<T, MODE><<<dim3(MODE == kFwd || !g.dz ? 1 : parts, *blocks), kPartThreads, 0, st>>>(g, parts);
      return;
    }
    // The fewest threads whose eight vectors are a row: loads under way and workgroups at other stages are many then.  (Rows of half a
    // workgroup's vectors in one of twice the threads: 4096 x 32768 bf16 forward 67 us, so 54; loss 138 and 116; 8192 x 9000 fp32 84 and 50,
    // 151 and 124.)  Rows of up to 384 classes go to a part of a wave, element by element: vectors of so short rows are mostly ends.
    if (g.K <= 8) launch_small<T, 1, 8, MODE>(g, blocks, st);
    else if (g.K <= 32) launch_small<T, 8, 4, MODE>(g, blocks, st);
    else if (g.K <= 64) launch_small<T, 8, 8, MODE>(g, blocks, st);
    else if (g.K <= 128) launch_small<T, 16, 8, MODE>(g, blocks, st);
    else if (g.K <= 256) launch_small<T, 32, 8, MODE>(g, blocks, st);
    else if (g.K <= 384) launch_small<T, 64, 8, MODE>(g, blocks, st);
    else if (vecs <= 64 * 8) launch_rows<T, 64, 8, MODE>(g, blocks, st);
    else if (vecs <= 128 * 8) launch_rows<T, 128, 8, MODE>(g, blocks, st);
    else if (vecs <= 256 * 8) launch_rows<T, 256, 8, MODE>(g, blocks, st);
    else if (vecs <= 512 * 8) launch_rows<T, 512, 8, MODE>(g, blocks, st);
    else if (vecs <= 1024 * 8) launch_rows<T, 1024, 8, MODE>(g, blocks, st);
    else if (vecs <= 1024 * 16) launch_rows<T, 1024, 16, MODE>(g, blocks, st);
    else launch_rows<T, 1024, 0, MODE>(g, blocks, st);
    return;
  }
  // four pixels a lane where all that is read of them lies on its borders (and where that leaves the chip enough lanes)
  bool four = g.P % 4 == 0 && !misaligned(g.z, 4 * sizeof(T)) && !misaligned(g.dz, 4 * sizeof(T)) && g.rows >= 4 * 65536;
  for (const void* p : {(const void*)g.labels, (const void*)g.stat, (const void*)g.ent, (const void*)g.dlogp, (const void*)g.dent, (const void*)g.old, (const void*)g.ref, (const void*)g.w,
                        (const void*)g.logp, (const void*)g.ent_out, (const void*)g.stat_out})
    four = four && !misaligned(p, 16);
  four = four && (g.per_image || !misaligned(g.adv, 16));
  if (g.K <= 16) {
    *blocks = blocks_for<MODE>((g.rows + 256 * (four ? 4 : 1) - 1) / (256 * (four ? 4 : 1)));
    auto kernel = four ? (g.K <= 4 ? k_planes<T, 4, 4, MODE> : g.K <= 6 ? k_planes<T, 4, 6, MODE> : g.K <= 8 ? k_planes<T, 4, 8, MODE>
                                                             : g.K <= 12 ? k_planes<T, 4, 12, MODE> : k_planes<T, 4, 16, MODE>)
                       : (g.K <= 8 ? k_planes<T, 1, 8, MODE> : k_planes<T, 1, 16, MODE>);
    kernel<<<*blocks, 256, 0, st>>>(g);
  } else {
    const size_t strips = (g.rows + 64 * (four ? 4 : 1) - 1) / (64 * (four ? 4 : 1));
    *blocks = blocks_for<MODE>(strips);
    int waves = 1;                     // until the chip has its fill of them, or a wave would have too few classes
    while (waves < 16 && strips * waves < 4096 && g.K / waves >= 16) waves *= 2;
    auto kernel = four ? k_planes_long<T, 4, MODE> : k_planes_long<T, 1, MODE>;
    kernel<<<*blocks, 64 * waves, waves > 1 ? waves * 3 * 64 * (four ? 4 : 1) * sizeof(float) : 0, st>>>(g);
  }
}

}  // namespace
}  // namespace rotconv
