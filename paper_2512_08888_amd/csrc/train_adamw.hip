// Operators over many parameter tensors at once (see include/unettrain.h): the norm of all gradients with the factor
// that clips it, and the AdamW step with states in 32 or in 8 bits.
//
// A list is cut into chunks of one tensor each; a table in device memory says of every chunk what a workgroup needs to know,
// so one launch covers tensors of any number and size, a chunk to a workgroup.  The last workgroup to end (atomic tickets
// that the list holds) finishes the call: it adds the chunks' sums in a fixed order, or advances the step number.
// Both are HBM bound: a few operations an element.  31 M parameters (the 59 tensors of a UNet of widths 64 to 1024, fp32 gradients): the
// norm reads 124 MB in 27 us (22.7 of them the reading, 1.4 the tickets, 3.4 the end), the step reads and writes 0.93 GB with
// fp32 states in 148 us (6.3 TB/s) and 0.50 GB with 8-bit states in 85 us (5.9).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstdint>
#include <new>
#include <vector>

#include "glue_elt.h"
#include "rotconv.h"
#include "unettrain.h"

namespace {

constexpr int kBlock = 32;             // elements that share a scale; a tensor's states start on multiples of it
constexpr int kThreads = 256;
constexpr uint32_t kStepChunk = 4 * kThreads;          // elements of a step's chunk: four a lane
constexpr int kStaged = 2048;          // sums of chunks that the end of the norm holds in LDS
constexpr int kFan = 64;               // ticket counters of a launch, a cache line each
constexpr uint32_t kMostWorkgroups = (1u << 24) - 1;   // of a launch: fewer than 2^32 threads

// The chunks of a list: what a workgroup needs to know, in one read
struct NormChunk {
  const void* g;
  uint32_t n, vec;                     // elements; 1: the gradient can be read four elements at a time
};
struct StepChunk {
  float* p;
  const void* g;
  uint16_t* copy;
  uint64_t pos;                        // of the states
  float wd;
  uint32_t n, vec, reserved;           // vec: of all three
};
struct Row {                           // a tensor's chunks in the norm's cut
  uint32_t first, count;
};

}  // namespace

struct train_list {
  int device = -1, count = 0, bf16 = 0;
  uint64_t elements = 0;
  bool trains = true;                  // every tensor has a param
  void* memory = nullptr;              // device: the tables below
  uint32_t nnorm = 0, nstep = 0;
  uint32_t* tickets = nullptr;         // kFan + 1 counters, 32 words apart, 0 between calls
  StepChunk* step = nullptr;
  NormChunk* norm = nullptr;
  Row* rows = nullptr;
};

namespace rotconv {
namespace {

typedef uint16_t us4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf4 __attribute__((ext_vector_type(4)));

int finish() { return hipGetLastError() == hipSuccess ? ROTCONV_OK : ROTCONV_ERR_LAUNCH; }

__device__ __forceinline__ void load_g4(const float* g, float* v) {
  const f4 a = *reinterpret_cast<const f4*>(g);
#pragma unroll
  for (int k = 0; k < 4; ++k) v[k] = a[k];
}
__device__ __forceinline__ void load_g4(const uint16_t* g, float* v) {
  const us4 a = *reinterpret_cast<const us4*>(g);
#pragma unroll
  for (int k = 0; k < 4; ++k) v[k] = bf16_to_f32(a[k]);
}

// A step reads and writes every value once and far more of them than the caches hold: past the caches (nontemporal).
template <typename T> __device__ __forceinline__ T stream_load(const T* p) { return __builtin_nontemporal_load(p); }
template <typename T> __device__ __forceinline__ void stream_store(T* p, T v) { __builtin_nontemporal_store(v, p); }

// Whether this workgroup is the last of its launch to come here.  Every workgroup of the grid calls it exactly once; the
// tickets are 0 again afterwards.  Atomics on one counter take 12 ns each, one after the other (23 us for 1934 workgroups,
// half of the norm of 31 M gradients), so a workgroup draws from one of 64 counters, and the last of each from a further
// one.  No fence: a release at device scope writes back an XCD's whole L2 (the same norm: 153 us).  What the last workgroup
// reads of the others has to go through memory by itself (store_shared, load_shared).
__device__ __forceinline__ bool draw_last(uint32_t* ticket, uint32_t of) {
  const bool last = __hip_atomic_fetch_add(ticket, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == of - 1;
  if (last) __hip_atomic_store(ticket, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return last;
}
__device__ __forceinline__ bool last_of_grid(uint32_t* tickets) {
  __shared__ int last;
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");       // this wave's stores have arrived
  __syncthreads();
  if (threadIdx.x == 0) {
    const uint32_t mine = blockIdx.x % kFan, of = (gridDim.x - mine + kFan - 1) / kFan;
    last = draw_last(tickets + 32 * (1 + mine), of) && draw_last(tickets, min(gridDim.x, (uint32_t)kFan));
  }
  __syncthreads();
  return last;
}
// one value through memory, past the caches that XCDs do not share
__device__ __forceinline__ void store_shared(double* p, double v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ double load_shared(const double* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// A lane's value moved within its row of sixteen lanes, and sums over rows and waves: the same in all their lanes
template <int CTRL>
__device__ __forceinline__ uint32_t moved(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true);
}
constexpr int kSwap1 = 0xb1, kSwap2 = 0x4e, kMirror8 = 0x141, kMirror16 = 0x140;     // lanes 1 0 3 2; 2 3 0 1; 7 .. 0; 15 .. 0
template <int CTRL>
__device__ __forceinline__ double moved(double v) {
  const uint64_t w = __builtin_bit_cast(uint64_t, v);
  return __builtin_bit_cast(double, (uint64_t)moved<CTRL>((uint32_t)(w >> 32)) << 32 | moved<CTRL>((uint32_t)w));
}
__device__ __forceinline__ double row_sum(double v) {
  v += moved<kSwap1>(v);
  v += moved<kSwap2>(v);
  v += moved<kMirror8>(v);
  return v + moved<kMirror16>(v);
}
__device__ __forceinline__ double lane_of(double v, int lane) {
  const uint64_t w = __builtin_bit_cast(uint64_t, v);
  return __builtin_bit_cast(double, (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(w >> 32), lane) << 32 |
                                        (uint32_t)__builtin_amdgcn_readlane((int)w, lane));
}
__device__ __forceinline__ double wave_sum(double v) {
  v = row_sum(v);
  return (lane_of(v, 0) + lane_of(v, 16)) + (lane_of(v, 32) + lane_of(v, 48));
}
// sum over the workgroup, in every thread; red: one double a wave
__device__ __forceinline__ double block_sum(double v, double* red) {
  v = wave_sum(v);
  __syncthreads();
  if (threadIdx.x % 64 == 0) red[threadIdx.x / 64] = v;
  __syncthreads();
  double s = 0;
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) s += red[w];
  return s;
}

// Squares are added in 64 bits: no gradient is so large or so small that its square is lost, and a NaN or an infinity
// stays one.  The last workgroup adds the chunks' sums from LDS, sixteen lanes a tensor (a wave a tensor, each sum from
// memory where another XCD left it: 56 us for 31 M gradients, most of it here).
template <typename T>
__global__ __launch_bounds__(kThreads) void k_grad_norm(const NormChunk* __restrict__ chunks, const Row* __restrict__ rows, int count,
                                                        float max_norm, float* __restrict__ norms, train_control* ctl,
                                                        double* part, uint32_t* tickets) {
  __shared__ double red[kThreads / 64];
  __shared__ double sums[kStaged];
  {
    const NormChunk r = chunks[blockIdx.x];
    const T* g = static_cast<const T*>(r.g);
    const uint32_t n = r.n;
    double s = 0;
    const uint32_t nv = r.vec ? n / 4 : 0;
    uint32_t i = threadIdx.x;
    // Eight loads in flight, through the caches: the step reads the gradients again (31 M in fp32, norm and step together:
    // 160 us, and 166 with loads past them, though the norm alone takes 24.5 us then instead of 27.4)
    for (; i + 7 * kThreads < nv; i += 8 * kThreads) {
      float v[8][4];
#pragma unroll
      for (int u = 0; u < 8; ++u) load_g4(g + 4 * (i + u * kThreads), v[u]);
#pragma unroll
      for (int u = 0; u < 8; ++u)
#pragma unroll
        for (int k = 0; k < 4; ++k) s += (double)v[u][k] * v[u][k];
    }
    for (; i < nv; i += kThreads) {
      float v[4];
      load_g4(g + 4 * i, v);
#pragma unroll
      for (int k = 0; k < 4; ++k) s += (double)v[k] * v[k];
    }
    for (i = 4 * nv + threadIdx.x; i < n; i += kThreads) {
      const double v = Elt<T>::ld(g + i);
      s += v * v;
    }
    s = block_sum(s, red);
    if (threadIdx.x == 0) store_shared(part + blockIdx.x, s);
  }
  if (!last_of_grid(tickets)) return;
  const uint32_t nchunks = gridDim.x;
  const bool staged = nchunks <= (uint32_t)kStaged;
  if (staged) {
    constexpr int each = kStaged / kThreads;
    double v[each];
#pragma unroll
    for (int u = 0; u < each; ++u) v[u] = load_shared(part + min(threadIdx.x + u * kThreads, nchunks - 1));
#pragma unroll
    for (int u = 0; u < each; ++u) sums[threadIdx.x + u * kThreads] = v[u];
    __syncthreads();
  }
  double total = 0;
  const int lane = threadIdx.x % 16;
  constexpr int ahead = 4, apart = kThreads / 16;
  for (int k0 = threadIdx.x / 16; k0 < count; k0 += ahead * apart) {
    Row r[ahead];
#pragma unroll
    for (int u = 0; u < ahead; ++u) r[u] = rows[min(k0 + u * apart, count - 1)];
#pragma unroll
    for (int u = 0; u < ahead; ++u) {
      const int k = k0 + u * apart;
      if (k >= count) break;
      double s = 0;
      if (staged) {
#pragma unroll 8
        for (uint32_t c = lane; c < r[u].count; c += 16) s += sums[r[u].first + c];
      } else {
#pragma unroll 8
        for (uint32_t c = lane; c < r[u].count; c += 16) s += load_shared(part + r[u].first + c);
      }
      s = row_sum(s);
      if (lane == 0) {
        if (norms) norms[k] = (float)sqrt(s);
        total += s;
      }
    }
  }
  total = block_sum(total, red);
  if (threadIdx.x == 0) {
    const double norm = sqrt(total), r = max_norm / norm;
    ctl->norm = (float)norm;
    ctl->coef = r >= 1 ? 1.f : (float)r;
    ctl->clip = 1;
    ctl->nonfinite = !(norm < (double)INFINITY);
  }
}

// 32 well-mixed bits of a counter: two rounds of xor-shift and multiplication by odd constants (the golden ratio's and
// the square root of two's first 32 bits)
__device__ __forceinline__ uint32_t mix32(uint32_t x) {
  x = (x ^ (x >> 16)) * 0x9E3779B9u;
  x = (x ^ (x >> 15)) * 0x6A09E667u;
  return x ^ (x >> 16);
}

// Exponent byte (e8m0) of a block: the smallest 2^e with top <= 448 * 2^e, and 2^-e.  top: >= 0 or NaN; an infinity and
// NaN give the NaN byte, whose block reads back as NaN.
__device__ __forceinline__ uint32_t scale_byte(float top, float* inv) {
  const uint32_t bits = __float_as_uint(top);
  const int e = (int)(bits >> 23) - 135 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);
  const uint32_t byte = bits >= 0x7f800000u ? 255u : (uint32_t)(max(e, -127) + 127);
  // 2^(127 - byte): 2^-120 to 2^127, since no finite top needs a byte above 247
  *inv = byte == 255u ? NAN : ldexpf(1.f, 127 - (int)byte);
  return byte;
}
// 2^-127 (denormal in fp32) to 2^127
__device__ __forceinline__ float scale_value(uint32_t byte) { return byte == 255u ? NAN : ldexpf(1.f, (int)byte - 127); }

// largest magnitude of the eight lanes that hold a block (32 elements, four a lane), compared as bits: a NaN is above an
// infinity
__device__ __forceinline__ float block_top(const float* v) {
  uint32_t t = 0;
#pragma unroll
  for (int k = 0; k < 4; ++k) t = max(t, __float_as_uint(v[k]) & 0x7fffffffu);
  t = max(t, moved<kSwap1>(t));
  t = max(t, moved<kSwap2>(t));
  t = max(t, moved<kMirror8>(t));
  return __uint_as_float(t);
}

__device__ __forceinline__ uint32_t e4m3_x4(const float* q) {
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_pk_fp8_f32(q[0], q[1], w, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(q[2], q[3], w, true);
  return w;
}
__device__ __forceinline__ void from_e4m3_x4(uint32_t w, float scale, float* v) {
  v[0] = __builtin_amdgcn_cvt_f32_fp8(w, 0) * scale;
  v[1] = __builtin_amdgcn_cvt_f32_fp8(w, 1) * scale;
  v[2] = __builtin_amdgcn_cvt_f32_fp8(w, 2) * scale;
  v[3] = __builtin_amdgcn_cvt_f32_fp8(w, 3) * scale;
}

// Four 0 <= q <= 448 onto the e4m3 grid, up with the probability of the part cut off, a positive value (q itself may be too small
// for fp32) to no less than the smallest code.  random: 16 bits, times 16.  The twenty bits below e4m3's three of the mantissa
// take them as a carry; values whose grid has the step 2^-9 (below 2^-6) are moved to [2^-6, 2^-5) for that, where fp32 has the
// same bits for it.  rest: has the sign of what q lacks of the value that it was rounded from.  Where the bits end exactly on a
// code, that says whether the value reaches it: the code is then the one that arithmetic without rounding gives (of 31 M elements
// some 15 were not).
__device__ __forceinline__ void round_up_or_down(float* q, const uint32_t* random, const float* rest, const bool* positive) {
  uint32_t sum[4], least = ~0u;
  float shift[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    shift[k] = q[k] < 0x1p-6f ? 0x1p-6f : 0.f;
    sum[k] = __float_as_uint(q[k] + shift[k]) + random[k];
    least = min(least, sum[k] & 0xfffffu);
  }
  if (least == 0) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float lacks = q[k] - (q[k] + shift[k] - shift[k]);
      sum[k] -= (sum[k] & 0xfffffu) == 0 && (lacks < 0.f || (lacks == 0.f && rest[k] < 0.f));
    }
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float r = __uint_as_float(sum[k] & 0xfff00000u) - shift[k];
    q[k] = positive[k] ? fmaxf(r, 0x1p-9f) : 0.f;
  }
}

// The factor of a step's gradients: a clip factor that a step has used, and that nobody has written over, counts no more.
__device__ __forceinline__ float factor(const train_control& c) {
  return c.clip == 2 && __float_as_uint(c.coef) == __float_as_uint(c.spent) ? 1.f : c.coef;
}

struct Step {                          // what a step's elements share
  float b1, c1, b2, c2;                // beta, 1 - beta
  float eps, coef, root;               // root: 1 / sqrt(1 - beta2^t)
  float rate, lr;                      // rate: lr / (1 - beta1^t)
  uint32_t key;
  int t, skip;
};

__device__ __forceinline__ double power(double b, int t) {
  double r = 1;
  for (; t > 0; t >>= 1, b *= b)
    if (t & 1) r *= b;
  return r;
}

// m and v of one element, and its parameter: every operation is rounded by itself, the quotient too (31 M parameters: 148 us with the
// division and with the reciprocal instruction).
__device__ __forceinline__ void adamw(const Step& s, float wd, float grad, float& p, float& m, float& v) {
#pragma clang fp contract(off)
  const float g = grad * s.coef;
  m = m * s.b1 + g * s.c1;
  v = v * s.b2 + g * g * s.c2;
  p = p - p * (wd * s.lr) - m / (sqrtf(v) * s.root + s.eps) * s.rate;
}
// The same in 8 bits.  v holds sqrt(v); its square is formed and decayed in 64 bits, and rest tells the root's rounding (see
// round_up_or_down).  The quotient, which no state depends on, is a product with the instruction's reciprocal (2 ulp of the update).
// Bound by instructions as much as by memory (31 M parameters: 85 us, 86 with sqrtf()).  So the square is narrowed for a first
// root that one step of Newton's makes good to its last bit, with v and the gradient 2^32 times as large for room below.
// FAR: for any square, by a root in 64 bits; else for blocks whose largest sqrt(v) is from 2^-48 to 2^30, and an eps from 2^-64:
// what is too small for fp32 there has the smallest code, and does not show beside eps.
constexpr float kLift = 0x1p32f;
template <bool FAR>
__device__ __forceinline__ void adamw_mx8(const Step& s, const train_adamw& opt, float wd, float grad, float& p, float& m, float& v,
                                          float& rest, bool& positive) {
#pragma clang fp contract(off)
  const float g = grad * s.coef;
  m = m * s.b1 + g * s.c1;
  const double exact = (double)grad * (FAR ? (double)s.coef : (double)s.coef * kLift);
  const double square = fma(opt.beta2, (double)v * v, (1 - opt.beta2) * (exact * exact));
  positive = square > 0;
  float update;
  if constexpr (FAR) {
    const double root = sqrt(square);
    v = (float)root;
    rest = root > v ? 1.f : root < v ? -1.f : 0.f;
    update = m / (v * s.root + s.eps);
  } else {
    const float x = (float)square, y = __builtin_amdgcn_rsqf(fmaxf(x, FLT_MIN)), first = x * y;
    v = fmaf(fmaf(-first, first, x), 0.5f * y, first);                  // sqrt(x) to half of the last bit, and a little
    rest = (float)fma(-(double)v, (double)v, square);
    update = m * __builtin_amdgcn_rcpf(v * (s.root / kLift) + s.eps);
  }
  p = p - p * (wd * s.lr) - update * s.rate;
}

template <typename T> struct Grad4;
template <> struct Grad4<float> {
  f4 a;
  __device__ __forceinline__ void load(const float* p) { a = stream_load(reinterpret_cast<const f4*>(p)); }
  __device__ __forceinline__ void set(int k, float v) { a[k] = v; }
  __device__ __forceinline__ float get(int k) const { return a[k]; }
};
template <> struct Grad4<uint16_t> {
  us4 a;
  __device__ __forceinline__ void load(const uint16_t* p) { a = stream_load(reinterpret_cast<const us4*>(p)); }
  __device__ __forceinline__ void set(int k, uint16_t v) { a[k] = v; }
  __device__ __forceinline__ float get(int k) const { return bf16_to_f32(a[k]); }
};

// A workgroup takes a chunk, four elements a lane: all loads first, and while they are under way its first wave works out
// what the step's elements share.  The chunks are small and the workgroups many, so that what the chip reads and writes at a
// time lies close together: 31 M parameters with fp32 states take 183 us with 16384 elements to a workgroup (each then walks
// its own 64 KB of every array), 149 us with 1024.
template <typename T, bool MX8>
__global__ __launch_bounds__(kThreads) void k_adamw(const StepChunk* __restrict__ chunks, train_adamw opt,
                                                    void* mp, void* vp, uint8_t* msp, uint8_t* vsp, train_control* ctl,
                                                    uint32_t* tickets, int ends) {
  __shared__ Step shared;
  const uint32_t i = 4 * threadIdx.x;
  const StepChunk r = chunks[blockIdx.x];
  const T* g = static_cast<const T*>(r.g);
  const int have = i < r.n ? (int)min(4u, r.n - i) : 0;
  const bool whole = r.vec && have == 4;
  const bool inside = i < (r.n + kBlock - 1) / kBlock * kBlock;       // whole blocks, that is eight lanes together
  const uint64_t at = r.pos + i;
  f4 pv = {0.f, 0.f, 0.f, 0.f}, fm, fv;
  Grad4<T> gv = {};
  uint32_t cm, cv, sm, sv;
  if (whole) {
    pv = stream_load(reinterpret_cast<const f4*>(r.p + i));
    gv.load(g + i);
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (k < have) pv[k] = r.p[i + k], gv.set(k, g[i + k]);
  }
  if (inside) {
    if constexpr (MX8) {
      cm = stream_load(reinterpret_cast<const uint32_t*>(mp) + at / 4);
      cv = stream_load(reinterpret_cast<const uint32_t*>(vp) + at / 4);
      sm = msp[at / kBlock];
      sv = vsp[at / kBlock];
    } else {
      fm = stream_load(reinterpret_cast<const f4*>(static_cast<const float*>(mp) + at));
      fv = stream_load(reinterpret_cast<const f4*>(static_cast<const float*>(vp) + at));
    }
  }
  if (threadIdx.x < 64) {              // even lanes for beta1, odd ones for beta2
    const int t = ctl->step + 1;
    const float lr = ctl->lr;
    const float left = (float)(1 - power(threadIdx.x % 2 ? opt.beta2 : opt.beta1, t));
    const float scaled = threadIdx.x % 2 ? 1.f / sqrtf(left) : lr / left;
    const float root = __shfl(scaled, 1);
    if (threadIdx.x == 0)
      shared = Step{(float)opt.beta1, (float)(1 - opt.beta1), (float)opt.beta2, (float)(1 - opt.beta2), opt.eps, factor(*ctl), root, scaled, lr,
                    opt.seed + (uint32_t)t * 0x9E3779B9u, t, ctl->nonfinite};
  }
  __syncthreads();
  const Step s = shared;
  // The first lane alone reads the control block, and has done so: who draws the last ticket knows that nobody will again.
  auto end = [&] {
    if (!ends || threadIdx.x != 0) return;             // (more launches of this step follow)
    const uint32_t mine = blockIdx.x % kFan, of = (gridDim.x - mine + kFan - 1) / kFan;
    if (!draw_last(tickets + 32 * (1 + mine), of) || !draw_last(tickets, min(gridDim.x, (uint32_t)kFan))) return;
    if (s.skip) {
      ctl->skipped += 1, ctl->nonfinite = 0;
      ctl->coef = 1.f, ctl->clip = 0;                  // of a norm that was not finite
      return;
    }
    ctl->step = s.t;
    if (ctl->clip == 1) ctl->clip = 2, ctl->spent = ctl->coef;
  };
  if (s.skip || !inside) {             // (the first lane is inside)
    end();
    return;
  }
  float p[4];
  if constexpr (MX8) {
    float m[4], v[4], rest[4], inv;
    bool positive[4];
    from_e4m3_x4(cm, scale_value(sm), m);
    from_e4m3_x4(cv, scale_value(sv) * kLift, v);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      p[k] = pv[k];
      adamw_mx8<false>(s, opt, r.wd, gv.get(k), p[k], m[k], v[k], rest[k], positive[k]);
    }
    float top = block_top(v);
    float lower = 1.f / kLift;
    if (!(top >= 0x1p-48f * kLift && top <= 0x1p30f * kLift) || s.eps < 0x1p-64f) {       // the lanes of a block go together
      lower = 1.f;
      from_e4m3_x4(cm, scale_value(sm), m);
      from_e4m3_x4(cv, scale_value(sv), v);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        p[k] = pv[k];
        adamw_mx8<true>(s, opt, r.wd, gv.get(k), p[k], m[k], v[k], rest[k], positive[k]);
      }
      top = block_top(v);
    }
    const uint32_t vb = scale_byte(top * lower, &inv);
    inv *= lower;
    uint32_t random[4];                    // sixteen random bits an element
#pragma unroll
    for (int k = 0; k < 4; k += 2) {
      const uint32_t h = mix32((uint32_t)((at + k) >> 1) + s.key);
      random[k] = h << 4 & 0xffff0u, random[k + 1] = h >> 12 & 0xffff0u;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = v[k] * inv;
    round_up_or_down(v, random, rest, positive);
    stream_store(reinterpret_cast<uint32_t*>(vp) + at / 4, e4m3_x4(v));
    const uint32_t mb = scale_byte(block_top(m), &inv);
#pragma unroll
    for (int k = 0; k < 4; ++k) m[k] = m[k] * inv;
    stream_store(reinterpret_cast<uint32_t*>(mp) + at / 4, e4m3_x4(m));
    if (at % kBlock == 0) msp[at / kBlock] = (uint8_t)mb, vsp[at / kBlock] = (uint8_t)vb;
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      float m = fm[k], v = fv[k];
      p[k] = pv[k];
      adamw(s, r.wd, gv.get(k), p[k], m, v);
      fm[k] = m, fv[k] = v;
    }
    stream_store(reinterpret_cast<f4*>(static_cast<float*>(mp) + at), fm);
    stream_store(reinterpret_cast<f4*>(static_cast<float*>(vp) + at), fv);
  }
  if (whole) {
    stream_store(reinterpret_cast<f4*>(r.p + i), f4{p[0], p[1], p[2], p[3]});
    if (r.copy)
      stream_store(reinterpret_cast<us4*>(r.copy + i),
                   __builtin_bit_cast(us4, __builtin_convertvector(f4{p[0], p[1], p[2], p[3]}, bf4)));
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (k < have) {
        r.p[i + k] = p[k];
        if (r.copy) r.copy[i + k] = f32_to_bf16(p[k]);
      }
  }
  end();
}

__global__ void k_control_init(train_control* ctl, int step, float lr) {
  train_control c = {};
  c.step = step;
  c.lr = lr;
  c.coef = 1.f;
  *ctl = c;
}

bool on_its_device(const train_list* l) {
  int dev = 0;
  return hipGetDevice(&dev) == hipSuccess && dev == l->device;
}
bool misaligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }

}  // namespace
}  // namespace rotconv

using namespace rotconv;

extern "C" {

int train_list_create(const train_tensor* tensors, int count, int grad_dtype, train_list** out) {
  if (!tensors || !out) return ROTCONV_ERR_NULL;
  if (count < 1) return ROTCONV_ERR_SHAPE;
  if (grad_dtype != ROTCONV_F32 && grad_dtype != ROTCONV_BF16) return ROTCONV_ERR_UNSUPPORTED;
  const uintptr_t ge = grad_dtype == ROTCONV_BF16 ? 2 : 4;
  uint64_t total = 0;
  for (int k = 0; k < count; ++k) {
    const train_tensor& t = tensors[k];
    if (!t.grad || (!t.param != !tensors[0].param) || (t.copy && !t.param)) return ROTCONV_ERR_NULL;
    if (t.n < 1 || t.n > (1ull << 40) || total > (1ull << 44)) return ROTCONV_ERR_SHAPE;
    if (!(t.weight_decay >= 0.f) || t.reserved != 0 || misaligned(t.param, 4) || misaligned(t.grad, ge) || misaligned(t.copy, 2))
      return ROTCONV_ERR_UNSUPPORTED;
    total += (t.n + kBlock - 1) / kBlock * kBlock;
  }
  // The norm's chunks: from 1024 elements (fewer leave lanes idle) to 16384, then larger only where there would be more
  // sums than eight times what its end holds in LDS.
  uint64_t size = 1024;
  while ((size < 16384 && total / size > (uint64_t)kStaged) || total / size > 8ull * kStaged) size *= 2;
  uint64_t nnorm = 0, nstep = 0;
  for (int k = 0; k < count; ++k) nnorm += (tensors[k].n + size - 1) / size, nstep += (tensors[k].n + kStepChunk - 1) / kStepChunk;
  // The norm is one launch, at least a workgroup a tensor; a step may be several.
  if (nnorm > kMostWorkgroups || nstep > 0x7fffffffu) return ROTCONV_ERR_SHAPE;
  train_list* l = nullptr;
  try {
    std::vector<Row> rows(count);
    std::vector<NormChunk> norm;
    std::vector<StepChunk> step;
    norm.reserve(nnorm);
    if (tensors[0].param) step.reserve(nstep);
    uint64_t base = 0;
    for (int k = 0; k < count; ++k) {
      const train_tensor& t = tensors[k];
      const char* g = static_cast<const char*>(t.grad);
      rows[k] = Row{(uint32_t)norm.size(), (uint32_t)((t.n + size - 1) / size)};
      for (uint64_t at = 0; at < t.n; at += size)
        norm.push_back(NormChunk{g + at * ge, (uint32_t)std::min(size, t.n - at), misaligned(t.grad, 4 * ge) ? 0u : 1u});
      const uint32_t vec = !misaligned(t.param, 16) && !misaligned(t.grad, 4 * ge) && !misaligned(t.copy, 8);
      for (uint64_t at = 0; t.param && at < t.n; at += kStepChunk)
        step.push_back(StepChunk{t.param + at, g + at * ge, t.copy ? t.copy + at : nullptr, base + at, t.weight_decay,
                                 (uint32_t)std::min<uint64_t>(kStepChunk, t.n - at), vec, 0});
      base += (t.n + kBlock - 1) / kBlock * kBlock;
    }
    l = new train_list;
    l->count = count;
    l->bf16 = grad_dtype == ROTCONV_BF16;
    l->elements = base;
    l->trains = tensors[0].param != nullptr;
    l->nnorm = (uint32_t)norm.size();
    l->nstep = (uint32_t)step.size();
    const std::vector<uint32_t> tickets((kFan + 1) * 32, 0);
    const size_t ticket_bytes = tickets.size() * sizeof(uint32_t), step_bytes = step.size() * sizeof(StepChunk);
    const size_t norm_bytes = norm.size() * sizeof(NormChunk), row_bytes = rows.size() * sizeof(Row);
    bool ok = hipGetDevice(&l->device) == hipSuccess &&
              hipMalloc(&l->memory, ticket_bytes + step_bytes + norm_bytes + row_bytes) == hipSuccess;
    if (ok) {
      char* p = static_cast<char*>(l->memory);
      auto put = [&](const void* from, size_t bytes) {
        void* to = p;
        ok = ok && (bytes == 0 || hipMemcpy(to, from, bytes, hipMemcpyHostToDevice) == hipSuccess);
        p += bytes;
        return to;
      };
      l->tickets = static_cast<uint32_t*>(put(tickets.data(), ticket_bytes));
      l->step = static_cast<StepChunk*>(put(step.data(), step_bytes));
      l->norm = static_cast<NormChunk*>(put(norm.data(), norm_bytes));
      l->rows = static_cast<Row*>(put(rows.data(), row_bytes));
    }
    if (!ok) {
      (void)hipGetLastError();
      train_list_destroy(l);
      return ROTCONV_ERR_LAUNCH;
    }
  } catch (const std::exception&) {
    train_list_destroy(l);
    return ROTCONV_ERR_LAUNCH;
  }
  *out = l;
  return ROTCONV_OK;
}

int train_list_destroy(train_list* l) {
  if (!l) return ROTCONV_OK;
  if (l->memory) (void)hipFree(l->memory);
  delete l;
  return ROTCONV_OK;
}

uint64_t train_list_elements(const train_list* l) { return l ? l->elements : 0; }
size_t train_list_workspace_bytes(const train_list* l) { return l ? (size_t)l->nnorm * sizeof(double) : 0; }

int train_control_init(train_control* control, int step, float lr, void* stream) {
  if (!control) return ROTCONV_ERR_NULL;
  if (step < 0 || step == INT32_MAX) return ROTCONV_ERR_SHAPE;         // (the next step's number is an int32_t too)
  if (misaligned(control, 4)) return ROTCONV_ERR_UNSUPPORTED;
  k_control_init<<<1, 1, 0, static_cast<hipStream_t>(stream)>>>(control, step, lr);
  return finish();
}

int train_grad_norm(const train_list* l, float max_norm, float* norms, train_control* control, void* ws, size_t ws_bytes,
                    void* stream) {
  if (!l || !control) return ROTCONV_ERR_NULL;
  if (!(max_norm > 0.f) || !on_its_device(l) || misaligned(control, 4) || misaligned(norms, 4)) return ROTCONV_ERR_UNSUPPORTED;
  if (!ws || misaligned(ws, 8) || ws_bytes < train_list_workspace_bytes(l)) return ROTCONV_ERR_WORKSPACE;
  auto kernel = l->bf16 ? k_grad_norm<uint16_t> : k_grad_norm<float>;
  kernel<<<l->nnorm, kThreads, 0, static_cast<hipStream_t>(stream)>>>(l->norm, l->rows, l->count, max_norm, norms, control,
                                                                      static_cast<double*>(ws), l->tickets);
  return finish();
}

int train_adamw_step(const train_list* l, const train_adamw* o, void* m, void* v, uint8_t* m_scale, uint8_t* v_scale,
                     train_control* control, void* stream) {
  if (!l || !o || !m || !v || !control) return ROTCONV_ERR_NULL;
  const bool mx8 = o->state == TRAIN_STATE_MX8;
  if (mx8 ? (!m_scale || !v_scale) : (m_scale || v_scale)) return ROTCONV_ERR_NULL;
  if (!l->trains || !on_its_device(l) || (!mx8 && o->state != TRAIN_STATE_F32) || o->reserved != 0) return ROTCONV_ERR_UNSUPPORTED;
  if (!(o->beta1 >= 0 && o->beta1 < 1 && o->beta2 >= 0 && o->beta2 < 1) || !(o->eps >= FLT_MIN)) return ROTCONV_ERR_UNSUPPORTED;
  if (misaligned(m, mx8 ? 4 : 16) || misaligned(v, mx8 ? 4 : 16) || misaligned(control, 4)) return ROTCONV_ERR_UNSUPPORTED;
  // LDS that nobody uses keeps five workgroups on a CU where eight would fit: with fp32 states their streams then get in one
  // another's way less (31 M parameters: 163 us with eight, 149 us with five or four); 8-bit states need all eight to keep
  // enough bytes under way (89 us with eight, 112 us with five, when the whole took that long).
  const size_t lds = mx8 ? 0 : 32000;
  auto kernel = mx8 ? (l->bf16 ? k_adamw<uint16_t, true> : k_adamw<float, true>) : (l->bf16 ? k_adamw<uint16_t, false> : k_adamw<float, false>);
  for (uint32_t done = 0; done < l->nstep;) {
    const uint32_t now = std::min(l->nstep - done, kMostWorkgroups);
    kernel<<<now, kThreads, lds, static_cast<hipStream_t>(stream)>>>(l->step + done, *o, m, v, m_scale, v_scale, control, l->tickets,
                                                                     done + now == l->nstep);
    done += now;
  }
  return finish();
}

}  // extern "C"
