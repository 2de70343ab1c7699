// Operators over many parameter tensors at once (see include/unettrain.h): the norm of all gradients with the factor
// that clips it, and the AdamW step with states in 32 or in 8 bits.
//
// A list is cut into chunks of one tensor each; a table in device memory names every chunk's tensor, so one launch
// covers tensors of any number and size.  The workgroups of a launch walk the chunks in steps of the grid and the last
// one to end (an atomic ticket in the control block) finishes the call: it adds the chunks' sums in a fixed order, or
// advances the step number.  Both kernels are HBM bound.
#include <hip/hip_runtime.h>

#include <algorithm>
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
constexpr int kMaxGrid = 2048;         // workgroups of a launch: eight to a CU, and so few tickets that they cost nothing
constexpr int kStaged = 2048;          // sums of chunks that the end of the norm holds in LDS

struct Row {
  float* p;
  const void* g;
  uint16_t* copy;
  uint64_t n, base;                    // elements; where its states start
  uint32_t first_chunk, chunks;
  float wd;
  uint32_t vec;                        // 1: param, gradient and copy can be read four elements at a time
};
struct Chunk {
  uint32_t row, index;
};

}  // namespace

struct train_list {
  int device = -1, count = 0, bf16 = 0;
  uint32_t chunk = 0, nchunks = 0;
  uint64_t elements = 0;
  bool trains = true;                  // every tensor has a param
  Row* rows = nullptr;                 // device
  Chunk* chunks = nullptr;             // device
};

namespace rotconv {
namespace {

typedef uint16_t us4 __attribute__((ext_vector_type(4)));

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

// Whether this workgroup is the last of its launch to come here.  Every workgroup of the grid calls it exactly once; the
// ticket is 0 again afterwards.  No fence: a release at device scope writes back an XCD's whole L2, and 2048 of them held
// the norm of 31 M gradients at 153 us and their AdamW step at 495 us.  What the last workgroup reads of the others has
// to go through memory by itself (store_shared, load_shared).
__device__ __forceinline__ bool last_of_grid(uint32_t* ticket) {
  __shared__ uint32_t mine;
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");       // this wave's stores have arrived
  __syncthreads();
  if (threadIdx.x == 0) {
    mine = __hip_atomic_fetch_add(ticket, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (mine == gridDim.x - 1) __hip_atomic_store(ticket, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  __syncthreads();
  return mine == gridDim.x - 1;
}
// one value through memory, past the caches that XCDs do not share
__device__ __forceinline__ void store_shared(double* p, double v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ double load_shared(const double* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int m = 32; m > 0; m >>= 1) v += __shfl_xor(v, m);
  return v;
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
__global__ __launch_bounds__(kThreads) void k_grad_norm(const Row* __restrict__ rows, const Chunk* __restrict__ chunks,
                                                        uint32_t nchunks, uint32_t chunk, int count, float max_norm,
                                                        float* __restrict__ norms, train_control* ctl, double* part) {
  __shared__ double red[kThreads / 64];
  __shared__ double sums[kStaged];
  for (uint32_t c = blockIdx.x; c < nchunks; c += gridDim.x) {
    const Chunk ch = chunks[c];
    const Row& r = rows[ch.row];
    const T* g = static_cast<const T*>(r.g);
    const uint64_t at = (uint64_t)ch.index * chunk;
    const uint32_t n = (uint32_t)min((uint64_t)chunk, r.n - at);
    g += at;
    double s = 0;
    const uint32_t nv = r.vec ? n / 4 : 0;
    uint32_t i = threadIdx.x;
    for (; i + 7 * kThreads < nv; i += 8 * kThreads) {       // eight loads in flight
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
    if (threadIdx.x == 0) store_shared(part + c, s);
  }
  if (!last_of_grid(&ctl->ticket[0])) return;
  const bool staged = nchunks <= (uint32_t)kStaged;
  if (staged) {
    for (uint32_t c = threadIdx.x; c < nchunks; c += kThreads) sums[c] = load_shared(part + c);
    __syncthreads();
  }
  double total = 0;
  const int lane = threadIdx.x % 16;
  for (int k = threadIdx.x / 16; k < count; k += kThreads / 16) {
    const uint32_t c0 = rows[k].first_chunk, nc = rows[k].chunks;
    double s = 0;
    for (uint32_t c = lane; c < nc; c += 16) s += staged ? sums[c0 + c] : load_shared(part + c0 + c);
#pragma unroll
    for (int m = 8; m > 0; m >>= 1) s += __shfl_xor(s, m);
    if (lane == 0) {
      if (norms) norms[k] = (float)sqrt(s);
      total += s;
    }
  }
  total = block_sum(total, red);
  if (threadIdx.x == 0) {
    const double norm = sqrt(total), r = max_norm / norm;
    ctl->norm = (float)norm;
    ctl->coef = r >= 1 ? 1.f : (float)r;
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
  // 2^(127 - byte) as fp32; the smallest are denormal
  *inv = byte == 255u ? NAN : ldexpf(1.f, 127 - (int)byte);
  return byte;
}
__device__ __forceinline__ float scale_value(uint32_t byte) { return byte == 255u ? NAN : ldexpf(1.f, (int)byte - 127); }

// largest magnitude of the eight lanes that hold a block (32 elements, four a lane), compared as bits: a NaN is above an
// infinity
__device__ __forceinline__ float block_top(const float* v) {
  uint32_t t = 0;
#pragma unroll
  for (int k = 0; k < 4; ++k) t = max(t, __float_as_uint(v[k]) & 0x7fffffffu);
#pragma unroll
  for (int m = 1; m < 8; m <<= 1) t = max(t, (uint32_t)__shfl_xor((int)t, m));
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

// 0 <= q <= 448 onto the e4m3 grid, up with the probability of the part cut off (u uniform in [0, 1)), a positive q to no
// less than the smallest code.  The grid's step is 2^(exponent - 3), 2^-9 below 2^-6.
__device__ __forceinline__ float round_up_or_down(float q, float u) {
  const uint32_t e = max(__float_as_uint(q) >> 23, 121u) - 3;
  const float step = __uint_as_float(e << 23), inv = __uint_as_float((254u - e) << 23);
  const float n = floorf(q * inv + u);
  return q > 0.f ? fmaxf(n, 1.f) * step : q;      // 0 and NaN stay
}

struct Step {                          // what a step's elements share
  float b1, c1, b2, c2;                // beta, 1 - beta
  float eps, coef, root;               // root: 1 / sqrt(1 - beta2^t)
  float rate, lr;                      // rate: lr / (1 - beta1^t)
  uint32_t key;
};

__device__ __forceinline__ double power(double b, int t) {
  double r = 1;
  for (; t > 0; t >>= 1, b *= b)
    if (t & 1) r *= b;
  return r;
}

// m and v of one element, and its parameter.  Every operation is rounded by itself: a state in 8 bits then takes the
// same code wherever this formula is evaluated in fp32.
__device__ __forceinline__ void adamw(const Step& s, float wd, float grad, float& p, float& m, float& v, float& root) {
#pragma clang fp contract(off)
  const float g = grad * s.coef;
  m = m * s.b1 + g * s.c1;
  v = v * s.b2 + g * g * s.c2;
  root = sqrtf(v);
  const float update = m / (root * s.root + s.eps);
  p = p - p * (wd * s.lr) - update * s.rate;
}

template <typename T, bool MX8>
__global__ __launch_bounds__(kThreads) void k_adamw(const Row* __restrict__ rows, const Chunk* __restrict__ chunks,
                                                    uint32_t nchunks, uint32_t chunk, train_adamw opt, void* mp, void* vp,
                                                    uint8_t* msp, uint8_t* vsp, train_control* ctl) {
  const int t = ctl->step + 1;
  const bool skip = ctl->nonfinite != 0;
  if (!skip) {
    Step s;
    s.b1 = (float)opt.beta1;
    s.c1 = (float)(1 - opt.beta1);
    s.b2 = (float)opt.beta2;
    s.c2 = (float)(1 - opt.beta2);
    s.eps = opt.eps;
    s.coef = ctl->coef;
    s.lr = ctl->lr;
    s.root = (float)(1 / sqrt(1 - power(opt.beta2, t)));
    s.rate = (float)(s.lr / (1 - power(opt.beta1, t)));
    s.key = opt.seed + (uint32_t)t * 0x9E3779B9u;
    for (uint32_t c = blockIdx.x; c < nchunks; c += gridDim.x) {
      const Chunk ch = chunks[c];
      const Row& r = rows[ch.row];
      const uint64_t at = (uint64_t)ch.index * chunk;
      const uint32_t n = (uint32_t)min((uint64_t)chunk, r.n - at);
      const uint32_t np = (n + kBlock - 1) / kBlock * kBlock;       // whole blocks: the states' padding is there
      float* p = r.p + at;
      const T* g = static_cast<const T*>(r.g) + at;
      uint16_t* copy = r.copy ? r.copy + at : nullptr;
      const uint64_t pos = r.base + at;
      // four elements a lane; a block's eight lanes are in or out together
      for (uint32_t i = 4 * threadIdx.x; i < np; i += 4 * kThreads) {
        const int have = i < n ? (int)min(4u, n - i) : 0;
        const bool whole = r.vec && have == 4;
        float pv[4] = {0, 0, 0, 0}, gv[4] = {0, 0, 0, 0}, m[4], v[4], root[4];
        if (whole) {
          load_g4(p + i, pv);
          load_g4(g + i, gv);
        } else {
          for (int k = 0; k < have; ++k) pv[k] = p[i + k], gv[k] = Elt<T>::ld(g + i + k);
        }
        const uint64_t at4 = pos + i, blk = at4 / kBlock;
        if (MX8) {
          from_e4m3_x4(reinterpret_cast<const uint32_t*>(mp)[at4 / 4], scale_value(msp[blk]), m);
          from_e4m3_x4(reinterpret_cast<const uint32_t*>(vp)[at4 / 4], scale_value(vsp[blk]), v);
#pragma unroll
          for (int k = 0; k < 4; ++k) v[k] = v[k] * v[k];
        } else {
          load_g4(static_cast<const float*>(mp) + at4, m);
          load_g4(static_cast<const float*>(vp) + at4, v);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) adamw(s, r.wd, gv[k], pv[k], m[k], v[k], root[k]);
        if (whole) {
          *reinterpret_cast<f4*>(p + i) = f4{pv[0], pv[1], pv[2], pv[3]};
          if (copy) *reinterpret_cast<us4*>(copy + i) = us4{f32_to_bf16(pv[0]), f32_to_bf16(pv[1]), f32_to_bf16(pv[2]), f32_to_bf16(pv[3])};
        } else {
          for (int k = 0; k < have; ++k) {
            p[i + k] = pv[k];
            if (copy) copy[i + k] = f32_to_bf16(pv[k]);
          }
        }
        if (MX8) {
          float inv;
          const uint32_t mb = scale_byte(block_top(m), &inv);
#pragma unroll
          for (int k = 0; k < 4; ++k) m[k] = m[k] * inv;
          reinterpret_cast<uint32_t*>(mp)[at4 / 4] = e4m3_x4(m);
          const uint32_t vb = scale_byte(block_top(root), &inv);
#pragma unroll
          for (int k = 0; k < 4; k += 2) {       // sixteen random bits an element
            const uint32_t h = mix32((uint32_t)((at4 + k) >> 1) + s.key);
            root[k] = round_up_or_down(root[k] * inv, (float)(h & 0xffffu) * 0x1p-16f);
            root[k + 1] = round_up_or_down(root[k + 1] * inv, (float)(h >> 16) * 0x1p-16f);
          }
          reinterpret_cast<uint32_t*>(vp)[at4 / 4] = e4m3_x4(root);
          if (at4 % kBlock == 0) msp[blk] = (uint8_t)mb, vsp[blk] = (uint8_t)vb;
        } else {
          *reinterpret_cast<f4*>(static_cast<float*>(mp) + at4) = f4{m[0], m[1], m[2], m[3]};
          *reinterpret_cast<f4*>(static_cast<float*>(vp) + at4) = f4{v[0], v[1], v[2], v[3]};
        }
      }
    }
  }
  // the step number and the flag change only when every workgroup has read them
  if (last_of_grid(&ctl->ticket[1]) && threadIdx.x == 0) {
    if (skip) {
      ctl->skipped += 1;
      ctl->nonfinite = 0;
    } else {
      ctl->step = t;
    }
  }
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
  // A chunk has at least 1024 elements (fewer leave lanes idle).  Beyond one chunk for each workgroup of a full launch it
  // grows to 16384 (larger ones leave CUs idle at the end), and further only where there would be more than eight times
  // the sums that the end of the norm holds in LDS.
  uint64_t chunk = 1024;
  while ((chunk < 16384 && total / chunk > (uint64_t)kMaxGrid) || total / chunk > 8ull * kStaged) chunk *= 2;
  uint64_t nchunks = 0;
  for (int k = 0; k < count; ++k) nchunks += (tensors[k].n + chunk - 1) / chunk;
  if (nchunks > 0x7fffffffu) return ROTCONV_ERR_SHAPE;
  train_list* l = nullptr;
  try {
    std::vector<Row> rows(count);
    std::vector<Chunk> chunks;
    chunks.reserve(nchunks);
    uint64_t base = 0;
    for (int k = 0; k < count; ++k) {
      const train_tensor& t = tensors[k];
      Row& r = rows[k];
      r = Row{t.param, t.grad, t.copy, t.n, base, (uint32_t)chunks.size(), (uint32_t)((t.n + chunk - 1) / chunk), t.weight_decay, 0};
      r.vec = !misaligned(t.param, 16) && !misaligned(t.grad, 4 * ge) && !misaligned(t.copy, 8);
      for (uint32_t c = 0; c < r.chunks; ++c) chunks.push_back(Chunk{(uint32_t)k, c});
      base += (t.n + kBlock - 1) / kBlock * kBlock;
    }
    l = new train_list;
    l->count = count;
    l->bf16 = grad_dtype == ROTCONV_BF16;
    l->chunk = (uint32_t)chunk;
    l->nchunks = (uint32_t)nchunks;
    l->elements = base;
    l->trains = tensors[0].param != nullptr;
    const bool ok = hipGetDevice(&l->device) == hipSuccess &&
                    hipMalloc(reinterpret_cast<void**>(&l->rows), rows.size() * sizeof(Row)) == hipSuccess &&
                    hipMalloc(reinterpret_cast<void**>(&l->chunks), chunks.size() * sizeof(Chunk)) == hipSuccess &&
                    hipMemcpy(l->rows, rows.data(), rows.size() * sizeof(Row), hipMemcpyHostToDevice) == hipSuccess &&
                    hipMemcpy(l->chunks, chunks.data(), chunks.size() * sizeof(Chunk), hipMemcpyHostToDevice) == hipSuccess;
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
  if (l->rows) (void)hipFree(l->rows);
  if (l->chunks) (void)hipFree(l->chunks);
  delete l;
  return ROTCONV_OK;
}

uint64_t train_list_elements(const train_list* l) { return l ? l->elements : 0; }
size_t train_list_workspace_bytes(const train_list* l) { return l ? (size_t)l->nchunks * sizeof(double) : 0; }

int train_control_init(train_control* control, int step, float lr, void* stream) {
  if (!control) return ROTCONV_ERR_NULL;
  if (step < 0) return ROTCONV_ERR_SHAPE;
  if (misaligned(control, 4)) return ROTCONV_ERR_UNSUPPORTED;
  k_control_init<<<1, 1, 0, static_cast<hipStream_t>(stream)>>>(control, step, lr);
  return finish();
}

int train_grad_norm(const train_list* l, float max_norm, float* norms, train_control* control, void* ws, size_t ws_bytes,
                    void* stream) {
  if (!l || !control) return ROTCONV_ERR_NULL;
  if (!(max_norm > 0.f) || !on_its_device(l) || misaligned(control, 4) || misaligned(norms, 4)) return ROTCONV_ERR_UNSUPPORTED;
  if (!ws || misaligned(ws, 8) || ws_bytes < train_list_workspace_bytes(l)) return ROTCONV_ERR_WORKSPACE;
  const unsigned grid = std::min<uint32_t>(l->nchunks, kMaxGrid);
  auto kernel = l->bf16 ? k_grad_norm<uint16_t> : k_grad_norm<float>;
  kernel<<<grid, kThreads, 0, static_cast<hipStream_t>(stream)>>>(l->rows, l->chunks, l->nchunks, l->chunk, l->count, max_norm,
                                                                  norms, control, static_cast<double*>(ws));
  return finish();
}

int train_adamw_step(const train_list* l, const train_adamw* o, void* m, void* v, uint8_t* m_scale, uint8_t* v_scale,
                     train_control* control, void* stream) {
  if (!l || !o || !m || !v || !control) return ROTCONV_ERR_NULL;
  const bool mx8 = o->state == TRAIN_STATE_MX8;
  if (mx8 ? (!m_scale || !v_scale) : (m_scale || v_scale)) return ROTCONV_ERR_NULL;
  if (!l->trains || !on_its_device(l) || (!mx8 && o->state != TRAIN_STATE_F32) || o->reserved != 0) return ROTCONV_ERR_UNSUPPORTED;
  if (!(o->beta1 >= 0 && o->beta1 < 1 && o->beta2 >= 0 && o->beta2 < 1) || !(o->eps > 0.f)) return ROTCONV_ERR_UNSUPPORTED;
  if (misaligned(m, mx8 ? 4 : 16) || misaligned(v, mx8 ? 4 : 16) || misaligned(control, 4)) return ROTCONV_ERR_UNSUPPORTED;
  const unsigned grid = std::min<uint32_t>(l->nchunks, kMaxGrid);
  auto kernel = mx8 ? (l->bf16 ? k_adamw<uint16_t, true> : k_adamw<float, true>)
                    : (l->bf16 ? k_adamw<uint16_t, false> : k_adamw<float, false>);
  kernel<<<grid, kThreads, 0, static_cast<hipStream_t>(stream)>>>(l->rows, l->chunks, l->nchunks, l->chunk, *o, m, v, m_scale,
                                                                  v_scale, control);
  return finish();
}

}  // extern "C"
