// Muon's step over many matrices (see include/unettrain.h): momentum, Newton-Schulz products, update.
//
// Every matrix is held with its shorter side n as rows (transposed where it is tall), X [n][m].  An iteration is three products:
//     A = X X^T (symmetric)      B = b A + c A^2 (symmetric)      X <- a X + B X
// One launch makes a step of all matrices: a table in device memory gives every workgroup its matrix and tile.
//
// Numbers.  The operands of the matrix instructions are fp16: everything here is bounded, so its range can be used in full
// with fixed powers of two, and it has three more bits than bf16 at the same rate.  |X|_F = 1 at first, and p(x) = a x + b x^3 + c x^5 maps
// [0, 1.21] into [0, 1.21]: singular values of X stay below 1.21, eigenvalues of A below 1.46, those of B within [-2.81, 0], and no
// element is larger than the largest of them.  X and A are held times 2^15, B times 2^14.  Two things keep the digits that matter:
//   - X is held as the sum of two fp16 numbers.  The products read the upper one; the term a X, by which small singular
//     values grow 3.4-fold an iteration, takes both.  (Else the upper's rounding grows with them: momenta of rank 16 beside noise
//     of a tenth come out 1e-2 off, with it 2e-4.)
//   - The diagonals of A and of the polynomial are kept in fp32 and applied by themselves: rows of gradients are nearly
//     orthogonal, so that the diagonals are most of them, and their rounding would shift all singular values together (random
//     256 x 1024: 1.4e-3 off, without it 5e-4).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstdint>
#include <new>
#include <vector>

#include "glue_elt.h"
#include "rotconv.h"
#include "train_control.h"
#include "unettrain.h"

namespace {

constexpr int kThreads = 256;
constexpr int kPad = 32;               // elements: a stack's momentum starts on a multiple
constexpr int kTile = 128;             // of the products
constexpr int kDepth = 64;             // elements that a step of a product adds up
constexpr uint32_t kChunk = 4096;      // elements of the momentum's pass, to a workgroup
constexpr int kTurn = 64;              // edge of the tiles by which X is first written
constexpr uint32_t kMostWorkgroups = (1u << 24) - 1;

struct Matrix {
  float* p;
  const void* g;
  uint16_t* copy;
  uint64_t pos;                        // of the momentum
  uint32_t rows, cols, n, m;           // n = min, m = max
  uint32_t ldn, ldm;                   // n, m up to a multiple of kDepth; what is between is 0
  uint32_t tall, vec;                  // vec: gradient and momentum can be read four elements at a time
  float wd, scale;
  uint32_t first, chunks;              // in the momentum's pass
  // byte offsets in the workspace: X's upper parts before and after an iteration, its lower part, A, B; the diagonals
  uint64_t x[2], low, a, b, da, db;
};
struct Tile {
  uint32_t matrix, i, j;
};

}  // namespace

struct train_matrices {
  int device = -1, bf16 = 0;
  uint64_t elements = 0;
  size_t workspace = 0, inverse = 0, sums = 0;         // byte offsets: 1 / |u| of every matrix, the chunks' sums
  void* memory = nullptr;
  Matrix* matrices = nullptr;
  Tile *chunk = nullptr, *turn = nullptr, *square = nullptr, *wide = nullptr;
  uint32_t count = 0, nchunk = 0, nturn = 0, nsquare = 0, nwide = 0;
};

namespace rotconv {
namespace {

typedef _Float16 half;
typedef half h2 __attribute__((ext_vector_type(2)));
typedef half h4 __attribute__((ext_vector_type(4)));
typedef half h8 __attribute__((ext_vector_type(8)));
typedef float f16v __attribute__((ext_vector_type(16)));
typedef uint16_t us4 __attribute__((ext_vector_type(4)));

constexpr float kA = 3.4445f, kB = -4.7750f, kC = 2.0315f;
constexpr float kHeld = 0x1p15f;       // X and A as they are held; B: half of that
constexpr float kLow = 0x1p11f;        // the lower part beside the upper

__device__ __forceinline__ double lanes_sum(double v) {
#pragma unroll
  for (int k = 32; k > 0; k /= 2) v += __shfl_xor(v, k);
  return v;
}

// momentum and u of one element
__device__ __forceinline__ float next_momentum(float m, float g, float mu) {
#pragma clang fp contract(off)
  return m * mu + g;
}
__device__ __forceinline__ float direction(float m, float g, float mu, int nesterov) {
#pragma clang fp contract(off)
  return nesterov ? g + m * mu : m;
}

// momentum <- mu momentum + g, and the sum of u's squares of every chunk, in 64 bits
template <typename T>
__global__ __launch_bounds__(kThreads) void k_momentum(const Matrix* __restrict__ mats, const Tile* __restrict__ chunks, train_muon opt,
                                                       float* __restrict__ momentum, const train_control* __restrict__ ctl, double* sums) {
  __shared__ double red[kThreads / 64];
  if (ctl->nonfinite) return;
  const Tile c = chunks[blockIdx.x];
  const Matrix& x = mats[c.matrix];
  const uint64_t from = (uint64_t)c.i * kChunk, size = (uint64_t)x.rows * x.cols;
  const uint32_t n = (uint32_t)min((uint64_t)kChunk, size - from);
  const T* g = static_cast<const T*>(x.g) + from;
  float* m = momentum + x.pos + from;
  const float coef = factor(*ctl), mu = opt.momentum;
  double s = 0;
  const uint32_t nv = x.vec ? n / 4 : 0;
  for (uint32_t i = threadIdx.x; i < nv; i += kThreads) {
    f4 mv = *reinterpret_cast<const f4*>(m + 4 * i);
    float gv[4];
    if constexpr (sizeof(T) == 4) Elt<T>::ldv(g + 4 * i, gv);
    else Elt<T>::ldh(g + 4 * i, gv);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float gk = gv[k] * coef;
      mv[k] = next_momentum(mv[k], gk, mu);
      const double u = direction(mv[k], gk, mu, opt.nesterov);
      s += u * u;
    }
    *reinterpret_cast<f4*>(m + 4 * i) = mv;
  }
  for (uint32_t i = 4 * nv + threadIdx.x; i < n; i += kThreads) {
    const float gk = Elt<T>::ld(g + i) * coef;
    const float mk = m[i] = next_momentum(m[i], gk, mu);
    const double u = direction(mk, gk, mu, opt.nesterov);
    s += u * u;
  }
  s = lanes_sum(s);
  if (threadIdx.x % 64 == 0) red[threadIdx.x / 64] = s;
  __syncthreads();
  if (threadIdx.x == 0) sums[blockIdx.x] = red[0] + red[1] + red[2] + red[3];
}

// 1 / (|u| + eps) of every matrix, a wave each
__global__ __launch_bounds__(64) void k_inverse_norm(const Matrix* __restrict__ mats, float eps, const double* __restrict__ sums,
                                                     float* __restrict__ inverse) {
  const Matrix& x = mats[blockIdx.x];
  double s = 0;
  for (uint32_t c = threadIdx.x; c < x.chunks; c += 64) s += sums[x.first + c];
  s = lanes_sum(s);
  if (threadIdx.x == 0) inverse[blockIdx.x] = (float)(1.0 / (sqrt(s) + (double)eps));
}

// v = X times 2^15, as two fp16 numbers
__device__ __forceinline__ void split(float v, half* upper, half* lower) {
  const half u = (half)v;
  *upper = u;
  *lower = (half)((v - (float)u) * kLow);
}
__device__ __forceinline__ float joined(half upper, half lower) { return (float)upper + (float)lower * (1.f / kLow); }

// X from u, tiles of 64 x 64 of the matrix as it lies in memory; the columns up to ldm are 0 in both of X's buffers
template <typename T>
__global__ __launch_bounds__(kThreads) void k_start(const Matrix* __restrict__ mats, const Tile* __restrict__ tiles, train_muon opt,
                                                    const float* __restrict__ momentum, const train_control* __restrict__ ctl,
                                                    const float* __restrict__ inverse, char* ws) {
  __shared__ float turned[kTurn][kTurn + 1];
  if (ctl->nonfinite) return;
  const Tile t = tiles[blockIdx.x];
  const Matrix& x = mats[t.matrix];
  const float coef = factor(*ctl), mu = opt.momentum, scale = inverse[t.matrix] * kHeld;
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const T* g = static_cast<const T*>(x.g);
  const float* m = momentum + x.pos;
  for (int k = wave; k < kTurn; k += 4) {
    const uint32_t r = t.i * kTurn + k, c = t.j * kTurn + lane;
    float v = 0.f;
    if (r < x.rows && c < x.cols) {
      const uint64_t at = (uint64_t)r * x.cols + c;
      v = direction(m[at], Elt<T>::ld(g + at) * coef, mu, opt.nesterov) * scale;
    }
    turned[k][lane] = v;
  }
  __syncthreads();
  half *upper = reinterpret_cast<half*>(ws + x.x[0]), *other = reinterpret_cast<half*>(ws + x.x[1]), *lower = reinterpret_cast<half*>(ws + x.low);
  const uint32_t ti = x.tall ? t.j : t.i, tj = x.tall ? t.i : t.j;
  for (int k = wave; k < kTurn; k += 4) {
    const uint32_t i = ti * kTurn + k, j = tj * kTurn + lane;
    if (i >= x.n || j >= x.ldm) continue;
    const uint64_t at = (uint64_t)i * x.ldm + j;
    half u, l;
    split(x.tall ? turned[lane][k] : turned[k][lane], &u, &l);
    upper[at] = u, lower[at] = l;
    if (j >= x.m) other[at] = (half)0.f;
  }
}

enum Product { kGram, kPoly, kApply, kLast };

// One tile of 128 x 128 of a product, four waves of 64 x 64.
//   kGram   A = X X^T      kPoly   B = b A + c A^2      (tiles on and above the diagonal; the others are their mirror images)
//   kApply  X <- a X + B X      kLast   the same, into the parameters
template <int KIND>
__global__ __launch_bounds__(kThreads) void k_product(const Matrix* __restrict__ mats, const Tile* __restrict__ tiles, char* ws, int from,
                                                      const train_control* __restrict__ ctl) {
  __shared__ __attribute__((aligned(16))) half sa[kTile * kDepth];
  __shared__ __attribute__((aligned(16))) half sb[kTile * kDepth];
  if (ctl->nonfinite) return;
  const Tile t = tiles[blockIdx.x];
  const Matrix& x = mats[t.matrix];
  const uint32_t n = x.n, ldn = x.ldn, ldm = x.ldm;
  const half* X = reinterpret_cast<const half*>(ws + x.x[from]);
  const half* A = reinterpret_cast<const half*>(ws + x.a);
  const half* left = KIND == kGram ? X : KIND == kPoly ? A : reinterpret_cast<const half*>(ws + x.b);
  const half* right = KIND == kPoly ? A : X;
  const uint32_t ldl = KIND == kGram ? ldm : ldn, ldr = KIND == kPoly ? ldn : ldm, depth = KIND == kGram ? ldm : ldn;
  const int tid = threadIdx.x, lane = tid % 64, wr = tid / 128, wc = tid / 64 % 2;
  f16v acc[2][2] = {};
  for (uint32_t k0 = 0; k0 < depth; k0 += kDepth) {
    h8 va[4], vb[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const uint32_t r = tid / 8 + 32 * u, c = tid % 8;
      va[u] = *reinterpret_cast<const h8*>(left + (uint64_t)min(t.i * kTile + r, n - 1) * ldl + k0 + 8 * c);
      if constexpr (KIND == kGram || KIND == kPoly) {
        vb[u] = *reinterpret_cast<const h8*>(right + (uint64_t)min(t.j * kTile + r, n - 1) * ldr + k0 + 8 * c);
      } else {
        const uint32_t k = tid / 16 + 16 * u, j = min(t.j * kTile + 8 * (tid % 16), ldm - 8);
        vb[u] = *reinterpret_cast<const h8*>(right + (uint64_t)min(k0 + k, n - 1) * ldr + j);
      }
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int r = tid / 8 + 32 * u, c = tid % 8;
      *reinterpret_cast<h8*>(sa + r * kDepth + (c ^ (r & 7)) * 8) = va[u];
      if constexpr (KIND == kGram || KIND == kPoly) {
        *reinterpret_cast<h8*>(sb + r * kDepth + (c ^ (r & 7)) * 8) = vb[u];
      } else {
        const int k = tid / 16 + 16 * u;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int j = 8 * (tid % 16) + e;
          sb[j * kDepth + ((k / 8) ^ (j & 7)) * 8 + k % 8] = vb[u][e];
        }
      }
    }
    __syncthreads();
#pragma unroll
    for (int kk = 0; kk < kDepth / 16; ++kk) {
      h8 fa[2], fb[2];
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const int ra = wr * 64 + q * 32 + lane % 32, rb = wc * 64 + q * 32 + lane % 32, c = kk * 2 + lane / 32;
        fa[q] = *reinterpret_cast<const h8*>(sa + ra * kDepth + (c ^ (ra & 7)) * 8);
        fb[q] = *reinterpret_cast<const h8*>(sb + rb * kDepth + (c ^ (rb & 7)) * 8);
      }
#pragma unroll
      for (int p = 0; p < 2; ++p)
#pragma unroll
        for (int q = 0; q < 2; ++q) acc[p][q] = __builtin_amdgcn_mfma_f32_32x32x16_f16(fa[p], fb[q], acc[p][q], 0, 0, 0);
    }
  }
  float* da = reinterpret_cast<float*>(ws + x.da);
  float* db = reinterpret_cast<float*>(ws + x.db);
  const float lr = KIND == kLast ? ctl->lr : 0.f;
#pragma unroll
  for (int p = 0; p < 2; ++p)
#pragma unroll
    for (int q = 0; q < 2; ++q)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const uint32_t i = t.i * kTile + wr * 64 + p * 32 + 8 * (e / 4) + 4 * (lane / 32) + e % 4;
        const uint32_t j = t.j * kTile + wc * 64 + q * 32 + lane % 32;
        const float v = acc[p][q][e];
        if constexpr (KIND == kGram || KIND == kPoly) {
          half* out = reinterpret_cast<half*>(ws + (KIND == kGram ? x.a : x.b));
          float w = 0.f;
          if (i < n && j < n) {
            if constexpr (KIND == kGram) {
              w = v * (1.f / kHeld);
              if (i == j) da[i] = v * (1.f / (kHeld * kHeld));
            } else {
              const float held = (float)A[(uint64_t)i * ldn + j], di = da[i], dj = da[j];
              w = held * (0.5f * (kB + kC * (di + dj))) + v * (0.5f * kC / kHeld);
              if (i == j) db[i] = kA + di * (kB + kC * di) + kC * (v * (1.f / (kHeld * kHeld)));
            }
            if (i == j) w = 0.f;
          }
          if (i < n && j < ldn) out[(uint64_t)i * ldn + j] = (half)w;
          if (t.i != t.j && j < n && i < ldn) out[(uint64_t)j * ldn + i] = (half)w;
        } else {
          if (i >= n || j >= x.m) continue;
          const uint64_t at = (uint64_t)i * ldm + j;
          half* low = reinterpret_cast<half*>(ws + x.low);
          const float w = db[i] * joined(X[at], low[at]) + v * (2.f / kHeld);
          if constexpr (KIND == kApply) {
            half u, l;
            split(w, &u, &l);
            reinterpret_cast<half*>(ws + x.x[1 - from])[at] = u;
            low[at] = l;
          } else {
            const uint64_t to = x.tall ? (uint64_t)j * x.cols + i : (uint64_t)i * x.cols + j;
            float r = x.p[to];
            r = r - r * (x.wd * lr) - w * (x.scale * lr / kHeld);
            x.p[to] = r;
            if (x.copy) x.copy[to] = f32_to_bf16(r);
          }
        }
      }
}

__global__ void k_step_end(train_control* ctl) { end_step(ctl, ctl->nonfinite, ctl->step + 1); }

int finish() { return hipGetLastError() == hipSuccess ? ROTCONV_OK : ROTCONV_ERR_LAUNCH; }
bool misaligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }
uint64_t up(uint64_t n, uint64_t to) { return (n + to - 1) / to * to; }

}  // namespace
}  // namespace rotconv

using namespace rotconv;

extern "C" {

int train_matrices_create(const train_matrix* matrices, int count, int grad_dtype, train_matrices** out) {
  if (!matrices || !out) return ROTCONV_ERR_NULL;
  if (count < 1) return ROTCONV_ERR_SHAPE;
  if (grad_dtype != ROTCONV_F32 && grad_dtype != ROTCONV_BF16) return ROTCONV_ERR_UNSUPPORTED;
  const uintptr_t ge = grad_dtype == ROTCONV_BF16 ? 2 : 4;
  uint64_t nchunk = 0, nturn = 0, nsquare = 0, nwide = 0, all = 0;
  for (int k = 0; k < count; ++k) {
    const train_matrix& t = matrices[k];
    if (!t.param || !t.grad) return ROTCONV_ERR_NULL;
    if (t.count < 1 || t.rows < 1 || t.cols < 1) return ROTCONV_ERR_SHAPE;
    const uint64_t n = std::min(t.rows, t.cols), m = std::max(t.rows, t.cols), c = t.count;
    if (n > 32768 || m > (1u << 24) || c > (1ull << 40) / (n * m)) return ROTCONV_ERR_SHAPE;
    if (!(t.weight_decay >= 0.f && t.weight_decay <= FLT_MAX) || !(std::fabs(t.scale) <= FLT_MAX) || t.reserved != 0 || misaligned(t.param, 4) ||
        misaligned(t.grad, ge) || misaligned(t.copy, 2))
      return ROTCONV_ERR_UNSUPPORTED;
    const uint64_t tn = (n + kTile - 1) / kTile, tm = (m + kTile - 1) / kTile;
    nchunk += c * ((n * m + kChunk - 1) / kChunk), nturn += c * (up(n, kTurn) / kTurn) * (up(m, kTurn) / kTurn);
    nsquare += c * tn * (tn + 1) / 2, nwide += c * tn * tm, all += c;
    if (all > 65535 || std::max(std::max(nchunk, nturn), std::max(nsquare, nwide)) > kMostWorkgroups) return ROTCONV_ERR_SHAPE;
  }
  train_matrices* l = nullptr;
  try {
    std::vector<Matrix> mats;
    std::vector<Tile> chunk, turn, square, wide;
    mats.reserve(all), chunk.reserve(nchunk), turn.reserve(nturn), square.reserve(nsquare), wide.reserve(nwide);
    uint64_t base = 0, at = up(all * sizeof(float), 256);
    const uint64_t sums = at;
    at = up(at + nchunk * sizeof(double), 256);
    auto room = [&](uint64_t bytes) {
      const uint64_t here = at;
      at = up(at + bytes, 256);
      return here;
    };
    for (int k = 0; k < count; ++k) {
      const train_matrix& t = matrices[k];
      const uint64_t size = (uint64_t)t.rows * t.cols;
      for (int i = 0; i < t.count; ++i) {
        Matrix x = {};
        x.p = t.param + i * size;
        x.g = static_cast<const char*>(t.grad) + i * size * ge;
        x.copy = t.copy ? t.copy + i * size : nullptr;
        x.pos = base + i * size;
        x.rows = t.rows, x.cols = t.cols, x.tall = t.rows > t.cols;
        x.n = std::min(t.rows, t.cols), x.m = std::max(t.rows, t.cols);
        x.ldn = (uint32_t)up(x.n, kDepth), x.ldm = (uint32_t)up(x.m, kDepth);
        x.vec = !misaligned(x.g, 4 * ge) && x.pos % 4 == 0;
        x.wd = t.weight_decay, x.scale = t.scale;
        x.first = (uint32_t)chunk.size(), x.chunks = (uint32_t)((size + kChunk - 1) / kChunk);
        const uint64_t wide_bytes = (uint64_t)x.n * x.ldm * sizeof(half), square_bytes = (uint64_t)x.n * x.ldn * sizeof(half);
        x.x[0] = room(wide_bytes), x.x[1] = room(wide_bytes), x.low = room(wide_bytes);
        x.a = room(square_bytes), x.b = room(square_bytes);
        x.da = room(x.n * sizeof(float)), x.db = room(x.n * sizeof(float));
        const uint32_t id = (uint32_t)mats.size();
        for (uint32_t c = 0; c < x.chunks; ++c) chunk.push_back(Tile{id, c, 0});
        for (uint32_t r = 0; r * kTurn < x.rows; ++r)
          for (uint32_t c = 0; c * kTurn < x.cols; ++c) turn.push_back(Tile{id, r, c});
        for (uint32_t r = 0; r * kTile < x.n; ++r) {
          for (uint32_t c = r; c * kTile < x.n; ++c) square.push_back(Tile{id, r, c});
          for (uint32_t c = 0; c * kTile < x.m; ++c) wide.push_back(Tile{id, r, c});
        }
        mats.push_back(x);
      }
      base += up(size * t.count, kPad);
    }
    l = new train_matrices;
    l->bf16 = grad_dtype == ROTCONV_BF16;
    l->elements = base;
    l->sums = sums, l->workspace = at;
    l->count = (uint32_t)mats.size(), l->nchunk = (uint32_t)chunk.size(), l->nturn = (uint32_t)turn.size();
    l->nsquare = (uint32_t)square.size(), l->nwide = (uint32_t)wide.size();
    const size_t tiles = (size_t)l->nchunk + l->nturn + l->nsquare + l->nwide;
    bool ok = hipGetDevice(&l->device) == hipSuccess &&
              hipMalloc(&l->memory, mats.size() * sizeof(Matrix) + tiles * sizeof(Tile)) == hipSuccess;
    if (ok) {
      char* p = static_cast<char*>(l->memory);
      auto put = [&](const void* from, size_t bytes) {
        void* to = p;
        ok = ok && hipMemcpy(to, from, bytes, hipMemcpyHostToDevice) == hipSuccess;
        p += bytes;
        return to;
      };
      l->matrices = static_cast<Matrix*>(put(mats.data(), mats.size() * sizeof(Matrix)));
      l->chunk = static_cast<Tile*>(put(chunk.data(), chunk.size() * sizeof(Tile)));
      l->turn = static_cast<Tile*>(put(turn.data(), turn.size() * sizeof(Tile)));
      l->square = static_cast<Tile*>(put(square.data(), square.size() * sizeof(Tile)));
      l->wide = static_cast<Tile*>(put(wide.data(), wide.size() * sizeof(Tile)));
    }
    if (!ok) {
      (void)hipGetLastError();
      train_matrices_destroy(l);
      return ROTCONV_ERR_LAUNCH;
    }
  } catch (const std::exception&) {
    train_matrices_destroy(l);
    return ROTCONV_ERR_LAUNCH;
  }
  *out = l;
  return ROTCONV_OK;
}

int train_matrices_destroy(train_matrices* l) {
  if (!l) return ROTCONV_OK;
  if (l->memory) (void)hipFree(l->memory);
  delete l;
  return ROTCONV_OK;
}

uint64_t train_matrices_elements(const train_matrices* l) { return l ? l->elements : 0; }
size_t train_matrices_workspace_bytes(const train_matrices* l) { return l ? l->workspace : 0; }

int train_muon_step(const train_matrices* l, const train_muon* o, float* momentum, train_control* control, void* ws, size_t ws_bytes,
                    void* stream) {
  if (!l || !o || !momentum || !control) return ROTCONV_ERR_NULL;
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev != l->device) return ROTCONV_ERR_UNSUPPORTED;
  if (!(o->momentum >= 0.f && o->momentum < 1.f) || !(o->eps >= FLT_MIN && o->eps <= FLT_MAX) || (o->nesterov != 0 && o->nesterov != 1) || o->steps < 1 ||
      o->steps > 16 || (o->keep != 0 && o->keep != 1) || o->reserved != 0 || misaligned(momentum, 16) || misaligned(control, 4))
    return ROTCONV_ERR_UNSUPPORTED;
  if (!ws || misaligned(ws, 16) || ws_bytes < l->workspace) return ROTCONV_ERR_WORKSPACE;
  const hipStream_t st = static_cast<hipStream_t>(stream);
  char* w = static_cast<char*>(ws);
  float* inverse = reinterpret_cast<float*>(w + l->inverse);
  double* sums = reinterpret_cast<double*>(w + l->sums);
  auto first = l->bf16 ? k_momentum<uint16_t> : k_momentum<float>;
  first<<<l->nchunk, kThreads, 0, st>>>(l->matrices, l->chunk, *o, momentum, control, sums);
  k_inverse_norm<<<l->count, 64, 0, st>>>(l->matrices, o->eps, sums, inverse);
  auto start = l->bf16 ? k_start<uint16_t> : k_start<float>;
  start<<<l->nturn, kThreads, 0, st>>>(l->matrices, l->turn, *o, momentum, control, inverse, w);
  for (int k = 0; k < o->steps; ++k) {
    k_product<kGram><<<l->nsquare, kThreads, 0, st>>>(l->matrices, l->square, w, k % 2, control);
    k_product<kPoly><<<l->nsquare, kThreads, 0, st>>>(l->matrices, l->square, w, k % 2, control);
    if (k + 1 < o->steps) k_product<kApply><<<l->nwide, kThreads, 0, st>>>(l->matrices, l->wide, w, k % 2, control);
    else k_product<kLast><<<l->nwide, kThreads, 0, st>>>(l->matrices, l->wide, w, k % 2, control);
  }
  if (!o->keep) k_step_end<<<1, 1, 0, st>>>(control);
  return finish();
}

}  // extern "C"
