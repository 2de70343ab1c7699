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
  uint32_t tall, vec, even;            // vec: gradient and momentum can be read four elements at a time; even: the rows of p and copy
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

// X from u, tiles of 64 x 64 of the matrix as it lies in memory; the columns up to ldm are 0 (and stay so: a product of zeros)
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
  half *upper = reinterpret_cast<half*>(ws + x.x[0]), *lower = reinterpret_cast<half*>(ws + x.low);
  const uint32_t ti = x.tall ? t.j : t.i, tj = x.tall ? t.i : t.j;
  for (int k = wave; k < kTurn; k += 4) {
    const uint32_t i = ti * kTurn + k, j = tj * kTurn + lane;
    if (i >= x.n || j >= x.ldm) continue;
    const uint64_t at = (uint64_t)i * x.ldm + j;
    half u, l;
    split(x.tall ? turned[lane][k] : turned[k][lane], &u, &l);
    upper[at] = u, lower[at] = l;
  }
}

enum Product { kGram, kPoly, kApply, kLast };

// A wave's lanes bring 16 bytes each from memory to 1 KB of LDS in a row.
__device__ __forceinline__ void bring(const half* from, half* to) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)from, (__attribute__((address_space(3))) void*)to, 16, 0, 0);
}
// Rows r0 .. r0 + R - 1 (the last row again behind it) and kDepth columns of a matrix, a row of 128 bytes in LDS; its eight pieces of
// 16 bytes are exchanged by the row's number, so that the lanes of a fragment, a row each, meet all banks.
template <int R, int T>
__device__ __forceinline__ void bring_rows(const half* from, uint32_t ld, uint32_t r0, uint32_t rows, uint32_t k0, half* to) {
  const int tid = threadIdx.x, wave = tid / 64;
#pragma unroll
  for (int u = 0; u < R * 8 / T; ++u) {
    const int piece = u * T + tid, r = piece / 8, c = (piece % 8) ^ (r & 7);
    bring(from + (uint64_t)min(r0 + r, rows - 1) * ld + k0 + 8 * c, to + (u * T + wave * 64) * 8);
  }
}
__device__ __forceinline__ h8 fragment(const half* tile, int r, int c) { return *reinterpret_cast<const h8*>(tile + r * kDepth + (c ^ (r & 7)) * 8); }
// kDepth rows (the last again behind it) and C columns; the pieces of four neighbouring rows are moved 64 bytes apart.
template <int C, int T>
__device__ __forceinline__ void bring_columns(const half* from, uint32_t ld, uint32_t j0, uint32_t rows, uint32_t k0, half* to) {
  const int tid = threadIdx.x, wave = tid / 64;
  constexpr int P = C / 8;
#pragma unroll
  for (int u = 0; u < kDepth * P / T; ++u) {
    const int piece = u * T + tid, k = piece / P, c = (piece % P) ^ ((k & 3) << 2 & (P - 1));
    bring(from + (uint64_t)min(k0 + k, rows - 1) * ld + min(j0 + 8 * c, ld - 8), to + (u * T + wave * 64) * 8);
  }
}
// Eight rows k .. k + 7 of a column for each lane: columns j .. j + 31, the upper half of the lanes eight rows further.  The
// instruction turns a block of 4 rows x 16 columns for sixteen lanes: lane 4 r + q gives the address of row r's columns 4 q .., and gets
// column 4 r + q.
template <int C>
__device__ __forceinline__ h8 turned_fragment(const half* tile, int k, int j, int lane) {
  typedef short s4 __attribute__((ext_vector_type(4)));
  constexpr int P = C / 8;
  h8 v;
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const int row = k + 8 * (lane / 32) + 4 * e + lane % 16 / 4, col = j + lane % 32 / 16 * 16 + 4 * (lane % 4);
    const half* at = tile + row * C + ((col / 8) ^ ((row & 3) << 2 & (P - 1))) * 8 + col % 8;
    const h4 w = __builtin_bit_cast(h4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4*)at));
#pragma unroll
    for (int q = 0; q < 4; ++q) v[4 * e + q] = w[q];
  }
  return v;
}

// One tile of TM x TN of a product, WM x WN waves.
//   kGram   A = X X^T      kPoly   B = b A + c A^2      (tiles on and above the diagonal; the others are their mirror images)
//   kApply  X <- a X + B X      kLast   the same, into the parameters
template <int KIND, int TM, int TN, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN) void k_product(const Matrix* __restrict__ mats, const Tile* __restrict__ tiles, char* ws, int from,
                                                          const train_control* __restrict__ ctl) {
  constexpr int T = 64 * WM * WN, FM = TM / WM / 32, FN = TN / WN / 32;
  constexpr bool kSquare = KIND == kGram || KIND == kPoly;
  __shared__ __attribute__((aligned(16))) half a0[TM * kDepth], b0[TN * kDepth], a1[TM * kDepth], b1[TN * kDepth];
  if (ctl->nonfinite) return;
  const Tile t = tiles[blockIdx.x];
  const Matrix& x = mats[t.matrix];
  const uint32_t n = x.n, ldn = x.ldn, ldm = x.ldm;
  const half* X = reinterpret_cast<const half*>(ws + x.x[from]);
  const half* A = reinterpret_cast<const half*>(ws + x.a);
  const half* left = KIND == kGram ? X : KIND == kPoly ? A : reinterpret_cast<const half*>(ws + x.b);
  const half* right = KIND == kPoly ? A : X;
  const uint32_t ldl = KIND == kGram ? ldm : ldn, ldr = KIND == kPoly ? ldn : ldm, depth = KIND == kGram ? ldm : ldn;
  const int tid = threadIdx.x, lane = tid % 64, wr = tid / 64 / WN, wc = tid / 64 % WN;
  f16v acc[FM][FN] = {};
  auto load = [&](uint32_t k0, half* sa, half* sb) {
    bring_rows<TM, T>(left, ldl, t.i * TM, n, k0, sa);
    if constexpr (kSquare) bring_rows<TN, T>(right, ldr, t.j * TN, n, k0, sb);
    else bring_columns<TN, T>(right, ldr, t.j * TN, n, k0, sb);
  };
  auto multiply = [&](const half* __restrict__ sa, const half* __restrict__ sb) {
#pragma unroll
    for (int kk = 0; kk < kDepth / 16; ++kk) {
      h8 fa[FM], fb[FN];
#pragma unroll
      for (int q = 0; q < FM; ++q) fa[q] = fragment(sa, (wr * FM + q) * 32 + lane % 32, kk * 2 + lane / 32);
#pragma unroll
      for (int q = 0; q < FN; ++q)
        fb[q] = kSquare ? fragment(sb, (wc * FN + q) * 32 + lane % 32, kk * 2 + lane / 32)
                        : turned_fragment<TN>(sb, kk * 16, (wc * FN + q) * 32, lane);
#pragma unroll
      for (int p = 0; p < FM; ++p)
#pragma unroll
        for (int q = 0; q < FN; ++q) acc[p][q] = __builtin_amdgcn_mfma_f32_32x32x16_f16(fa[p], fb[q], acc[p][q], 0, 0, 0);
    }
  };
  auto arrived = [] {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
  };
  load(0, a0, b0);
  arrived();
  uint32_t k0 = 0;
  for (; k0 + kDepth < depth; k0 += 2 * kDepth) {
    load(k0 + kDepth, a1, b1);
    multiply(a0, b0);
    arrived();
    if (k0 + 2 * kDepth < depth) load(k0 + 2 * kDepth, a0, b0);
    multiply(a1, b1);
    arrived();
  }
  if (k0 < depth) {
    multiply(a0, b0);
    __syncthreads();
  }
  // What each wave holds, blocks of 32 x 32 one after the other, goes through 4 KB of its own in LDS, so that memory sees
  // eight elements a lane, four lanes a row.
  static_assert(TM * kDepth * sizeof(half) >= WM * WN * 4096, "a block of each wave");
  float* block = reinterpret_cast<float*>(a0) + tid / 64 * 1024;
  auto place = [](int r, int c) { return r * 32 + (((c / 4) ^ (r & 7)) * 4) + c % 4; };
  auto settle = [] {                   // this wave's LDS accesses, in order
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_wave_barrier();
  };
  float* da = reinterpret_cast<float*>(ws + x.da);
  float* db = reinterpret_cast<float*>(ws + x.db);
  const float lr = KIND == kLast ? ctl->lr : 0.f;
#pragma unroll
  for (int p = 0; p < FM; ++p)
#pragma unroll
    for (int q = 0; q < FN; ++q) {
      const uint32_t i0 = t.i * TM + (wr * FM + p) * 32, j0 = t.j * TN + (wc * FN + q) * 32;
      if (i0 >= n || j0 >= (kSquare ? ldn : ldm)) continue;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const float v = acc[p][q][e];
        block[place(8 * (e / 4) + 4 * (lane / 32) + e % 4, lane % 32)] = v;
      }
      settle();
      // eight elements of the block, along a row or along a column
      auto along_row = [&](int r, int c, float* v) {
        *reinterpret_cast<f4*>(v) = *reinterpret_cast<const f4*>(block + place(r, c));
        *reinterpret_cast<f4*>(v + 4) = *reinterpret_cast<const f4*>(block + place(r, c + 4));
      };
      auto along_column = [&](int r, int c, float* v) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = block[place(r + e, c)];
      };
      if constexpr (kSquare) {
        half* out = reinterpret_cast<half*>(ws + (KIND == kGram ? x.a : x.b));
        // out[i][j ..], from the sums v
        auto write = [&](uint32_t i, uint32_t j, const float* v) {
          if (i >= n || j >= ldn) return;
          h8 w;
          if constexpr (KIND == kGram) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              if (i == j + e) da[i] = v[e] * (1.f / (kHeld * kHeld));
              w[e] = i == j + e || j + e >= n ? (half)0.f : (half)(v[e] * (1.f / kHeld));
            }
          } else {
            const h8 held = *reinterpret_cast<const h8*>(A + (uint64_t)i * ldn + j);
            const float di = da[i];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const float dj = da[min(j + e, n - 1)];
              if (i == j + e) db[i] = kA + di * (kB + kC * di) + kC * (v[e] * (1.f / (kHeld * kHeld)));
              w[e] = i == j + e || j + e >= n ? (half)0.f : (half)((float)held[e] * (0.5f * (kB + kC * (di + dj))) + v[e] * (0.5f * kC / kHeld));
            }
          }
          *reinterpret_cast<h8*>(out + (uint64_t)i * ldn + j) = w;
        };
#pragma unroll
        for (int h = 0; h < 32; h += 16) {
          const int r = h + lane / 4, c = lane % 4 * 8;
          float v[8];
          along_row(r, c, v);
          write(i0 + r, j0 + c, v);
          if (t.i != t.j) {
            along_column(c, r, v);
            write(j0 + r, i0 + c, v);
          }
        }
      } else {
        half* low = reinterpret_cast<half*>(ws + x.low);
#pragma unroll
        for (int h = 0; h < 32; h += 16) {
          const int r = h + lane / 4, c = lane % 4 * 8;
          const uint32_t i = i0 + r, j = j0 + c;
          if (i < n && j < ldm) {
            const uint64_t at = (uint64_t)i * ldm + j;
            float v[8];
            along_row(r, c, v);
            const h8 hi = *reinterpret_cast<const h8*>(X + at), lo = *reinterpret_cast<const h8*>(low + at);
            const float d = db[i];
            h8 u, l;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              v[e] = d * joined(hi[e], lo[e]) + v[e] * (2.f / kHeld);
              if constexpr (KIND == kApply) {
                half ue, le;
                split(v[e], &ue, &le);
                u[e] = ue, l[e] = le;
              }
            }
            if constexpr (KIND == kApply) {
              *reinterpret_cast<h8*>(reinterpret_cast<half*>(ws + x.x[1 - from]) + at) = u;
              *reinterpret_cast<h8*>(low + at) = l;
            } else {
              *reinterpret_cast<f4*>(block + place(r, c)) = *reinterpret_cast<f4*>(v);
              *reinterpret_cast<f4*>(block + place(r, c + 4)) = *reinterpret_cast<f4*>(v + 4);
            }
          }
        }
        if constexpr (KIND == kLast) {
          settle();
          const float keep = x.wd * lr, move = x.scale * lr / kHeld;
#pragma unroll
          for (int h = 0; h < 32; h += 16) {
            float v[8];
            uint32_t row, col;
            if (x.tall) {
              along_column(lane % 4 * 8, h + lane / 4, v);
              row = j0 + h + lane / 4, col = i0 + lane % 4 * 8;
            } else {
              along_row(h + lane / 4, lane % 4 * 8, v);
              row = i0 + h + lane / 4, col = j0 + lane % 4 * 8;
            }
            if (row >= x.rows) continue;
            const uint64_t at = (uint64_t)row * x.cols + col;
            auto updated = [&](float r, float o) { return r - r * keep - o * move; };
            if (x.even && col + 8 <= x.cols) {
#pragma unroll
              for (int e = 0; e < 8; e += 4) {
                f4 r = *reinterpret_cast<const f4*>(x.p + at + e);
#pragma unroll
                for (int k = 0; k < 4; ++k) r[k] = updated(r[k], v[e + k]);
                *reinterpret_cast<f4*>(x.p + at + e) = r;
                if (x.copy) *reinterpret_cast<us4*>(x.copy + at + e) = us4{f32_to_bf16(r[0]), f32_to_bf16(r[1]), f32_to_bf16(r[2]), f32_to_bf16(r[3])};
              }
            } else {
#pragma unroll
              for (int e = 0; e < 8; ++e)
                if (col + e < x.cols) {
                  const float r = updated(x.p[at + e], v[e]);
                  x.p[at + e] = r;
                  if (x.copy) x.copy[at + e] = f32_to_bf16(r);
                }
            }
          }
        }
      }
      settle();
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
        x.even = !misaligned(x.p, 16) && !misaligned(x.copy, 8) && x.cols % 4 == 0;
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
    k_product<kGram, 128, 128, 2, 2><<<l->nsquare, kThreads, 0, st>>>(l->matrices, l->square, w, k % 2, control);
    k_product<kPoly, 128, 128, 2, 2><<<l->nsquare, kThreads, 0, st>>>(l->matrices, l->square, w, k % 2, control);
    if (k + 1 < o->steps) k_product<kApply, 128, 128, 2, 2><<<l->nwide, kThreads, 0, st>>>(l->matrices, l->wide, w, k % 2, control);
    else k_product<kLast, 128, 128, 2, 2><<<l->nwide, kThreads, 0, st>>>(l->matrices, l->wide, w, k % 2, control);
  }
  if (!o->keep) k_step_end<<<1, 1, 0, st>>>(control);
  return finish();
}

}  // extern "C"
