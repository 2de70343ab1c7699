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
//     of a tenth come out 1e-2 off, with it 4e-4.)
//   - The diagonals of A and of the polynomial are kept in fp32 and applied by themselves: rows of gradients are nearly
//     orthogonal, so that the diagonals are most of them, and their rounding would shift all singular values together (random
//     256 x 1024: 1.7e-3 off, without it 5e-4).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstdint>
#include <new>
#include <type_traits>
#include <utility>
#include <vector>

#include "glue_elt.h"
#include "rotconv.h"
#include "train_control.h"
#include "unettrain.h"

namespace {

constexpr int kThreads = 256;
constexpr int kPad = 32;               // elements: a stack's momentum starts on a multiple
constexpr int kTile = 128;             // edge of the products' tiles
constexpr int kSmall = 64;             // of A^2's, where tiles of 128 would leave CUs idle
constexpr int kDepth = 64;             // elements that a step of a product adds up
// Columns of X's tiles where a list's products add up kDeep steps or more on an average (one launch serves all of its matrices, by one kind of
// tile): fewer bytes through the caches, but fewer workgroups and larger ends.  Steps over 8 matrices of 768 x 3200 by tiles of 128 x 128 610 us, by
// 128 x 256 654; of 1024 x 4096 1179 and 1188; 4 of 1536 x 1536 and 2 of 1536 x 6144 1373 and 1370; 8 of 2048 x 8192 6935 and 6480; 4 of 4096 x 4096
// 7604 and 6970.
constexpr int kWide = 256;
constexpr uint32_t kDeep = 24;
constexpr uint32_t kSlots = 512;       // workgroups of the products that the chip holds at a time
constexpr int kTurn = 64;              // edge of the tiles by which X is first written
constexpr uint32_t kMostWorkgroups = (1u << 24) - 1;

struct Matrix {
  float* p;
  const void* g;
  uint16_t* copy;
  uint64_t pos;                        // of the momentum
  uint32_t rows, cols, n, m;           // n = min, m = max
  uint32_t ldn, ldm;                   // elements from row to row (leading()); what a product reads behind n and m is 0
  uint32_t tall, vec, even;            // vec: gradient and momentum can be read four elements at a time; even: the rows of p and copy, eight
  float wd, scale;
  uint32_t first, chunks;              // in the momentum's pass
  // byte offsets in the workspace: X's upper parts before and after an iteration, its lower part, A, B; the diagonals
  uint64_t x[2], low, a, b, da, db;
};
struct Tile {
  uint32_t matrix, i, j;
};
// A tile, or steps k0 .. k1 - 1 of its product: their sums then go to a place of their own in the workspace.
struct Unit {
  uint32_t matrix, i, j, k0, k1, place;
};
constexpr uint32_t kWhole = ~0u;
struct Join {                          // a tile whose sums lie in `count` places
  uint32_t matrix, i, j, first, count;
};

}  // namespace

struct train_matrices {
  int device = -1, bf16 = 0;
  uint64_t elements = 0;
  size_t workspace = 0, sums = 0, parts = 0;           // byte offsets: the chunks' sums, the units'
  uint32_t size = 0;                                   // elements of a chunk
  int small = 0, wide = 0;                             // A^2 by tiles of 64; X by tiles of kWide columns
  uint32_t least = 0;                                  // matrices, where all of them are small enough for a workgroup; blocks of the widest
  uint32_t widest = 0;
  void* memory = nullptr;
  uint32_t* tickets = nullptr;                         // 0 between calls
  Matrix* matrices = nullptr;
  Tile *chunk = nullptr, *turn = nullptr;
  Unit *gram = nullptr, *poly = nullptr, *apply = nullptr, *last = nullptr;
  Join* join = nullptr;
  uint32_t nchunk = 0, nturn = 0, ngram = 0, npoly = 0, napply = 0, nlast = 0, njoin = 0;
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
                                                       uint32_t chunk, float* __restrict__ momentum, const train_control* __restrict__ ctl,
                                                       double* sums) {
  __shared__ double red[kThreads / 64];
  if (ctl->nonfinite) return;
  const Tile c = chunks[blockIdx.x];
  const Matrix x = mats[c.matrix];
  const uint64_t from = (uint64_t)c.i * chunk, size = (uint64_t)x.rows * x.cols;
  const uint32_t n = (uint32_t)min((uint64_t)chunk, size - from);
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

// 2^15 / (|u| + eps), from the sum of u's squares, as two factors that an element takes one after the other: together they need not be a
// normal fp32 number (a matrix of zeros beside an eps below 9.6e-35, elements near 2^127), and lift, a power of two, is 1 where they are.
// u's elements are no larger than |u|, so that none overflows between the two, and what falls below 2^-149 there is 0 in fp16.
struct Factor {
  float lift, scale;
};
__device__ __forceinline__ Factor factor_to_unit(double squares, float eps) {
  const double f = (double)kHeld / (sqrt(squares) + (double)eps);
  const bool large = f > 0x1p100, small = f < 0x1p-100;
  return {large ? 0x1p100f : small ? 0x1p-100f : 1.f, (float)(f * (large ? 0x1p-100 : small ? 0x1p100 : 1.0))};
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
                                                    const double* __restrict__ sums, char* ws) {
  __shared__ float turned[kTurn][kTurn + 1];
  __shared__ double red[kThreads / 64];
  if (ctl->nonfinite) return;
  const Tile t = tiles[blockIdx.x];
  const Matrix x = mats[t.matrix];
  const int tid = threadIdx.x;
  const float coef = factor(*ctl), mu = opt.momentum;
  const T* g = static_cast<const T*>(x.g);
  const float* m = momentum + x.pos;
  // (four gradients of 16 bits are half a vector: a whole one needs a border of 16 bytes of its own)
  const bool pieces = x.vec && x.cols % 8 == 0, whole = sizeof(T) == 4 || reinterpret_cast<uintptr_t>(g) % 16 == 0;
  float v[2][8];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint32_t r = t.i * kTurn + tid / 8 + 32 * h, c = t.j * kTurn + tid % 8 * 8;
    const uint64_t at = (uint64_t)r * x.cols + c;
    float gv[8] = {}, mv[8] = {};
    if (r < x.rows && c < x.cols) {
      if (pieces) {
        Elt<float>::ldv(m + at, mv), Elt<float>::ldv(m + at + 4, mv + 4);
        if (whole) {
          Elt<T>::ldv(g + at, gv);
          if constexpr (sizeof(T) == 4) Elt<T>::ldv(g + at + 4, gv + 4);
        } else if constexpr (sizeof(T) == 2) {
          Elt<T>::ldh(g + at, gv), Elt<T>::ldh(g + at + 4, gv + 4);
        }
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (c + e < x.cols) mv[e] = m[at + e], gv[e] = Elt<T>::ld(g + at + e);
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) v[h][e] = direction(mv[e], gv[e] * coef, mu, opt.nesterov);
  }
  // X's factor, by every workgroup for itself while its loads are under way
  double s = 0;
  for (uint32_t c = tid; c < x.chunks; c += kThreads) s += sums[x.first + c];
  s = lanes_sum(s);
  if (tid % 64 == 0) red[tid / 64] = s;
  __syncthreads();
  const Factor unit = factor_to_unit((red[0] + red[1]) + (red[2] + red[3]), opt.eps);
  if (x.tall) {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int e = 0; e < 8; ++e) turned[tid / 8 + 32 * h][tid % 8 * 8 + e] = v[h][e];
    __syncthreads();
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int e = 0; e < 8; ++e) v[h][e] = turned[tid % 8 * 8 + e][tid / 8 + 32 * h];
  }
  const uint32_t ti = x.tall ? t.j : t.i, tj = x.tall ? t.i : t.j;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint32_t i = ti * kTurn + tid / 8 + 32 * h, j = tj * kTurn + tid % 8 * 8;
    if (i >= x.n) continue;
    h8 u, l;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      half ue, le;
      split(v[h][e] * unit.lift * unit.scale, &ue, &le);
      u[e] = ue, l[e] = le;
    }
    const uint64_t at = (uint64_t)i * x.ldm + j;
    *reinterpret_cast<h8*>(reinterpret_cast<half*>(ws + x.x[0]) + at) = u;
    *reinterpret_cast<h8*>(reinterpret_cast<half*>(ws + x.low) + at) = l;
  }
}

// By every workgroup of a step's last launch, when all its waves have what they want of the control block (skip, and two more values): the
// last of them advances it.  (A barrier alone does not wait for loads under way.)
__device__ __forceinline__ void end_of_step(train_control* ctl, int skip, float one, float two, uint32_t* tickets) {
  asm volatile("" ::"v"(skip), "v"(one), "v"(two));
  __syncthreads();
  if (threadIdx.x == 0 && last_to_come(tickets)) end_step(ctl, skip, ctl->step + 1);
}

enum Product { kGram, kPoly, kApply, kLast };

// A wave's lanes bring 16 bytes each from memory to 1 KB of LDS in a row.  In assembler, without an output register, so that the
// products alone say when it has to have arrived (step() below): the compiler would wait for all loads under way before reading
// an LDS array that a loop fills.
__device__ __forceinline__ void bring(const half* from, half* to) {
  const uint32_t at = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)to);
  // (m0, where the instruction takes the place in LDS from, is the compiler's to set, so that it keeps nothing else there; what reads it so has to
  // wait for an instruction behind that)
  asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"{m0}"(at), "v"(from) : "memory");
}
// Rows r0 .. r0 + R - 1 (the last row again behind it) and kDepth columns of a matrix, a row of 128 bytes in LDS; its eight pieces of
// 16 bytes are exchanged by the row's number, two rows alike, so that sixteen lanes of a fragment, a row each, meet all 64 banks.
template <int R, int D, int T>
__device__ __forceinline__ void bring_rows(const half* from, uint32_t ld, uint32_t r0, uint32_t rows, uint32_t k0, half* to) {
  const int tid = threadIdx.x, wave = tid / 64;
  constexpr int P = D / 8;
#pragma unroll
  for (int u = 0; u < R * P / T; ++u) {
    const int piece = u * T + tid, r = piece / P, c = (piece % P) ^ (r / (16 / P) & (P - 1));
    bring(from + (uint64_t)min(r0 + r, rows - 1) * ld + k0 + 8 * c, to + (u * T + wave * 64) * 8);
  }
}
template <int D>
__device__ __forceinline__ h8 fragment(const half* tile, int r, int c) {
  constexpr int P = D / 8;
  return *reinterpret_cast<const h8*>(tile + r * D + (c ^ (r / (16 / P) & (P - 1))) * 8);
}
// kDepth rows (the last again behind it) and C columns; the pieces of four neighbouring rows are moved 64 bytes apart.
template <int C, int D, int T>
__device__ __forceinline__ void bring_columns(const half* from, uint32_t ld, uint32_t j0, uint32_t rows, uint32_t k0, half* to) {
  const int tid = threadIdx.x, wave = tid / 64;
  constexpr int P = C / 8;
#pragma unroll
  for (int u = 0; u < D * P / T; ++u) {
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

// What becomes of a tile's sums.
//   kGram   A = X X^T      kPoly   B = b A + c A^2      (tiles on and above the diagonal; the others are their mirror images)
//   kApply  X <- a X + B X      kLast   the same, into the parameters
// A wave's blocks of up to 64 x 64 go one after the other through LDS of its own, so that memory sees eight elements a lane and whole
// lines a row, and what they are joined with is loaded all at once before.
template <int KIND, int TM, int TN, int WM, int WN>
struct Finish {
  static constexpr int kMost = KIND == kApply ? 32 : 64;         // (three workgroups of kApply share a CU: see k_product)
  static constexpr int kRows = TM / WM < kMost ? TM / WM : kMost, kCols = TN / WN < 64 ? TN / WN : 64;       // of a block
  static constexpr int kBytes = WM * WN * kRows * kCols * sizeof(float);
  static constexpr bool kSquare = KIND == kGram || KIND == kPoly;
  // eight elements a lane: along the rows kAcross lanes a row, along the columns kDown lanes a column
  static constexpr int kAcross = kCols / 8, kDown = kRows / 8, kPass = kRows * kAcross / 64, kTurnPass = kCols * kDown / 64;

  // pieces of four elements exchanged so that neither direction's lanes meet in a bank
  static __device__ __forceinline__ int place(int r, int c) { return r * kCols + (((c / 4) ^ ((r ^ r / 8) & (kCols / 4 - 1))) * 4) + c % 4; }
  static __device__ __forceinline__ void settle() {              // this wave's LDS accesses, in order
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_wave_barrier();
  }
  static __device__ __forceinline__ void along_row(const float* block, int r, int c, float* v) {
    *reinterpret_cast<f4*>(v) = *reinterpret_cast<const f4*>(block + place(r, c));
    *reinterpret_cast<f4*>(v + 4) = *reinterpret_cast<const f4*>(block + place(r, c + 4));
  }
  static __device__ __forceinline__ void along_column(const float* block, int r, int c, float* v) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = block[place(r + e, c)];
  }

  // out[i][j .. j + 7] of a symmetric product, from its sums v; held: A's elements there, di, dj: its diagonal's.  The diagonal itself
  // is left 0.
  static __device__ __forceinline__ void symmetric(const Matrix& x, half* out, uint32_t i, uint32_t j, const float* v, const h8& held, float di,
                                                   const float* dj) {
    h8 w;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float r;
      if constexpr (KIND == kGram) r = v[e] * (1.f / kHeld);
      else r = (float)held[e] * (0.5f * (kB + kC * (di + dj[e]))) + v[e] * (0.5f * kC / kHeld);
      w[e] = i == j + e || j + e >= x.n ? (half)0.f : (half)r;
    }
    if (i < x.n && j < x.ldn) *reinterpret_cast<h8*>(out + (uint64_t)i * x.ldn + j) = w;
  }

  static __device__ __forceinline__ void tile(const Matrix& x, uint32_t ti, uint32_t tj, const f16v (&acc)[TM / WM / 32][TN / WN / 32], int wave, float* block,
                                              char* ws, int from, float lr) {
    const int lane = threadIdx.x % 64, wr = wave / WN, wc = wave % WN;
    const uint32_t n = x.n, ldn = x.ldn, ldm = x.ldm;
#pragma unroll
    for (int bp = 0; bp < TM / WM / kRows; ++bp)
#pragma unroll
      for (int bq = 0; bq < TN / WN / kCols; ++bq) {
        const uint32_t i0 = ti * TM + wr * (TM / WM) + bp * kRows, j0 = tj * TN + wc * (TN / WN) + bq * kCols;
        if (i0 >= n || j0 >= (kSquare ? ldn : ldm)) continue;
        const int r0 = lane / kAcross, c0 = lane % kAcross * 8, rt = lane % kDown * 8, ct = lane / kDown;
        auto hold = [&] {
#pragma unroll
          for (int p = 0; p < kRows / 32; ++p)
#pragma unroll
            for (int q = 0; q < kCols / 32; ++q)
#pragma unroll
              for (int e = 0; e < 16; ++e) {
                const float v = acc[bp * (kRows / 32) + p][bq * (kCols / 32) + q][e];
                block[place(p * 32 + 8 * (e / 4) + 4 * (lane / 32) + e % 4, q * 32 + lane % 32)] = v;
              }
          settle();
        };
        if constexpr (kSquare) {
          const half* A = reinterpret_cast<const half*>(ws + x.a);
          half* out = reinterpret_cast<half*>(ws + (KIND == kGram ? x.a : x.b));
          float *da = reinterpret_cast<float*>(ws + x.da), *db = reinterpret_cast<float*>(ws + x.db);
          const bool mirror = ti != tj;
          // a lane's columns are the same in all passes, its rows are not
          auto pass = [&](uint32_t i, uint32_t j, auto passes, int step, auto read) {
            constexpr int P = decltype(passes)::value;
            h8 held[P] = {};
            float di[P] = {}, dj[8] = {};
            if constexpr (KIND == kPoly) {
              const uint32_t at = min(j, ldn - 8);
#pragma unroll
              for (int h = 0; h < P; ++h) {
                const uint32_t row = min(i + h * step, n - 1);
                held[h] = *reinterpret_cast<const h8*>(A + (uint64_t)row * ldn + at);
                di[h] = da[row];
              }
              Elt<float>::ldv(da + at, dj), Elt<float>::ldv(da + at + 4, dj + 4);  // (ldn of them: what is behind the last is not used)
            }
#pragma unroll
            for (int h = 0; h < P; ++h) {
              float v[8];
              read(h * step, v);
              symmetric(x, out, i + h * step, j, v, held[h], di[h], dj);
            }
          };
          hold();
          if (i0 == j0 && lane < kRows && i0 + lane < n) {
            const float v = block[place(lane, lane)] * (1.f / (kHeld * kHeld));
            if constexpr (KIND == kGram) da[i0 + lane] = v;
            else db[i0 + lane] = kA + da[i0 + lane] * (kB + kC * da[i0 + lane]) + kC * v;
          }
          pass(i0 + r0, j0 + c0, std::integral_constant<int, kPass>{}, 64 / kAcross, [&](int h, float* v) { along_row(block, r0 + h, c0, v); });
          if (mirror)
            pass(j0 + ct, i0 + rt, std::integral_constant<int, kTurnPass>{}, 64 / kDown, [&](int h, float* v) { along_column(block, rt, ct + h, v); });
        } else {
          const half* X = reinterpret_cast<const half*>(ws + (from ? x.x[1] : x.x[0]));
          half* low = reinterpret_cast<half*>(ws + x.low);
          const float* db = reinterpret_cast<const float*>(ws + x.db);
          h8 hi[kPass], lo[kPass];
          float d[kPass];
#pragma unroll
          for (int h = 0; h < kPass; ++h) {
            const uint32_t i = min(i0 + r0 + h * (64 / kAcross), n - 1);
            const uint64_t at = (uint64_t)i * ldm + min(j0 + c0, ldm - 8);
            hi[h] = *reinterpret_cast<const h8*>(X + at), lo[h] = *reinterpret_cast<const h8*>(low + at);
            d[h] = db[i];
          }
          hold();
#pragma unroll
          for (int h = 0; h < kPass; ++h) {
            const int r = r0 + h * (64 / kAcross);
            const uint32_t i = i0 + r, j = j0 + c0;
            float v[8];
            along_row(block, r, c0, v);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = d[h] * joined(hi[h][e], lo[h][e]) + v[e] * (2.f / kHeld);
            if constexpr (KIND == kApply) {
              h8 u, l;
#pragma unroll
              for (int e = 0; e < 8; ++e) {
                half ue, le;
                split(v[e], &ue, &le);
                u[e] = ue, l[e] = le;
              }
              if (i < n && j < ldm) {
                const uint64_t at = (uint64_t)i * ldm + j;
                *reinterpret_cast<h8*>(reinterpret_cast<half*>(ws + (from ? x.x[0] : x.x[1])) + at) = u;
                *reinterpret_cast<h8*>(low + at) = l;
              }
            } else {
              *reinterpret_cast<f4*>(block + place(r, c0)) = f4{v[0], v[1], v[2], v[3]};
              *reinterpret_cast<f4*>(block + place(r, c0 + 4)) = f4{v[4], v[5], v[6], v[7]};
            }
          }
          if constexpr (KIND == kLast) {
            settle();
            if (x.tall) update<kTurnPass, true>(x, block, j0 + ct, i0 + rt, rt, ct, lr);
            else update<kPass, false>(x, block, i0 + r0, j0 + c0, r0, c0, lr);
          }
        }
        settle();
      }
  }
  // the parameters from a block of X, by rows of the matrix as it lies in memory (TALL: the block's columns)
  template <int PASSES, bool TALL>
  static __device__ __forceinline__ void update(const Matrix& x, const float* block, uint32_t row0, uint32_t col, int r0, int c0, float lr) {
    constexpr int kStep = 64 / (TALL ? kDown : kAcross);
    const float keep = x.wd * lr, move = x.scale * lr / kHeld;
    auto updated = [&](float r, float o) { return r - r * keep - o * move; };
    auto read = [&](int h, float* v) {
      if constexpr (TALL) along_column(block, r0, c0 + h * kStep, v);
      else along_row(block, r0 + h * kStep, c0, v);
    };
    if (x.even) {
      if (col >= x.cols) return;
      f4 old[PASSES][2];
#pragma unroll
      for (int h = 0; h < PASSES; ++h)
#pragma unroll
        for (int e = 0; e < 2; ++e) old[h][e] = *reinterpret_cast<const f4*>(x.p + (uint64_t)min(row0 + h * kStep, x.rows - 1) * x.cols + col + 4 * e);
#pragma unroll
      for (int h = 0; h < PASSES; ++h) {
        float v[8];
        read(h, v);
        if (row0 + h * kStep >= x.rows) continue;
        const uint64_t at = (uint64_t)(row0 + h * kStep) * x.cols + col;
        float r[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) r[e] = updated(old[h][e / 4][e % 4], v[e]);
        *reinterpret_cast<f4*>(x.p + at) = f4{r[0], r[1], r[2], r[3]};
        *reinterpret_cast<f4*>(x.p + at + 4) = f4{r[4], r[5], r[6], r[7]};
        if (x.copy) Elt<uint16_t>::stv(x.copy + at, r);
      }
      return;
    }
#pragma unroll 1
    for (int h = 0; h < PASSES; ++h) {
      float v[8];
      read(h, v);
      if (row0 + h * kStep >= x.rows) continue;
      const uint64_t at = (uint64_t)(row0 + h * kStep) * x.cols + col;
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (col + e < x.cols) {
          const float r = updated(x.p[at + e], v[e]);
          x.p[at + e] = r;
          if (x.copy) x.copy[at + e] = f32_to_bf16(r);
        }
    }
  }
};

// One tile of TM x TN of a product, or some of its steps, WM x WN waves.
template <int KIND, int TM, int TN, int WM, int WN, int D, int NS>
__global__ __launch_bounds__(64 * WM * WN) __attribute__((amdgpu_waves_per_eu(KIND == kApply && TN == kTile ? 3 : 2))) void k_product(const Matrix* __restrict__ mats, const Unit* __restrict__ units, char* ws, int from,
                                                          f4* parts, train_control* ctl, uint32_t* tickets) {
  constexpr int T = 64 * WM * WN, FM = TM / WM / 32, FN = TN / WN / 32;
  constexpr bool kSquare = KIND == kGram || KIND == kPoly;
  __shared__ __attribute__((aligned(16))) half stages[NS][(TM + TN) * D];
  const int skip = ctl->nonfinite;
  const float lr = KIND == kLast ? ctl->lr : 0.f;
  if (KIND == kLast && tickets) end_of_step(ctl, skip, lr, lr, tickets);
  if (skip) return;
  const Unit t = units[blockIdx.x];
  if (t.k0 == t.k1) return;
  const Matrix x = mats[t.matrix];
  const uint32_t n = x.n, ldn = x.ldn, ldm = x.ldm;
  const half* X = reinterpret_cast<const half*>(ws + (from ? x.x[1] : x.x[0]));
  const half* A = reinterpret_cast<const half*>(ws + x.a);
  const half* left = KIND == kGram ? X : KIND == kPoly ? A : reinterpret_cast<const half*>(ws + x.b);
  const half* right = KIND == kPoly ? A : X;
  const uint32_t ldl = KIND == kGram ? ldm : ldn, ldr = KIND == kPoly ? ldn : ldm;
  const int tid = threadIdx.x, lane = tid % 64, wr = tid / 64 / WN, wc = tid / 64 % WN;
  f16v acc[FM][FN] = {};
  auto load = [&](uint32_t k0, half* sa) {
    half* sb = sa + TM * D;
    bring_rows<TM, D, T>(left, ldl, t.i * TM, n, k0, sa);
    if constexpr (kSquare) bring_rows<TN, D, T>(right, ldr, t.j * TN, n, k0, sb);
    else bring_columns<TN, D, T>(right, ldr, t.j * TN, n, k0, sb);
  };
  auto multiply = [&](const half* sa) {
    const half* sb = sa + TM * D;
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) {
      h8 fa[FM], fb[FN];
#pragma unroll
      for (int q = 0; q < FM; ++q) fa[q] = fragment<D>(sa, (wr * FM + q) * 32 + lane % 32, kk * 2 + lane / 32);
#pragma unroll
      for (int q = 0; q < FN; ++q)
        fb[q] = kSquare ? fragment<D>(sb, (wc * FN + q) * 32 + lane % 32, kk * 2 + lane / 32)
                        : turned_fragment<TN>(sb, kk * 16, (wc * FN + q) * 32, lane);
#pragma unroll
      for (int p = 0; p < FM; ++p)
#pragma unroll
        for (int q = 0; q < FN; ++q) acc[p][q] = __builtin_amdgcn_mfma_f32_32x32x16_f16(fa[p], fb[q], acc[p][q], 0, 0, 0);
    }
  };
  // Before step k, what it needs has arrived (later steps' loads stay on their way) and everybody is done with step k - 1, whose
  // place step k + NS - 1 takes.  The last steps load the last columns again, into places that nobody reads any more.
  constexpr int kLoads = (TM + TN) * (D / 8) / T;
  const uint32_t begin = t.k0 * (kDepth / D), last = t.k1 * (kDepth / D) - 1;
#pragma unroll
  for (int u = 0; u < NS - 1; ++u) load(min(begin + u, last) * D, stages[u]);
  uint32_t here = 0, next = NS - 1;
  for (uint32_t k = begin; k <= last; ++k) {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"i"((NS - 2) * kLoads) : "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    load(min(k + NS - 1, last) * D, stages[next]);
    multiply(stages[here]);
    here = here + 1 == NS ? 0 : here + 1;
    next = next + 1 == NS ? 0 : next + 1;
  }
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
  __syncthreads();
  if (t.place != kWhole) {             // as the lanes hold them
    f4* to = parts + (uint64_t)t.place * (TM * TN / 4) + tid;
#pragma unroll
    for (int p = 0; p < FM; ++p)
#pragma unroll
      for (int q = 0; q < FN; ++q)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          to[((p * FN + q) * 4 + e) * T] = f4{acc[p][q][4 * e], acc[p][q][4 * e + 1], acc[p][q][4 * e + 2], acc[p][q][4 * e + 3]};
    return;
  }
  using F = Finish<KIND, TM, TN, WM, WN>;
  static_assert(sizeof(stages) >= F::kBytes, "a block of each wave");
  F::tile(x, t.i, t.j, acc, tid / 64, reinterpret_cast<float*>(stages) + tid / 64 * (F::kBytes / (WM * WN) / sizeof(float)), ws, from, lr);
}

// The tiles of A whose sums units have left in places of their own: added in the places' order, and finished, a block of 32 x 32 a wave (and a
// workgroup: the places' sums are then on their way all at once; 31 M parameters of a stack, 158 tiles in up to 6 places: 10 us; 17 by
// whole tiles, 14 by blocks of 64 x 64).
__global__ __launch_bounds__(64) void k_join(const Matrix* __restrict__ mats, const Join* __restrict__ joins, char* ws, const f4* __restrict__ parts,
                                             const train_control* __restrict__ ctl) {
  constexpr int kEdge = kTile / 32;    // blocks of a tile
  using F = Finish<kGram, kTile, kTile, kEdge, kEdge>;
  __shared__ __attribute__((aligned(16))) float block[32 * 32];
  if (ctl->nonfinite) return;
  const Join t = joins[blockIdx.x / (kEdge * kEdge)];
  const Matrix x = mats[t.matrix];
  // the units' four waves hold 2 x 2 blocks each
  const int mine = blockIdx.x % (kEdge * kEdge), r = mine / kEdge, c = mine % kEdge;
  const f4* from = parts + (uint64_t)t.first * (kTile * kTile / 4) + ((r % 2) * 2 + c % 2) * 4 * kThreads + (r / 2 * 2 + c / 2) * 64 + threadIdx.x;
  f16v acc[1][1] = {};
#pragma unroll 4
  for (uint32_t q = 0; q < t.count; ++q, from += kTile * kTile / 4) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const f4 v = from[e * kThreads];
#pragma unroll
      for (int k = 0; k < 4; ++k) acc[0][0][4 * e + k] += v[k];
    }
  }
  F::tile(x, t.i, t.j, acc, mine, block, ws, 0, 0.f);
}

// Four elements at any element's address
template <typename T> struct Any4;
template <> struct Any4<float> {
  typedef float f4a __attribute__((ext_vector_type(4), aligned(4)));
  static __device__ __forceinline__ void ld(const float* p, float* v) {
    const f4a a = *reinterpret_cast<const f4a*>(p);
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = a[k];
  }
  static __device__ __forceinline__ void st(float* p, const float* v) { *reinterpret_cast<f4a*>(p) = f4a{v[0], v[1], v[2], v[3]}; }
};
template <> struct Any4<uint16_t> {
  typedef uint16_t us4a __attribute__((ext_vector_type(4), aligned(2)));
  static __device__ __forceinline__ void ld(const uint16_t* p, float* v) {
    const us4a a = *reinterpret_cast<const us4a*>(p);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const uint16_t b = a[k];
      v[k] = bf16_to_f32(b);
    }
  }
  static __device__ __forceinline__ void st(uint16_t* p, const float* v) {
    *reinterpret_cast<us4a*>(p) = us4a{f32_to_bf16(v[0]), f32_to_bf16(v[1]), f32_to_bf16(v[2]), f32_to_bf16(v[3])};
  }
};

// The whole step of a matrix with at most 64 rows (or columns) and 1024 columns (or rows), by one workgroup of sixteen waves: X stays in
// registers in 32 bits, blocks of 32 x 32 as the matrix instructions leave them, up to NT a wave, and its upper part in LDS for the products.
// For lists of such matrices alone: a step is one launch (eleven filters of a stack of widths 16, 32, 64: 36 us; by the products' launches 117).
constexpr uint32_t kLeastRows = 64, kLeastCols = 1024;
constexpr int kLeastThreads = 1024, kAcross = kLeastCols + 40, kAside = 72;      // elements from row to row in LDS: rows in banks of their own
template <typename T, int NT>
__global__ __launch_bounds__(kLeastThreads) void k_least(const Matrix* __restrict__ mats, train_muon opt, float* __restrict__ momentum,
                                                         train_control* ctl, uint32_t* tickets) {
  constexpr int kWaves = kLeastThreads / 64;
  __shared__ __attribute__((aligned(16))) half X[kLeastRows * kAcross];
  __shared__ __attribute__((aligned(16))) half A[kLeastRows * kAside];
  __shared__ __attribute__((aligned(16))) half B[kLeastRows * kAside];             // (as it is: its elements meet those of the diagonal, of order 1)
  __shared__ __attribute__((aligned(16))) float da[kLeastRows], db[kLeastRows];
  __shared__ double red[kWaves];
  const int skip = ctl->nonfinite;
  const float coef = factor(*ctl), mu = opt.momentum, lr = ctl->lr;
  if (tickets) end_of_step(ctl, skip, lr, coef, tickets);
  if (skip) return;
  const Matrix x = mats[blockIdx.x];
  const int tid = threadIdx.x, lane = tid % 64, wave = __builtin_amdgcn_readfirstlane(tid / 64);
  const int high = x.n > 32 ? 2 : 1, wide = (int)((x.m + 31) / 32), blocks = high * wide, K = high * 32;
  const T* g = static_cast<const T*>(x.g);
  float* m = momentum + x.pos;
  // element e of a lane in a block: row 8 (e / 4) + 4 (lane / 32) + e % 4, column lane % 32
  auto row_of = [&](int block, int e) { return (block % high) * 32 + 8 * (e / 4) + 4 * (lane / 32) + e % 4; };
  auto col_of = [&](int block) { return (block / high) * 32 + lane % 32; };
  // Calls use(e, place in memory, inside) for a lane's elements.  Blocks inside the matrix: a lane's place and what all lanes add to it.  Others:
  // outside the matrix the place is that of its last row or column, so that loads go without questions.
  auto each = [&](int block, auto use) {
    const uint32_t i0 = (block % high) * 32, j0 = (block / high) * 32;
    if (i0 + 32 <= x.n && j0 + 32 <= x.m) {
      const uint32_t across = x.tall ? 1 : x.cols, down = x.tall ? x.cols : 1, own = 4 * (lane / 32) * across + (lane % 32) * down;
#pragma unroll
      for (int e = 0; e < 16; ++e) use(e, own + ((i0 + 8 * (e / 4) + e % 4) * across + j0 * down), true);
    } else {
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const uint32_t i = row_of(block, e), j = col_of(block), ic = min(i, x.n - 1), jc = min(j, x.m - 1);
        use(e, x.tall ? jc * x.cols + ic : ic * x.cols + jc, i < x.n && j < x.m);
      }
    }
  };
  // Four elements side by side in memory, where a tall matrix holds a lane's: their places
  auto fours = [&](int block) { return x.tall && (uint32_t)(block % high) * 32 + 32 <= x.n && (uint32_t)(block / high) * 32 + 32 <= x.m; };
  auto place_of = [&](int block, int q) { return ((uint32_t)(block / high) * 32 + lane % 32) * x.cols + (uint32_t)(block % high) * 32 + 8 * q + 4 * (lane / 32); };
  f16v v[NT];
  double square = 0;
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int block = wave + t * kWaves;
    v[t] = f16v{};
    if (block >= blocks) continue;
    float gv[16], mv[16];
    if (fours(block)) {
#pragma unroll
      for (int q = 0; q < 4; ++q) Any4<T>::ld(g + place_of(block, q), gv + 4 * q), Any4<float>::ld(m + place_of(block, q), mv + 4 * q);
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const float gk = gv[e] * coef;
        mv[e] = next_momentum(mv[e], gk, mu);
        v[t][e] = direction(mv[e], gk, mu, opt.nesterov);
      }
#pragma unroll
      for (int q = 0; q < 4; ++q) Any4<float>::st(m + place_of(block, q), mv + 4 * q);
    } else {
      each(block, [&](int e, uint32_t at, bool) { gv[e] = Elt<T>::ld(g + at), mv[e] = m[at]; });
      each(block,  [&](int e, uint32_t at, bool inside) {
        const float gk = gv[e] * coef, mk = next_momentum(mv[e], gk, mu);
        if (inside) {
          m[at] = mk;
          v[t][e] = direction(mk, gk, mu, opt.nesterov);
        }
      });
    }
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const double u = v[t][e];
      square += u * u;
    }
  }
  square = lanes_sum(square);
  if (lane == 0) red[wave] = square;
  __syncthreads();
  double all = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) all += red[w];
  const Factor unit = factor_to_unit(all, opt.eps);
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int e = 0; e < 16; ++e) v[t][e] = v[t][e] * unit.lift * unit.scale;

  // The symmetric products by blocks of 16 x 16, one a wave: row and column of its four elements a lane
  const int edge = 2 * high, bi = wave / edge, bj = wave % edge, sj = bj * 16 + lane % 16, si = bi * 16 + 4 * (lane / 16);
  const bool works = wave < edge * edge;
  auto product = [&](const half* from, int across, int depth) {
    f4 sum = {};
    for (int k = 0; k < depth; k += 32) {
      const h8 fa = *reinterpret_cast<const h8*>(from + (bi * 16 + lane % 16) * across + k + 8 * (lane / 16));
      const h8 fb = *reinterpret_cast<const h8*>(from + (bj * 16 + lane % 16) * across + k + 8 * (lane / 16));
      sum = __builtin_amdgcn_mfma_f32_16x16x32_f16(fa, fb, sum, 0, 0, 0);
    }
    return sum;
  };
  for (int step = 0; step < opt.steps; ++step) {
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int block = wave + t * kWaves;
      if (block < blocks) {
        half* to = X + row_of(block, 0) * kAcross + col_of(block);
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const float r = v[t][e];
          to[(8 * (e / 4) + e % 4) * kAcross] = (half)r;
        }
      }
    }
    __syncthreads();
    float a[4] = {};
    if (works) {
      const f4 sum = product(X, kAcross, wide * 32);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float r = sum[e];
        a[e] = si + e == sj ? 0.f : (float)(half)(r * (1.f / kHeld));
        A[(si + e) * kAside + sj] = (half)a[e];
        if (si + e == sj) da[sj] = r * (1.f / (kHeld * kHeld));
      }
    }
    __syncthreads();
    if (works) {
      const f4 sum = product(A, kAside, K);
      const float dj = da[sj];
      const f4 di = *reinterpret_cast<const f4*>(da + si);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float s = sum[e] * (kC / (kHeld * kHeld)), d = di[e];
        B[(si + e) * kAside + sj] = si + e == sj ? (half)0.f : (half)(a[e] * ((kB + kC * (d + dj)) / kHeld) + s);
        if (si + e == sj) db[sj] = kA + d * (kB + kC * d) + s;
      }
    }
    __syncthreads();
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int own = wave + t * kWaves;
      if (own < blocks) {
        // a X + B X in the same registers
#pragma unroll
        for (int e = 0; e < 16; e += 4) {
          const f4 d = *reinterpret_cast<const f4*>(db + row_of(own, e));
#pragma unroll
          for (int k = 0; k < 4; ++k) v[t][e + k] = v[t][e + k] * d[k];
        }
        const half* rows = B + ((own % high) * 32 + lane % 32) * kAside + 8 * (lane / 32);
        const half* cols = X + (8 * (lane / 32) + lane % 16 / 4) * kAcross + (own / high) * 32 + lane % 32 / 16 * 16 + 4 * (lane % 4);
        for (int k = 0; k < K; k += 16) {
          const h8 fa = *reinterpret_cast<const h8*>(rows + k);
          h8 fb;
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            typedef short s4 __attribute__((ext_vector_type(4)));
            const h4 w = __builtin_bit_cast(h4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4*)(cols + (k + 4 * e) * kAcross)));
#pragma unroll
            for (int q = 0; q < 4; ++q) fb[4 * e + q] = w[q];
          }
          v[t] = __builtin_amdgcn_mfma_f32_32x32x16_f16(fa, fb, v[t], 0, 0, 0);
        }
      }
    }
    __syncthreads();
  }
  const float keep = x.wd * lr, move = x.scale * lr / kHeld;
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int block = wave + t * kWaves;
    if (block >= blocks) continue;
    float old[16];
    if (fours(block)) {
#pragma unroll
      for (int q = 0; q < 4; ++q) Any4<float>::ld(x.p + place_of(block, q), old + 4 * q);
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const float o = v[t][e];
        old[e] = old[e] - old[e] * keep - o * move;
      }
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        Any4<float>::st(x.p + place_of(block, q), old + 4 * q);
        if (x.copy) Any4<uint16_t>::st(x.copy + place_of(block, q), old + 4 * q);
      }
      continue;
    }
    each(block, [&](int e, uint32_t at, bool) { old[e] = x.p[at]; });
    each(block, [&](int e, uint32_t at, bool inside) {
      const float o = v[t][e], r = old[e] - old[e] * keep - o * move;
      if (inside) {
        x.p[at] = r;
        if (x.copy) x.copy[at] = f32_to_bf16(r);
      }
    });
  }
}

int finish() { return hipGetLastError() == hipSuccess ? ROTCONV_OK : ROTCONV_ERR_LAUNCH; }
bool misaligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }
// Workgroups go to the eight dies in turn, and each die has a cache of its own.  So the units, listed in an order in which neighbours share
// operands, are cut into eight runs of like work; a die's deepest units come first, so that none starts when the others end, and where a run
// is shorter than another, units without steps stand in.  (Matrices of 2048 x 2048 and 2048 x 5632, A: 590 MB through the caches where every
// die works on every matrix.)  ends: what a unit takes beside its steps, in steps, as measured: 32 for A (113 us for those matrices, 120 with
// 4), 4 for X (78 us for the 31 M parameters of a stack, 87 with 16 or 32, 91 not dealt).
std::vector<Unit> by_die(const std::vector<Unit>& in, uint64_t ends) {
  constexpr uint64_t kDies = 8;
  uint64_t work = 0, done = 0;
  for (const Unit& u : in) work += u.k1 - u.k0 + ends;
  std::vector<Unit> runs[kDies];
  for (const Unit& u : in) {
    runs[std::min(kDies - 1, done * kDies / work)].push_back(u);
    done += u.k1 - u.k0 + ends;
  }
  size_t most = 0;
  for (auto& r : runs) {
    std::stable_sort(r.begin(), r.end(), [](const Unit& p, const Unit& q) { return p.k1 - p.k0 > q.k1 - q.k0; });
    most = std::max(most, r.size());
  }
  std::vector<Unit> out;
  out.reserve(most * kDies);
  for (size_t k = 0; k < most; ++k)
    for (auto& r : runs) out.push_back(k < r.size() ? r[k] : Unit{});
  return out;
}
uint64_t up(uint64_t n, uint64_t to) { return (n + to - 1) / to * to; }
// Elements from row to row: whole lines of 128 bytes.  (An odd number of them, so that a tile's rows lie in other channels of the caches,
// gave nothing: rows of 2048 elements, 2.4 ms a step either way.)
uint32_t leading(uint32_t n) { return (uint32_t)up(n, kDepth); }

}  // namespace
}  // namespace rotconv

using namespace rotconv;

extern "C" {

int train_matrices_create(const train_matrix* matrices, int count, int grad_dtype, train_matrices** out) {
  if (!matrices || !out) return ROTCONV_ERR_NULL;
  if (count < 1) return ROTCONV_ERR_SHAPE;
  if (grad_dtype != ROTCONV_F32 && grad_dtype != ROTCONV_BF16) return ROTCONV_ERR_UNSUPPORTED;
  const uintptr_t ge = grad_dtype == ROTCONV_BF16 ? 2 : 4;
  uint64_t total = 0, nturn = 0, nsquare = 0, nsmall = 0, nwide = 0, all = 0, depth = 0, reach = 0;
  for (int k = 0; k < count; ++k) {
    const train_matrix& t = matrices[k];
    if (!t.param || !t.grad) return ROTCONV_ERR_NULL;
    if (t.count < 1 || t.rows < 1 || t.cols < 1) return ROTCONV_ERR_SHAPE;
    const uint64_t n = std::min(t.rows, t.cols), m = std::max(t.rows, t.cols), c = t.count;
    if (n > 32768 || m > (1u << 24) || c > (1ull << 40) / (n * m)) return ROTCONV_ERR_SHAPE;
    if (!(t.weight_decay >= 0.f && t.weight_decay <= FLT_MAX) || !(std::fabs(t.scale) <= FLT_MAX) || t.reserved != 0 || misaligned(t.param, 4) ||
        misaligned(t.grad, ge) || misaligned(t.copy, 2))
      return ROTCONV_ERR_UNSUPPORTED;
    const uint64_t tn = (n + kTile - 1) / kTile, tm = (m + kTile - 1) / kTile, ts = (n + kSmall - 1) / kSmall;
    nturn += c * (up(n, kTurn) / kTurn) * (up(m, kTurn) / kTurn);
    nsquare += c * tn * (tn + 1) / 2, nsmall += c * ts * (ts + 1) / 2, nwide += c * tn * tm;
    depth += c * tn * (tn + 1) / 2 * (up(m, kDepth) / kDepth);
    reach += c * tn * tm * (up(n, kDepth) / kDepth);
    all += c, total += c * n * m;
    if (all > 65535 || std::max(std::max(nturn, 16 * nsquare), std::max(nsmall, nwide)) > kMostWorkgroups) return ROTCONV_ERR_SHAPE;
  }
  // The momentum's chunks: from 1024 elements (fewer leave lanes idle) to 16384 where there are many.
  uint32_t size = 1024;
  while (size < 16384 && total / size > 2048) size *= 2;
  // Steps of a unit of A: so that all units together fill the chip evenly, but no fewer than pay for the sums' way through memory.
  const uint64_t most = std::max<uint64_t>(12, (depth + kSlots - 1) / kSlots);
  const bool small = nsquare < kSlots, wide = reach >= nwide * kDeep;
  bool least = true;
  uint32_t widest = 0;
  for (int k = 0; k < count; ++k) {
    const uint32_t n = std::min(matrices[k].rows, matrices[k].cols), m = std::max(matrices[k].rows, matrices[k].cols);
    least = least && n <= kLeastRows && m <= kLeastCols;
    widest = std::max(widest, (n > 32 ? 2 : 1) * ((m + 31) / 32));
  }
  train_matrices* l = nullptr;
  try {
    // Nothing that a step writes may be there twice: two workgroups would write it.
    std::vector<std::pair<uintptr_t, uintptr_t>> written;
    for (int k = 0; k < count; ++k) {
      const train_matrix& t = matrices[k];
      const uintptr_t n = (uintptr_t)t.count * (uintptr_t)t.rows * (uintptr_t)t.cols, p = reinterpret_cast<uintptr_t>(t.param);
      written.emplace_back(p, p + n * sizeof(float));
      if (t.copy) written.emplace_back(reinterpret_cast<uintptr_t>(t.copy), reinterpret_cast<uintptr_t>(t.copy) + n * sizeof(uint16_t));
    }
    std::sort(written.begin(), written.end());
    for (size_t k = 1; k < written.size(); ++k)
      if (written[k].first < written[k - 1].second) return ROTCONV_ERR_UNSUPPORTED;
    std::vector<Matrix> mats;
    std::vector<Tile> chunk, turn;
    std::vector<Unit> gram, poly, apply, last;
    std::vector<Join> join;
    mats.reserve(all), turn.reserve(nturn), apply.reserve(nwide);
    uint64_t base = 0, at = 0;
    auto room = [&](uint64_t bytes) {
      const uint64_t here = at;
      at = up(at + bytes, 256);
      return here;
    };
    for (int k = 0; k < count; ++k) {
      const train_matrix& t = matrices[k];
      const uint64_t each = (uint64_t)t.rows * t.cols;
      for (int i = 0; i < t.count; ++i) {
        Matrix x = {};
        x.p = t.param + i * each;
        x.g = static_cast<const char*>(t.grad) + i * each * ge;
        x.copy = t.copy ? t.copy + i * each : nullptr;
        x.pos = base + i * each;
        x.rows = t.rows, x.cols = t.cols, x.tall = t.rows > t.cols;
        x.n = std::min(t.rows, t.cols), x.m = std::max(t.rows, t.cols);
        x.ldn = leading(x.n), x.ldm = leading(x.m);
        x.vec = !misaligned(x.g, 4 * ge) && x.pos % 4 == 0;
        x.even = !misaligned(x.p, 16) && !misaligned(x.copy, 16) && x.cols % 8 == 0;
        x.wd = t.weight_decay, x.scale = t.scale;
        x.first = (uint32_t)chunk.size(), x.chunks = (uint32_t)((each + size - 1) / size);
        const uint64_t wide_bytes = (uint64_t)x.n * x.ldm * sizeof(half), square_bytes = (uint64_t)x.n * x.ldn * sizeof(half);
        x.x[0] = room(wide_bytes), x.x[1] = room(wide_bytes), x.low = room(wide_bytes);
        x.a = room(square_bytes), x.b = room(square_bytes);
        x.da = room(x.ldn * sizeof(float)), x.db = room(x.ldn * sizeof(float));
        const uint32_t id = (uint32_t)mats.size();
        for (uint32_t c = 0; c < x.chunks; ++c) chunk.push_back(Tile{id, c, 0});
        for (uint32_t r = 0; r * kTurn < x.rows; ++r)
          for (uint32_t c = 0; c * kTurn < x.cols; ++c) turn.push_back(Tile{id, r, c});
        mats.push_back(x);
      }
      base += up(each * t.count, kPad);
    }
    // Units of the products, neighbours with operands in common; the parts of A's tiles by their columns of X.
    std::vector<uint32_t> order(mats.size());
    for (uint32_t k = 0; k < order.size(); ++k) order[k] = k;
    std::stable_sort(order.begin(), order.end(), [&](uint32_t p, uint32_t q) { return mats[p].n > mats[q].n; });
    uint32_t places = 0;
    for (uint32_t id : order) {
      const Matrix& x = mats[id];
      const uint32_t tiles = (x.n + kTile - 1) / kTile, deep = (uint32_t)(up(x.m, kDepth) / kDepth), parts = (uint32_t)((deep + most - 1) / most);
      const uint32_t first = places;
      for (uint32_t q = 0; q < parts; ++q) {
        uint32_t tile = 0;
        for (uint32_t r = 0; r < tiles; ++r)
          for (uint32_t c = r; c < tiles; ++c, ++tile)
            gram.push_back(Unit{id, r, c, (uint32_t)((uint64_t)deep * q / parts), (uint32_t)((uint64_t)deep * (q + 1) / parts),
                                parts > 1 ? first + tile * parts + q : kWhole});
      }
      if (parts > 1) {
        for (uint32_t r = 0; r < tiles; ++r)
          for (uint32_t c = r; c < tiles; ++c, places += parts) join.push_back(Join{id, r, c, places, parts});
      }
      const uint32_t steps = (uint32_t)(up(x.n, kDepth) / kDepth), edge = small ? kSmall : kTile;
      for (uint32_t r = 0; r * edge < x.n; ++r)
        for (uint32_t c = r; c * edge < x.n; ++c) poly.push_back(Unit{id, r, c, 0, steps, kWhole});
      const uint32_t across = wide ? kWide : kTile;
      for (uint32_t c = 0; c * across < x.m; ++c)
        for (uint32_t r = 0; r < tiles; ++r) apply.push_back(Unit{id, r, c, 0, steps, kWhole});
      for (uint32_t c = 0; c * kTile < x.m; ++c)
        for (uint32_t r = 0; r < tiles; ++r) last.push_back(Unit{id, r, c, 0, steps, kWhole});
    }
    // (the last product, which waits for the parameters, takes its units as they are listed: 130 us for the stack, 140 and more dealt)
    gram = by_die(gram, 32), poly = by_die(poly, 8), apply = by_die(apply, 4);
    if (std::max(std::max(gram.size(), poly.size()), std::max(apply.size(), chunk.size())) > kMostWorkgroups) return ROTCONV_ERR_SHAPE;
    const uint64_t sums = room(chunk.size() * sizeof(double)), part_bytes = room((uint64_t)places * kTile * kTile * sizeof(float));
    l = new train_matrices;
    l->bf16 = grad_dtype == ROTCONV_BF16;
    l->elements = base;
    l->sums = sums, l->parts = part_bytes, l->workspace = at;
    l->size = size, l->small = small, l->wide = wide;
    if (least) {
      l->least = (uint32_t)mats.size(), l->widest = widest, l->workspace = 256;          // (nothing of it is used)
    }
    l->nchunk = (uint32_t)chunk.size(), l->nturn = (uint32_t)turn.size(), l->ngram = (uint32_t)gram.size();
    l->npoly = (uint32_t)poly.size(), l->napply = (uint32_t)apply.size(), l->nlast = (uint32_t)last.size();
    l->njoin = (uint32_t)join.size();
    const std::vector<uint32_t> tickets(kTicketWords, 0);
    const size_t tables = tickets.size() * sizeof(uint32_t) + mats.size() * sizeof(Matrix) + (chunk.size() + turn.size()) * sizeof(Tile) +
                          (gram.size() + poly.size() + apply.size() + last.size()) * sizeof(Unit) + join.size() * sizeof(Join);
    bool ok = hipGetDevice(&l->device) == hipSuccess &&
              hipMalloc(&l->memory, tables) == hipSuccess;
    if (ok) {
      char* p = static_cast<char*>(l->memory);
      auto put = [&](const void* from, size_t bytes) {
        void* to = p;
        ok = ok && (bytes == 0 || hipMemcpy(to, from, bytes, hipMemcpyHostToDevice) == hipSuccess);
        p += bytes;
        return to;
      };
      l->tickets = static_cast<uint32_t*>(put(tickets.data(), tickets.size() * sizeof(uint32_t)));
      l->matrices = static_cast<Matrix*>(put(mats.data(), mats.size() * sizeof(Matrix)));
      l->chunk = static_cast<Tile*>(put(chunk.data(), chunk.size() * sizeof(Tile)));
      l->turn = static_cast<Tile*>(put(turn.data(), turn.size() * sizeof(Tile)));
      l->gram = static_cast<Unit*>(put(gram.data(), gram.size() * sizeof(Unit)));
      l->poly = static_cast<Unit*>(put(poly.data(), poly.size() * sizeof(Unit)));
      l->apply = static_cast<Unit*>(put(apply.data(), apply.size() * sizeof(Unit)));
      l->last = static_cast<Unit*>(put(last.data(), last.size() * sizeof(Unit)));
      l->join = static_cast<Join*>(put(join.data(), join.size() * sizeof(Join)));
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
  uint32_t* tickets = o->keep ? nullptr : l->tickets;
  if (l->least) {
    auto kernel = l->widest <= 16 ? (l->bf16 ? k_least<uint16_t, 1> : k_least<float, 1>)
                  : l->widest <= 32 ? (l->bf16 ? k_least<uint16_t, 2> : k_least<float, 2>) : (l->bf16 ? k_least<uint16_t, 4> : k_least<float, 4>);
    kernel<<<l->least, kLeastThreads, 0, st>>>(l->matrices, *o, momentum, control, tickets);
    return finish();
  }
  char* w = static_cast<char*>(ws);
  double* sums = reinterpret_cast<double*>(w + l->sums);
  f4* parts = reinterpret_cast<f4*>(w + l->parts);
  auto first = l->bf16 ? k_momentum<uint16_t> : k_momentum<float>;
  first<<<l->nchunk, kThreads, 0, st>>>(l->matrices, l->chunk, *o, l->size, momentum, control, sums);
  auto start = l->bf16 ? k_start<uint16_t> : k_start<float>;
  start<<<l->nturn, kThreads, 0, st>>>(l->matrices, l->turn, *o, momentum, control, sums, w);
  auto poly = l->small ? k_product<kPoly, 64, 64, 2, 2, kDepth, 2> : k_product<kPoly, 128, 128, 2, 2, kDepth, 2>;
  auto apply = l->wide ? k_product<kApply, 128, kWide, 2, 2, 32, 3> : k_product<kApply, 128, 128, 2, 2, 32, 3>;
  for (int k = 0; k < o->steps; ++k) {
    k_product<kGram, 128, 128, 2, 2, kDepth, 2><<<l->ngram, kThreads, 0, st>>>(l->matrices, l->gram, w, k % 2, parts, control, tickets);
    if (l->njoin) k_join<<<16 * l->njoin, 64, 0, st>>>(l->matrices, l->join, w, parts, control);
    poly<<<l->npoly, kThreads, 0, st>>>(l->matrices, l->poly, w, k % 2, parts, control, tickets);
    if (k + 1 < o->steps)
      apply<<<l->napply, kThreads, 0, st>>>(l->matrices, l->apply, w, k % 2, parts, control, tickets);
    else
      k_product<kLast, 128, 128, 2, 2, kDepth, 2><<<l->nlast, kThreads, 0, st>>>(l->matrices, l->last, w, k % 2, parts, control, tickets);
  }
  return finish();
}

}  // extern "C"
