// Group normalisation with an activation, forward and backward (see include/unettrain.h).
//
// A workgroup takes a part of one group's map (NCHW) or of a run of whole groups' channels (channels last) into
// registers, sums it, and normalises it from there, so that the map is read once and written once: HBM bound, two bytes or
// four an element each way and some ten operations (twenty backward, and two maps read).  A call is
//   one launch, where a group (or run) fits one workgroup;
//   one, between one that empties slots and one for what was put off, where its parts exchange their sums (kFused);
//   two, where the map is small enough to be read again from the caches: sums, map (kTwo);
//   three, where a group has more parts than wait for one another: sums, their join, the map again (kSums).
// Backward, the last of these launches forms dgamma and dbeta, from the sums of every part of every channel.
//
// Measured, of a copy's 5.7 TB/s: forward bf16 4x128x256x256 in 32 groups 27 us (5.0 TB/s), fp32 4x64x512x512 101 us (5.3);
// backward bf16 4x64x512x512 83 us (4.8), fp32 143 us (5.6), channels last fp32 4x256x128x128 48 us (4.2); small maps by their
// launches: fp32 64x16x16 4 us, bf16 3x60x101x75 channels last 12 us.
//
// The wait is bounded and never needed for the result: a workgroup whose neighbours have not answered in time leaves its
// part to the launch behind, which finds all sums there.  So the kernel ends whatever else runs on the device and in
// whatever order its workgroups start.
//
// A part's forward sums are its mean and the squared deviations from it.  Deviations are taken from a point that a few values far
// from the others hardly move: the mean of the first vectors of a wave, channels last of a lane's first four pixels; parts, waves
// and rows are joined by their means' distances.  So sums of squares and squares of sums do not cancel, wherever a map's values
// lie and whichever of them is far out.  (From the part's first element, with that one 1000 deviations out, rstd of fp32
// 4x64x512x512 was off by 2.6e-3; now by 1.7e-7.  Of all maps tried the worst is off by 2e-6.)
#include <hip/hip_runtime.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstdint>

#include "glue_elt.h"
#include "rotconv.h"
#include "unettrain.h"

namespace rotconv {
namespace {

constexpr int kThreads = 512, kWaves = kThreads / 64;
constexpr int kMaxTeam = kThreads / 4;       // channels that a workgroup holds at once (NCHW), four lanes each at least
constexpr int kBatch = 4;                    // vectors under way at a time where a map is read without being held
// Workgroups that wait for one another, at most: as many as are on the device at a time, two to a CU.  (Three launches against
// one with 512 parts: backward fp32 64x1024x512 in 4 groups 121 and 96 us, channels last 2x64x512x512 in 2 150 and 119;
// with 256 parts 64 and 49.)
constexpr int kMaxSplit = 512;
constexpr int kOver = 18;                     // (kMaxSplit - 1) * kMaxSplit < 2^kOver
constexpr int kMaxRun = 1024;                // channels of a run (channels last)
// Of a map, up to which a shared group takes two launches.  (Two, and one that waits between two small ones: fp32 64x128x128
// in 4 groups, 4 MB, 9.2 and 11.7 us forward, 10.3 and 13.2 backward; bf16 channels last 4x64x128x128 in 8, 8 MB, 13.5 and
// 15.5, 19.2 and 20.8; fp32 4x64x128x128 in 4, 17 MB, 16.2 and 13.0, 20.4 and 15.6.  Of thirteen other maps, the six of 2 to 8 MB
// gain 0.6 to 3.3 us by two, one of 10.5 MB 1.4 forward and 0.5 backward; the six of 12 to 19 MB lose 0.8 to 6.0 but for one direction
// of two of them, 1.4 and 1.3.)
constexpr size_t kTwoBytes = 8u << 20;
constexpr int kMaxSlots = 2048;              // sums that a workgroup collects (channels last: of every group of its run)

int finish() { return hipGetLastError() == hipSuccess ? ROTCONV_OK : ROTCONV_ERR_LAUNCH; }

// ---- elements -------------------------------------------------------------------------------------
typedef uint32_t u4a __attribute__((ext_vector_type(4), aligned(2)));     // global memory takes any alignment
typedef uint32_t u2a __attribute__((ext_vector_type(2), aligned(2)));
typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
typedef float fl2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {          // nearest even, NaN stays NaN
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(fl2{a, b}, bf2));
}

// A map is read once: past the caches (nontemporal; backward of 4x64x512x512 bf16: 88 us without, 78 us with it)
template <typename T, typename E>
__device__ __forceinline__ T get_vector(const E* p) {
  return __builtin_nontemporal_load(reinterpret_cast<const T*>(p));
}

// V neighbouring elements as they lie in memory
template <typename E, int V> struct Raw;
template <int V> struct Raw<float, V> {
  static_assert(V == 4 || V == 1, "");
  uint32_t w[V];
  __device__ __forceinline__ void load(const float* p) {
    if constexpr (V == 4) {
      const u4a a = get_vector<u4a>(p);
#pragma unroll
      for (int k = 0; k < 4; ++k) w[k] = a[k];
    } else {
      w[0] = __float_as_uint(*p);
    }
  }
  __device__ __forceinline__ float get(int k) const { return __uint_as_float(w[k]); }
  __device__ __forceinline__ void set(int k, float v) { w[k] = __float_as_uint(v); }
  static __device__ __forceinline__ void store(float* p, const float* v) {
    if constexpr (V == 4) {
      *reinterpret_cast<u4a*>(p) = u4a{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
    } else {
      *p = v[0];
    }
  }
};
template <int V> struct Raw<uint16_t, V> {
  static_assert(V == 8 || V == 4 || V == 1, "");
  uint32_t w[(V + 1) / 2];
  __device__ __forceinline__ void load(const uint16_t* p) {
    if constexpr (V == 8) {
      const u4a a = get_vector<u4a>(p);
#pragma unroll
      for (int k = 0; k < 4; ++k) w[k] = a[k];
    } else if constexpr (V == 4) {
      const u2a a = get_vector<u2a>(p);
      w[0] = a[0], w[1] = a[1];
    } else {
      w[0] = *p;
    }
  }
  __device__ __forceinline__ float get(int k) const { return __uint_as_float(k % 2 ? w[k / 2] & 0xffff0000u : w[k / 2] << 16); }
  static __device__ __forceinline__ void store(uint16_t* p, const float* v) {
    if constexpr (V == 8) {
      *reinterpret_cast<u4a*>(p) = u4a{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
    } else if constexpr (V == 4) {
      *reinterpret_cast<u2a*>(p) = u2a{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
    } else {
      *p = (uint16_t)pack_bf16(v[0], v[0]);
    }
  }
};

// ---- the formula ----------------------------------------------------------------------------------
__device__ __forceinline__ float normalised(float x, float mean, float rstd) {
#pragma clang fp contract(off)
  return (x - mean) * rstd;
}
__device__ __forceinline__ float affine(float xh, float gamma, float beta) {
#pragma clang fp contract(off)
  return xh * gamma + beta;
}
// The exponential's argument is rounded once, which makes it off by |z| / 2 of its last bit; where z is so negative that this is much,
// z * sigmoid(z) and its slope are so small that it stays below 2^-24 of 1.  With the argument in two parts SiLU takes 3 % longer in
// fp32 (4x64x512x512 forward 105.6 us instead of 102.2) and 9 to 16 % in bf16, whose results lose it anyway.  The reciprocal
// instruction is off by one of its last bits.
__device__ __forceinline__ float sigmoid(float z) { return __builtin_amdgcn_rcpf(1.f + __expf(-z)); }
template <int ACT>
__device__ __forceinline__ float activate(float z) {
  if (ACT == TRAIN_ACT_RELU) return z <= 0.f ? 0.f : z;
  if (ACT == TRAIN_ACT_SILU) return z * sigmoid(z);
  return z;
}
template <int ACT>
__device__ __forceinline__ float through(float dy, float z) {      // dy * act'(z)
#pragma clang fp contract(off)
  if (ACT == TRAIN_ACT_RELU) return z > 0.f ? dy : 0.f;
  if (ACT == TRAIN_ACT_SILU) {
    const float s = sigmoid(z);
    return dy * (s * fmaf(z, 1.f - s, 1.f));
  }
  return dy;
}
// What an element adds to the sums of its channel.  Operations are fused or not as written: a part has the same sums
// whichever workgroup forms them.
__device__ __forceinline__ void add_fwd(float x, float first, float& s, float& s2) {
#pragma clang fp contract(off)
  const float d = x - first;
  s += d;
  s2 = fmaf(d, d, s2);
}
__device__ __forceinline__ void add_bwd(float xh, float dz, float& s, float& s2) {
#pragma clang fp contract(off)
  s += dz;
  s2 = fmaf(dz, xh, s2);
}

// The sum of dz over a part of a channel.  A ReLU's comparison leaves out an element whose z is NaN as if it were dead; where x, the
// statistics, gamma or beta make it so, the sum is NaN: xh is then too, and the sum of dz * xh with it, or gamma or beta themselves.
template <int ACT>
__device__ __forceinline__ float with_nan(float s, float s2, float gamma, float beta) {
  return ACT == TRAIN_ACT_RELU && (s2 != s2 || gamma != gamma || beta != beta) ? NAN : s;
}

// ---- sums -----------------------------------------------------------------------------------------
struct Pair {            // forward: mean, squared deviations from it; backward: sum of dz (or t), sum of dz * xh (or t * xh)
  float a, b;
};

// A lane's value moved within its row of sixteen lanes
template <int CTRL>
__device__ __forceinline__ float moved(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}
constexpr int kSwap1 = 0xb1, kSwap2 = 0x4e, kMirror8 = 0x141, kMirror16 = 0x140;     // lanes 1 0 3 2; 2 3 0 1; 7 .. 0; 15 .. 0
__device__ __forceinline__ float lane_of(float v, int lane) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), lane)); }
// over aligned runs of `width` lanes (4, 8, 16, 32 or 64; the same for the whole wave), in all of them
__device__ __forceinline__ float lanes_sum(float v, int width) {
  v += moved<kSwap1>(v);
  v += moved<kSwap2>(v);
  if (width == 4) return v;
  v += moved<kMirror8>(v);
  if (width == 8) return v;
  v += moved<kMirror16>(v);
  if (width == 16) return v;
  if (width == 32) return v + __shfl_xor(v, 16);
  return (lane_of(v, 0) + lane_of(v, 16)) + (lane_of(v, 32) + lane_of(v, 48));
}
__device__ __forceinline__ float wave_sum(float v) { return lanes_sum(v, 64); }

// Mean and squared deviations of `count` parts of size(i) elements, `total` together.  By one wave; the same in all lanes.
template <typename Get, typename Size>
__device__ __forceinline__ Pair join(int count, float total, Get get, Size size) {
  const float ref = get(0).a;
  float s = 0.f;
  for (int i = threadIdx.x % 64; i < count; i += 64) s += size(i) * (get(i).a - ref);
  const float mean = ref + wave_sum(s) / total;
  s = 0.f;
  float t = 0.f;                         // what the first mean lacks: much of its last bits where part 0 is far from the others
  for (int i = threadIdx.x % 64; i < count; i += 64) {
    const Pair p = get(i);
    const float d = p.a - mean, w = size(i) * d;
    t += w;
    s += p.b + w * d;
  }
  t = wave_sum(t);
  return Pair{mean + t / total, wave_sum(s) - t * (t / total)};
}
// The same of N parts by every lane for itself, read once
template <int N, typename Get, typename Size>
__device__ __forceinline__ Pair join_few(float total, Get get, Size size) {
  Pair o[N];
  float n[N], s = 0.f, t = 0.f, m2 = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) o[i] = get(i), n[i] = size(i);
#pragma unroll
  for (int i = 0; i < N; ++i) s += n[i] * (o[i].a - o[0].a);
  const float per = total > 0.f ? 1.f / total : 0.f, mean = o[0].a + s * per;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float d = o[i].a - mean, w = n[i] * d;
    t += w;
    m2 += o[i].b + w * d;
  }
  return Pair{mean + t * per, m2 - t * (t * per)};
}
template <typename Get>
__device__ __forceinline__ Pair add(int count, Get get) {
  float a = 0.f, b = 0.f;
  for (int i = threadIdx.x % 64; i < count; i += 64) {
    const Pair p = get(i);
    a += p.a, b += p.b;
  }
  return Pair{wave_sum(a), wave_sum(b)};
}

// ---- exchange -------------------------------------------------------------------------------------
// A slot is empty (all ones) until its owner writes it; a NaN is written in one fixed form, so that it never looks empty.
// A workgroup that has not seen all its slots in time writes nothing but its number into a list; the launch after that
// finds every slot full and does what is on the list.  late[0]: how many, from late[1] on: which.
constexpr unsigned long long kEmpty = ~0ull;
__device__ __forceinline__ uint32_t plain_bits(float v) { return v != v ? 0x7fc00000u : __float_as_uint(v); }
__device__ __forceinline__ void put(unsigned long long* slot, Pair p) {
  const unsigned long long v = (unsigned long long)plain_bits(p.b) << 32 | plain_bits(p.a);
  __hip_atomic_store(slot, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
// The value of a slot, waiting until `deadline` (of the constant clock); false: still empty
__device__ __forceinline__ bool get(const unsigned long long* slot, long long deadline, Pair* p) {
  for (;;) {
    const unsigned long long v = __hip_atomic_load(slot, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (v != kEmpty) {
      *p = Pair{__uint_as_float((uint32_t)v), __uint_as_float((uint32_t)(v >> 32))};
      return true;
    }
    if ((long long)wall_clock64() >= deadline) return false;
    __builtin_amdgcn_s_sleep(2);
  }
}
__global__ __launch_bounds__(256) void k_gn_empty(unsigned long long* slots, int n, uint32_t* late) {
  for (int i = blockIdx.x * 256 + threadIdx.x; i < n; i += gridDim.x * 256) slots[i] = kEmpty;
  if (blockIdx.x == 0 && threadIdx.x == 0) late[0] = 0;
}

// Makes the compiler forget what it knows of a register: the map then starts from the elements as loaded, instead of from
// every intermediate value of the sums kept alive across the wait (twice the registers, and spills).
__device__ __forceinline__ void forget(uint32_t& v) { asm volatile("" : "+v"(v)); }
template <typename R>
__device__ __forceinline__ void forget_vector(R& r) {
#pragma unroll
  for (unsigned k = 0; k < sizeof(r.w) / 4; ++k) forget(r.w[k]);
}
template <typename R, int J>
__device__ __forceinline__ void forget(R (&r)[J]) {
#pragma unroll
  for (int j = 0; j < J; ++j) forget_vector(r[j]);
}

enum Mode { kFused, kTwo, kSums };

struct Gn {
  // the problem
  int N, C, G, cg;
  size_t P;
  float eps;
  int act;
  // how it is cut: `split` workgroups for each group (NCHW) or run of channels (channels last)
  int mode, split, vec, per;           // per: vectors that a lane holds of each map
  int team_log, pieces;                // NCHW: lanes of a channel's piece (their logarithm), pieces of a channel
  size_t step;                         // NCHW: pixels of a piece (the last may have fewer)
  // Elements (NCHW) or pixels (channels last) of a workgroup's part: every period-th has `size_last`, the others `size`.
  // (For x < kMaxSplit: x / period == x * over >> kOver.)
  int period, over;
  float size, size_last;
  int one;                             // channels last: a vector's channels are of one group
  int run, runs, rows;                 // channels last: channels of a run, runs, pixels that a workgroup holds at once
  int wait;                            // ticks (10 ns) before a workgroup does without its neighbours
};
struct Maps {
  const void *x, *dy;
  void* out;                           // y or dx
  const float *gamma, *beta;
  float *mean, *rstd;                  // written forward (or NULL), read backward
  float *dgamma, *dbeta;               // backward, or NULL
  Pair* part;                          // see parts_of
  unsigned long long* slots;
  uint32_t* late;
  const float2* stat;                  // in three launches: mean and rstd forward, the two means of the gradient backward
};

__device__ __forceinline__ void put_off(const Maps& m) {
  m.late[1 + atomicAdd(m.late, 1u)] = (blockIdx.z * gridDim.y + blockIdx.y) * gridDim.x + blockIdx.x;
}
struct Parts {           // where the sums of part i of channel (NCHW forward: of group) c of image n lie
  int nhwc, per;
  size_t C;
  __device__ __forceinline__ size_t at(size_t n, size_t c, int i) const {
    return nhwc ? (n * per + i) * C + c : (n * C + c) * per + i;
  }
};

__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
  return v;
}
// over a workgroup of 256
__device__ __forceinline__ double block_sum(double v) {
  __shared__ double red[4];
  v = wave_sum(v);
  __syncthreads();
  if (threadIdx.x % 64 == 0) red[threadIdx.x / 64] = v;
  __syncthreads();
  return (red[0] + red[1]) + (red[2] + red[3]);
}
// dbeta and dgamma of channel c, by one wave
__device__ __forceinline__ void channel_gradient(const Gn& q, const Maps& m, const Parts& where, size_t c) {
  double s1 = 0, s2 = 0;
  for (int i = threadIdx.x % 64; i < q.N * where.per; i += 64) {
    const Pair p = m.part[where.at(i / where.per, c, i % where.per)];
    s1 += p.a;
    s2 += p.b;
  }
  s1 = wave_sum(s1);
  s2 = wave_sum(s2);
  if (threadIdx.x % 64) return;
  if (m.dbeta) m.dbeta[c] = (float)s1;
  if (m.dgamma) m.dgamma[c] = (float)s2;
}

// ---- NCHW -----------------------------------------------------------------------------------------
// A team of lanes (4 to 64, or the workgroup) holds one piece of one channel, `per` vectors a lane and the elements
// beyond the last whole vector one a lane.  Unit u of a group is piece u % pieces of channel u / pieces; workgroup k
// holds the units from k * (512 / team) on.
template <typename E, int V, int J, bool BWD, int ACT>
struct Nchw {
  const Gn& q;
  const Maps& m;
  size_t group;          // n * G + g
  int g, lane, unit0;    // unit0: of this lane's team in workgroup 0
  // what a workgroup holds: the first unit's address (the same for all lanes), a lane's offset from there
  size_t base = 0;
  uint32_t off = 0;
  Raw<E, V> x[J], dy[J];               // (dy: backward)
  float x1 = 0.f, dy1 = 0.f, ga = 1.f, be = 0.f, mu = 0.f, r = 0.f;
  int len = 0;           // 0: a team without a unit

  __device__ __forceinline__ Nchw(const Gn& q_, const Maps& m_, size_t n, int g_) : q(q_), m(m_), g(g_) {
    group = n * q.G + g;
    lane = threadIdx.x & (team() - 1);
    unit0 = threadIdx.x >> q.team_log;
  }
  __device__ __forceinline__ int team() const { return 1 << q.team_log; }
  __device__ __forceinline__ int units() const { return q.cg * q.pieces; }
  __device__ __forceinline__ int teams() const { return kThreads >> q.team_log; }
  __device__ __forceinline__ bool has(int j) const { return (lane + (j << q.team_log)) * V + V <= len; }
  __device__ __forceinline__ bool has_tail() const { return V > 1 && lane < len % V; }
  // a lane's vector j: a scalar step from its first
  template <typename T>
  __device__ __forceinline__ T* at(T* p, int j) const { return p + (uint32_t)((j << q.team_log) * V) + (off + (uint32_t)lane * V); }
  __device__ __forceinline__ uint32_t at_tail() const { return off + (uint32_t)(len - len % V + lane); }
  __device__ __forceinline__ void place(int k) {
    const int u0 = k * teams();                   // one piece, or pieces == 1
    const int cl0 = q.pieces == 1 ? u0 : q.split <= kMaxSplit ? k * q.over >> kOver : k / q.pieces;
    const int piece = q.pieces == 1 ? 0 : k - cl0 * q.pieces;
    base = (group * q.cg + cl0) * q.P + piece * q.step;
    const bool active = u0 + unit0 < units();
    const int cl = active ? unit0 : 0;
    const int c = g * q.cg + cl0 + cl;
    len = active ? (int)min(q.step, q.P - piece * q.step) : 0;
    off = (uint32_t)cl * (uint32_t)q.P;                                          // less than 512 * per * V
    if (m.gamma) ga = m.gamma[c];
    if (m.beta) be = m.beta[c];
    if (BWD) mu = m.mean[group], r = m.rstd[group];
  }
  // vectors first .. first + J of each lane
  __device__ __forceinline__ bool has(int first, int j) const { return (first == 0 || first + j < q.per) && has(first + j); }
  __device__ __forceinline__ void load(int first) {
    const E* xp = static_cast<const E*>(m.x) + base;
    const E* dp = static_cast<const E*>(m.dy) + base;
#pragma unroll
    for (int j = 0; j < J; ++j)
      if (has(first, j)) {
        x[j].load(at(xp, first + j));
        if (BWD) dy[j].load(at(dp, first + j));
      }
  }
  __device__ __forceinline__ void load_tail() {
    if (has_tail()) {
      x1 = Elt<E>::ld(static_cast<const E*>(m.x) + base + at_tail());
      if (BWD) dy1 = Elt<E>::ld(static_cast<const E*>(m.dy) + base + at_tail());
    }
  }
  // What the map needs of an element: in fp32 the sums leave xh and dz in the registers of x and dy.
  static constexpr bool FORM = BWD && sizeof(E) == 4;
  __device__ __forceinline__ void form(float& xv, float& dv) const {
    xv = normalised(xv, mu, r);
    dv = through<ACT>(dv, affine(xv, ga, be));
  }
  // Lanes that share a unit and need no barrier to add up: a team, or a wave of one
  __device__ __forceinline__ int width() const { return min(team(), 64); }
  // Of `vectors` of a unit that its lanes take in turn, those of this lane's wave (of its team, where that is less than a wave)
  __device__ __forceinline__ int share(int vectors) const {
    if (team() <= 64) return vectors;
    const int wave = threadIdx.x / 64;
    return (vectors >> q.team_log) * 64 + min(max((vectors & (team() - 1)) - wave * 64, 0), 64);
  }
  // A point near the mean of what this lane's team or wave holds of its unit: the mean of the first kNear vectors of each lane,
  // which are loaded.  (Not of all: that is two operations an element more.  The deviations' sums lose the more digits the smaller
  // a part of all this is, at worst the sixteenth, or in three launches the 64th.)
  static constexpr int kNear = J > 4 ? 1 : J;
  __device__ __forceinline__ float centre() const {
    const float first = len ? Elt<E>::ld(static_cast<const E*>(m.x) + base + off) : 0.f;
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < kNear; ++j)
      if (has(0, j)) {
#pragma unroll
        for (int e = 0; e < V; ++e) s += x[j].get(e) - first;
      }
    const int near = share(min(len / V, kNear << q.team_log));
    return first + lanes_sum(s, width()) / (float)max(near * V, 1);
  }
  __device__ __forceinline__ void add_one(float& xv, float& dv, float ref, Pair& s) const {
    if (BWD) {
      form(xv, dv);
      add_bwd(xv, dv, s.a, s.b);
    } else {
      add_fwd(xv, ref, s.a, s.b);
    }
  }
  __device__ __forceinline__ void add_loaded(int first, float ref, Pair& s) {
#pragma unroll
    for (int j = 0; j < J; ++j)
      if (has(first, j)) {
        if (FORM) forget_vector(x[j]), forget_vector(dy[j]);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          float xv = x[j].get(e), dv = BWD ? dy[j].get(e) : 0.f;
          add_one(xv, dv, ref, s);
          if constexpr (FORM) x[j].set(e, xv), dy[j].set(e, dv);
        }
        if (FORM) forget_vector(x[j]), forget_vector(dy[j]);
      }
  }
  __device__ __forceinline__ void add_tail(float ref, Pair& s) {
    if (has_tail()) {
      float xv = x1, dv = dy1;
      add_one(xv, dv, ref, s);
      if constexpr (FORM) x1 = xv, dy1 = dv;
    }
  }
  // Part k's sums, in all lanes, from every lane's own (of deviations from `ref`).  Ends with a barrier behind every use
  // of `red`.
  __device__ __forceinline__ Pair sums(Pair* red, int k, float ref, Pair own) {
    float s = own.a, s2 = own.b;
    s = lanes_sum(s, width());
    s2 = lanes_sum(s2, width());
    Pair p;
    if (BWD) {
      if (team() > 64) {                      // one unit
        if (threadIdx.x % 64 == 0) red[threadIdx.x / 64] = Pair{s, s2};
        __syncthreads();
        s = s2 = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) s += red[w].a, s2 += red[w].b;
        __syncthreads();
      }
      s = with_nan<ACT>(s, s2, ga, be);
      if (len && lane == 0) m.part[group * q.cg * q.pieces + k * teams() + unit0] = Pair{s, s2};
      p = Pair{s * ga, s2 * ga};
    } else {
      const int n = share(len / V) * V + (threadIdx.x < 64 || team() <= 64 ? len % V : 0);
      const float d = s / (float)max(n, 1);
      p = Pair{ref + d, s2 - s * d};
      if (team() > 64) {                      // one unit: its eight waves' parts
        if (threadIdx.x % 64 == 0) red[threadIdx.x / 64] = p, red[kWaves + threadIdx.x / 64].a = (float)n;
        __syncthreads();
        p = join_few<kWaves>((float)len, [&](int w) { return red[w]; }, [&](int w) { return red[kWaves + w].a; });
        __syncthreads();
      }
    }
    if (team() > 64) return p;
    if (len && lane == 0) red[unit0] = p;
    __syncthreads();
    const int count = min(teams(), units() - k * teams());
    if (BWD) {
      p = add(count, [&](int i) { return red[i]; });
    } else {
      const float each = (float)q.P;
      p = join(count, each * (float)count, [&](int i) { return red[i]; }, [&](int) { return each; });
    }
    __syncthreads();
    return p;
  }
  template <bool FORMED>
  __device__ __forceinline__ float one(float xv, float dv, float a, float b) const {
    if (!BWD) return activate<ACT>(affine(normalised(xv, a, b), ga, be));
    if (!FORMED) form(xv, dv);
    return r * (dv * ga - a - xv * b);
  }
  template <bool FORMED>
  __device__ __forceinline__ void vector(E* op, const Raw<E, V>& xr, const Raw<E, V>& dr, int j, float a, float b) const {
    float v[V];
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = one<FORMED>(xr.get(e), BWD ? dr.get(e) : 0.f, a, b);
    Raw<E, V>::store(at(op, j), v);
  }
  __device__ __forceinline__ void map(float a, float b) {
    forget(x);
    if (BWD) forget(dy);
    E* op = static_cast<E*>(m.out) + base;
#pragma unroll
    for (int j = 0; j < J; ++j)
      if (has(j)) vector<FORM>(op, x[j], dy[j], j, a, b);
    if (has_tail()) Elt<E>::st(op + at_tail(), one<FORM>(x1, dy1, a, b));
  }
  // the same of a part that is placed but not held
  __device__ __forceinline__ void map_from_memory(float a, float b) {
    E* op = static_cast<E*>(m.out) + base;
    for (int first = 0; first < q.per; first += J) {
      load(first);
#pragma unroll
      for (int j = 0; j < J; ++j)
        if (has(first, j)) vector<false>(op, x[j], dy[j], first + j, a, b);
    }
    load_tail();
    if (has_tail()) Elt<E>::st(op + at_tail(), one<false>(x1, dy1, a, b));
  }
};

__device__ __forceinline__ float size_of(const Gn& q, int part) {
  return part - (part * q.over >> kOver) * q.period == q.period - 1 ? q.size_last : q.size;
}

// A group's statistics (forward), or its gradient's means, from its workgroups' sums
template <bool BWD, typename Part>
__device__ __forceinline__ Pair settle(const Part& w, const Pair* all, Pair p, size_t group, bool tell) {
  const Gn& q = w.q;
  const float M = (float)q.cg * (float)q.P;
  if (q.split > 1) {
    if (BWD) p = add(q.split, [&](int i) { return all[i]; });
    else p = join(q.split, M, [&](int i) { return all[i]; }, [&](int i) { return size_of(q, i); });
  }
  if (BWD) return Pair{p.a / M, p.b / M};
  p.b = 1.f / sqrtf(p.b / M + q.eps);
  if (tell && threadIdx.x == 0) {
    if (w.m.mean) w.m.mean[group] = p.a;
    if (w.m.rstd) w.m.rstd[group] = p.b;
  }
  return p;
}

// The sums of all parts of a group into `all`; false (in every lane) where the deadline came first.  Starts and ends with
// a barrier.
__device__ __forceinline__ bool collect(const unsigned long long* slots, int count, long long deadline, Pair* all, int* missing) {
  if (threadIdx.x == 0) *missing = 0;
  __syncthreads();
  for (int i = threadIdx.x; i < count; i += kThreads) {
    Pair o;
    if (!get(slots + i, deadline, &o)) *missing = 1;
    all[i] = o;
  }
  __syncthreads();
  return !*missing;
}

// Sums, exchange and map of a part that stays in registers; in two launches the sums alone.  HBM bound: bf16 4x128x256x256 in
// 32 groups forward 25 us (5.4 TB/s), 4x64x512x512 backward 80 us (5.0).  512 threads: a group of the deep levels fits one
// workgroup, and two of sixteen vectors a lane (backward eight of each map) fill a CU's registers.
template <typename E, int V, int J, bool BWD, int ACT>
__global__ __launch_bounds__(kThreads, BWD || J == 16 ? 4 : 6) void k_gn_nchw(Gn q, Maps m) {
  __shared__ Pair red[kMaxTeam];
  __shared__ Pair all[kMaxSplit];
  __shared__ int missing;
  const int k = blockIdx.x;
  Nchw<E, V, J, BWD, ACT> w(q, m, blockIdx.z, blockIdx.y);
  w.place(k);
  w.load(0);
  w.load_tail();
  const float ref = BWD ? 0.f : w.centre();
  Pair p = {0.f, 0.f};
  w.add_loaded(0, ref, p);
  w.add_tail(ref, p);
  p = w.sums(red, k, ref, p);
  if (q.split > 1) {
    unsigned long long* slots = m.slots + w.group * q.split;
    if (threadIdx.x == 0) put(slots + k, p);
    if (q.mode == kTwo) return;
    if (!collect(slots, q.split, (long long)wall_clock64() + q.wait, all, &missing)) {
      if (threadIdx.x == 0) put_off(m);
      return;
    }
  }
  p = settle<BWD>(w, all, p, w.group, k == 0);
  w.map(p.a, p.b);
}

// The sums alone, of parts that need not fit the registers
template <typename E, int V, bool BWD, int ACT>
__global__ __launch_bounds__(kThreads) void k_gn_nchw_sums(Gn q, Maps m) {
  __shared__ Pair red[kMaxTeam];
  Nchw<E, V, kBatch, BWD, ACT> w(q, m, blockIdx.z, blockIdx.y);
  w.place(blockIdx.x);
  w.load(0);
  const float ref = BWD ? 0.f : w.centre();
  Pair p = {0.f, 0.f};
  for (int first = 0; first < q.per; first += kBatch) {
    Pair some = {0.f, 0.f};
    if (first) w.load(first);
    w.add_loaded(first, ref, some);
    p.a += some.a, p.b += some.b;
  }
  w.load_tail();
  w.add_tail(ref, p);
  p = w.sums(red, blockIdx.x, ref, p);
  if (!BWD && threadIdx.x == 0) m.part[w.group * q.split + blockIdx.x] = p;
}

// The map of parts that nobody holds: of those that the launch before has put off, or, in two or three launches, of all.
// Every slot is full now.  But in three launches also the channels' gradients, which need every part's sums.
template <typename E, int V, bool BWD, int ACT>
__global__ __launch_bounds__(kThreads) void k_gn_nchw_map(Gn q, Maps m) {
  __shared__ Pair all[kMaxSplit];
  __shared__ int missing;
  if (q.mode == kSums) {
    Nchw<E, V, kBatch, BWD, ACT> w(q, m, blockIdx.z, blockIdx.y);
    w.place(blockIdx.x);
    const float2 p = m.stat[w.group];
    w.map_from_memory(p.x, p.y);
    return;
  }
  if (BWD && (m.dgamma || m.dbeta))
    for (size_t c = blockIdx.x * kWaves + threadIdx.x / 64; c < (size_t)q.C; c += gridDim.x * kWaves)
      channel_gradient(q, m, Parts{0, q.pieces, (size_t)q.C}, c);
  const uint32_t count = q.mode == kTwo ? gridDim.x : q.split > 1 ? m.late[0] : 0;
  for (uint32_t i = blockIdx.x; i < count; i += gridDim.x) {
    const uint32_t wg = q.mode == kTwo ? i : m.late[1 + i];
    const uint32_t group = wg / q.split;
    const int k = wg % q.split;
    Nchw<E, V, kBatch, BWD, ACT> w(q, m, group / q.G, group % q.G);
    w.place(k);
    collect(m.slots + (size_t)group * q.split, q.split, 0, all, &missing);
    const Pair p = settle<BWD>(w, all, Pair{}, group, k == 0);
    w.map_from_memory(p.a, p.b);
    __syncthreads();
  }
}

// ---- channels last --------------------------------------------------------------------------------
// A workgroup holds q.rows * J pixels of a run of channels; a lane the same V channels of each of its J pixels.  ONE: these
// are of one group, whose statistics a lane then holds once.
template <typename E, int V, int J, bool ONE, bool BWD, int ACT>
struct Nhwc {
  static constexpr int S = ONE ? 1 : V;
  const Gn& q;
  const Maps& m;
  size_t n;
  int c0;                // first channel of the run
  int width;             // channels of the run that exist
  int c, row;            // this lane's first channel, within the run; its row
  bool in;
  // what a workgroup holds: its first pixel's address (the same for all lanes), its pixels
  size_t base = 0;
  int left = 0, each = 0, more = 0;    // each: whole rows of them, more: pixels beyond
  Raw<E, V> x[J], dy[J];               // (dy: backward)

  __device__ __forceinline__ Nhwc(const Gn& q_, const Maps& m_, size_t n_, int run) : q(q_), m(m_), n(n_) {
    c0 = run * q.run;
    width = min(q.run, q.C - c0);
    const int cols = q.run / V;
    c = (int)(threadIdx.x % cols) * V;
    row = (int)(threadIdx.x / cols);
    in = row < q.rows && c < width;
  }
  __device__ __forceinline__ bool has(int j) const { return in && j * q.rows + row < left; }
  template <typename T>
  __device__ __forceinline__ T* at(T* p, int j) const {
    return p + (size_t)(j * q.rows) * q.C + ((uint32_t)row * (uint32_t)q.C + (uint32_t)c);
  }
  __device__ __forceinline__ void place(int k) {
    const size_t p0 = (size_t)k * q.rows * q.per;
    base = (n * q.P + p0) * q.C + c0;
    left = (int)min((size_t)q.rows * q.per, q.P - p0);
    each = left / q.rows;
    more = left % q.rows;
  }
  // pixels first .. first + J of each lane
  __device__ __forceinline__ bool has(int first, int j) const { return (first == 0 || first + j < q.per) && has(first + j); }
  __device__ __forceinline__ void load(int first) {
    const E* xp = static_cast<const E*>(m.x) + base;
    const E* dp = static_cast<const E*>(m.dy) + base;
#pragma unroll
    for (int j = 0; j < J; ++j)
      if (has(first, j)) {
        x[j].load(at(xp, first + j));
        if (BWD) dy[j].load(at(dp, first + j));
      }
  }
  __device__ __forceinline__ size_t group(int e) const { return n * q.G + (c0 + min(c + e, width - 1)) / q.cg; }
  struct Scale {
    float ga[V], be[V], mean[S], rstd[S];
  };
  // What the map needs of an element: in fp32 the sums leave xh and dz in the registers of x and dy.
  static constexpr bool FORM = BWD && sizeof(E) == 4;
  __device__ __forceinline__ void form(float& xv, float& dv, const Scale& t, int e) const {
    const int h = ONE ? 0 : e;
    xv = normalised(xv, t.mean[h], t.rstd[h]);
    dv = through<ACT>(dv, affine(xv, t.ga[e], t.be[e]));
  }
  __device__ __forceinline__ Scale scale() const {
    Scale s;
#pragma unroll
    for (int e = 0; e < V; ++e) {
      s.ga[e] = m.gamma && in ? m.gamma[c0 + c + e] : 1.f;
      s.be[e] = m.beta && in ? m.beta[c0 + c + e] : 0.f;
    }
#pragma unroll
    for (int e = 0; e < S; ++e) s.mean[e] = BWD ? m.mean[group(e)] : 0.f, s.rstd[e] = BWD ? m.rstd[group(e)] : 0.f;
    return s;
  }

  // The points that deviations are taken from: this lane's first pixel, and from its fifth pixel on the means of the first four
  // (recentre), so that whichever is far out weighs no more than a sixteenth.
  __device__ __forceinline__ void centres(float* ref) const {
#pragma unroll
    for (int e = 0; e < V; ++e) ref[e] = has(0, 0) ? x[0].get(e) : 0.f;
  }
  __device__ __forceinline__ void recentre(int taken, float* ref, float* s, float* s2) const {
    const float n = min(pixels(row), (float)taken), per = n > 0.f ? 1.f / n : 0.f;
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const float d = s[e] * per, to = ref[e] + d;
      s2[e] -= s[e] * d;
      s[e] = n * (d - (to - ref[e]));
      ref[e] = to;
    }
  }
  __device__ __forceinline__ void add_loaded(int first, float* ref, const Scale& t, float* s, float* s2) {
#pragma unroll
    for (int j = 0; j < J; ++j) {
      if (!BWD && j == kBatch) recentre(kBatch, ref, s, s2);
      if (has(first, j)) {
        if (FORM) forget_vector(x[j]), forget_vector(dy[j]);
#pragma unroll
        for (int e = 0; e < V; ++e) {
          float xv = x[j].get(e), dv = BWD ? dy[j].get(e) : 0.f;
          if (BWD) {
            form(xv, dv, t, e);
            add_bwd(xv, dv, s[e], s2[e]);
            if constexpr (FORM) x[j].set(e, xv), dy[j].set(e, dv);
          } else {
            add_fwd(xv, ref[e], s[e], s2[e]);
          }
        }
        if (FORM) forget_vector(x[j]), forget_vector(dy[j]);
      }
    }
  }
  // Pixels of a row
  __device__ __forceinline__ float pixels(int i) const { return (float)(each + (i < more)); }
  // One channel's sums over count of the rows, or of what they have been joined to: get(i), of size(i) pixels.  From deviations
  // from the first: there are at most sixteen, and it weighs as much as another.
  template <typename Get, typename Size>
  static __device__ __forceinline__ Pair over_rows(int count, float& total, Get get, Size size) {
    const float ref = get(0).a;
    float s = 0.f, s2 = 0.f;
    total = 0.f;
    for (int i = 0; i < count; ++i) {
      const Pair o = get(i);
      const float n = size(i), d = o.a - ref, w = n * d;
      total += n;
      s += w;
      s2 += o.b + w * d;
    }
    const float d = total > 0.f ? s / total : 0.f;
    return Pair{ref + d, s2 - s * d};
  }
  template <typename Get>
  static __device__ __forceinline__ Pair add_rows(int count, Get get) {
    Pair t = {0.f, 0.f};
    for (int i = 0; i < count; ++i) {
      const Pair o = get(i);
      t.a += o.a, t.b += o.b;
    }
    return t;
  }
  // Sums of every channel of the run over this part's pixels, left in out[0 .. width), from every lane's own (of deviations
  // from `ref`).  buf: kThreads * V pairs; out: kMaxRun.
  __device__ __forceinline__ void sums(Pair* buf, Pair* out, const float* ref, float* s, float* s2) {
    // A lane's V pairs lie together, two at a time at places that turn with the lane (64 bytes apart, the same two of eight
    // lanes would share their banks).
    auto place_of = [](int l, int e) { return V < 8 ? l * V + e : l * V + (((e >> 1) ^ ((l >> 2) & 3)) << 1 | (e & 1)); };
    if (!BWD) {
      const float n = pixels(row), per = n > 0.f ? 1.f / n : 0.f;
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float d = s[e] * per;
        s2[e] -= s[e] * d;
        s[e] = ref[e] + d;
      }
    }
    __syncthreads();
    if (in) {
      if constexpr (V == 1) {
        buf[threadIdx.x] = Pair{s[0], s2[0]};
      } else {
#pragma unroll
        for (int e = 0; e < V; e += 2)
          *reinterpret_cast<f4*>(buf + place_of(threadIdx.x, e)) = f4{s[e], s2[e], s[e + 1], s2[e + 1]};
      }
    }
    __syncthreads();
    // rows together: as many lanes to a channel as there are; the pixels of what each joins lie behind `out` (width <= 256 then)
    const int lanes = kThreads / width, ch = threadIdx.x % width, part = threadIdx.x / width, cols = q.run / V;
    float* const sizes = reinterpret_cast<float*>(out + kMaxRun / 2);
    int rows = q.rows;
    if (lanes > 1) {
      const int count = part < lanes && part < rows ? (rows - 1 - part) / lanes + 1 : 0;
      auto get = [&](int i) { return buf[place_of((part + i * lanes) * cols + ch / V, ch % V)]; };
      Pair t = {0.f, 0.f};
      float total = 0.f;
      if (count) {
        // (lanes is more than two thirds of 512 / width, rows at most 512 * V / width: count is at most 1.5 * V)
        if (BWD) t = add_rows(count, get);
        else if (more == 0) t = over_rows(count, total, get, [&](int) { return (float)each; });
        else t = over_rows(count, total, get, [&](int i) { return pixels(part + i * lanes); });
      }
      rows = min(lanes, rows);
      __syncthreads();
      if (part < rows) {
        buf[part * q.run + ch] = t;
        if (!BWD && ch == 0) sizes[part] = total;
      }
      __syncthreads();
    }
    if (!BWD && lanes > 1 && rows > 4) {
      // sixteen lanes to a channel
      const int lane = threadIdx.x % 16;
      for (int i = threadIdx.x / 16; i < width; i += kThreads / 16) {
        auto get = [&](int j) { return buf[j * q.run + i]; };
        const float ref = get(0).a;
        float s = 0.f, t = 0.f, m2 = 0.f;
        for (int j = lane; j < rows; j += 16) s += sizes[j] * (get(j).a - ref);
        const float mean = ref + lanes_sum(s, 16) / (float)left;
        for (int j = lane; j < rows; j += 16) {
          const Pair o = get(j);
          const float d = o.a - mean, w = sizes[j] * d;
          t += w;
          m2 += o.b + w * d;
        }
        t = lanes_sum(t, 16);
        m2 = lanes_sum(m2, 16);
        if (lane == 0) out[i] = Pair{mean + t / (float)left, m2 - t * (t / (float)left)};
      }
    } else {
      for (int i = threadIdx.x; i < width; i += kThreads) {
        auto get = [&](int j) { return buf[lanes > 1 ? j * q.run + i : place_of(j * cols + i / V, i % V)]; };
        // (lanes == 1: width is above 256, rows at most 15)
        float total;
        Pair t = BWD ? add_rows(rows, get) : over_rows(rows, total, get, [&](int j) { return lanes > 1 ? sizes[j] : pixels(j); });
        if (BWD && ACT == TRAIN_ACT_RELU) t.a = with_nan<ACT>(t.a, t.b, m.gamma ? m.gamma[c0 + i] : 1.f, m.beta ? m.beta[c0 + i] : 0.f);
        out[i] = t;
      }
    }
    __syncthreads();
  }
  // stat(e): the group of this lane's channel e
  template <bool FORMED>
  __device__ __forceinline__ void vector(E* op, const Raw<E, V>& xr, const Raw<E, V>& dr, int j, const Scale& t, const Pair* p) const {
    float v[V];
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const int h = ONE ? 0 : e;
      float xv = xr.get(e), dv = BWD ? dr.get(e) : 0.f;
      if (!BWD) {
        v[e] = activate<ACT>(affine(normalised(xv, p[h].a, p[h].b), t.ga[e], t.be[e]));
      } else {
        if (!FORMED) form(xv, dv, t, e);
        v[e] = t.rstd[h] * (dv * t.ga[e] - p[h].a - xv * p[h].b);
      }
    }
    Raw<E, V>::store(at(op, j), v);
  }
  template <typename Stat>
  __device__ __forceinline__ void map(Stat stat) {
    forget(x);
    if (BWD) forget(dy);
    E* op = static_cast<E*>(m.out) + base;
    const Scale t = scale();
    Pair p[S];
#pragma unroll
    for (int e = 0; e < S; ++e) p[e] = stat(e);
#pragma unroll
    for (int j = 0; j < J; ++j)
      if (has(j)) vector<FORM>(op, x[j], dy[j], j, t, p);
  }
  // the same of a part that is placed but not held
  template <typename Stat>
  __device__ __forceinline__ void map_from_memory(Stat stat) {
    E* op = static_cast<E*>(m.out) + base;
    const Scale t = scale();
    Pair p[S];
#pragma unroll
    for (int e = 0; e < S; ++e) p[e] = stat(e);
    for (int first = 0; first < q.per; first += J) {
      load(first);
#pragma unroll
      for (int j = 0; j < J; ++j)
        if (has(first, j)) vector<false>(op, x[j], dy[j], first + j, t, p);
    }
  }
};

// A group's sums over its channels, of the part whose channels' sums `chan` holds.  By one wave.
template <bool BWD, typename Part>
__device__ __forceinline__ Pair of_group(const Part& w, const Pair* chan, int g, int part) {
  const int cg = w.q.cg;
  chan += g * cg;
  if (BWD)
    return add(cg, [&](int i) {
      const float ga = w.m.gamma ? w.m.gamma[w.c0 + g * cg + i] : 1.f;
      return Pair{chan[i].a * ga, chan[i].b * ga};
    });
  const float each = size_of(w.q, part);
  return join(cg, each * (float)cg, [&](int i) { return chan[i]; }, [&](int) { return each; });
}

// The statistics of a run's groups (forward), or their gradients' means, from `all` into `stat`; barriers before and after
template <bool BWD, typename Part>
__device__ __forceinline__ void settle(const Part& w, const Pair* all, Pair* stat, int run, int groups, bool tell) {
  const Gn& q = w.q;
  const float M = (float)q.cg * (float)q.P;
  __syncthreads();
  for (int g = threadIdx.x / 64; g < groups; g += kWaves) {
    Pair p;
    if (BWD) p = add(q.split, [&](int i) { return all[i * groups + g]; });
    else p = join(q.split, M, [&](int i) { return all[i * groups + g]; }, [&](int i) { return size_of(q, i) * (float)q.cg; });
    if (BWD) p = Pair{p.a / M, p.b / M};
    else p.b = 1.f / sqrtf(p.b / M + q.eps);
    if (threadIdx.x % 64 == 0) {
      stat[g] = p;
      const size_t to = w.n * q.G + (size_t)run * groups + g;
      if (!BWD && tell && w.m.mean) w.m.mean[to] = p.a;
      if (!BWD && tell && w.m.rstd) w.m.rstd[to] = p.b;
    }
  }
  __syncthreads();
}

// As k_gn_nchw, of a run of whole groups: as many channels as fill a cache line of every pixel (256 bytes instead of 128:
// backward bf16 4x128x256x256 in 8 groups 68 us instead of 57; every workgroup then collects twice the sums).  HBM bound:
// backward fp32 4x256x128x128 in 32 groups 43 us (4.7 TB/s).
template <typename E, int V, int J, bool ONE, bool BWD, int ACT>
__global__ __launch_bounds__(kThreads, 4) void k_gn_nhwc(Gn q, Maps m) {
  // 40 KB at most, four workgroups to a CU: what is collected takes the room of the lanes' sums
  constexpr int room = kThreads * V > kMaxSlots + 1 ? kThreads * V : kMaxSlots + 1;
  __shared__ __attribute__((aligned(16))) Pair buf[room];
  __shared__ Pair chan[kMaxRun];
  Pair* const all = buf;                      // [part][group]
  int* const missing = reinterpret_cast<int*>(buf + kMaxSlots);
  const int k = blockIdx.x, run = blockIdx.y;
  const int groups = q.run / q.cg;
  Nhwc<E, V, J, ONE, BWD, ACT> w(q, m, blockIdx.z, run);
  w.place(k);
  w.load(0);
  {
    float ref[V] = {}, s[V] = {}, s2[V] = {};
    if (BWD) {
      w.add_loaded(0, ref, w.scale(), s, s2);
    } else {
      w.centres(ref);
      w.add_loaded(0, ref, {}, s, s2);
    }
    w.sums(buf, chan, ref, s, s2);
  }
  if (BWD)
    for (int i = threadIdx.x; i < w.width; i += kThreads) m.part[(w.n * q.split + k) * q.C + w.c0 + i] = chan[i];
  unsigned long long* slots = m.slots + ((size_t)blockIdx.z * q.runs + run) * q.split * groups;
  for (int g = threadIdx.x / 64; g < groups; g += kWaves) {
    const Pair p = of_group<BWD>(w, chan, g, k);
    if (threadIdx.x % 64 == 0) {
      if (q.split > 1) put(slots + k * groups + g, p);
      else all[g] = p;
    }
  }
  if (q.mode == kTwo) return;
  if (q.split > 1 && !collect(slots, q.split * groups, (long long)wall_clock64() + q.wait, all, missing)) {
    if (threadIdx.x == 0) put_off(m);
    return;
  }
  settle<BWD>(w, all, chan, run, groups, k == 0);
  w.map([&](int e) { return chan[min(w.c + e, w.width - 1) / q.cg]; });
}

// The sums alone, of runs that need not be of whole groups and parts that need not fit the registers
template <typename E, int V, bool ONE, bool BWD, int ACT>
__global__ __launch_bounds__(kThreads) void k_gn_nhwc_sums(Gn q, Maps m) {
  __shared__ __attribute__((aligned(16))) Pair buf[kThreads * V];
  __shared__ Pair chan[kMaxRun];
  Nhwc<E, V, kBatch, ONE, BWD, ACT> w(q, m, blockIdx.z, blockIdx.y);
  w.place(blockIdx.x);
  float s[V] = {}, s2[V] = {};
  typename Nhwc<E, V, kBatch, ONE, BWD, ACT>::Scale t = {};
  if (BWD) t = w.scale();
  float ref[V] = {};
  w.load(0);
  if (!BWD) w.centres(ref);
  for (int first = 0; first < q.per; first += kBatch) {
    float some[V] = {}, some2[V] = {};
    if (first) w.load(first);
    w.add_loaded(first, ref, t, some, some2);
#pragma unroll
    for (int e = 0; e < V; ++e) s[e] += some[e], s2[e] += some2[e];
    if (!BWD && first == 0) w.recentre(kBatch, ref, s, s2);
  }
  w.sums(buf, chan, ref, s, s2);
  for (int i = threadIdx.x; i < w.width; i += kThreads) m.part[(w.n * q.split + blockIdx.x) * q.C + w.c0 + i] = chan[i];
}

// As k_gn_nchw_map, and bound as it is: bf16 4x64x512x512 in 16 groups, in three launches, 97 us forward and 140 backward.
template <typename E, int V, bool ONE, bool BWD, int ACT>
__global__ __launch_bounds__(kThreads) void k_gn_nhwc_map(Gn q, Maps m) {
  __shared__ Pair all[kMaxSlots];
  __shared__ Pair chan[kMaxRun];
  __shared__ int missing;
  if (q.mode == kSums) {
    Nhwc<E, V, kBatch, ONE, BWD, ACT> w(q, m, blockIdx.z, blockIdx.y);
    w.place(blockIdx.x);
    w.map_from_memory([&](int e) {
      const float2 s = m.stat[w.group(e)];
      return Pair{s.x, s.y};
    });
    return;
  }
  if (BWD && (m.dgamma || m.dbeta))
    for (size_t c = blockIdx.x * kWaves + threadIdx.x / 64; c < (size_t)q.C; c += gridDim.x * kWaves)
      channel_gradient(q, m, Parts{1, q.split, (size_t)q.C}, c);
  const int groups = q.run / q.cg;
  const uint32_t count = q.mode == kTwo ? gridDim.x : q.split > 1 ? m.late[0] : 0;
  for (uint32_t i = blockIdx.x; i < count; i += gridDim.x) {
    const uint32_t wg = q.mode == kTwo ? i : m.late[1 + i];
    const size_t cluster = wg / q.split;
    const int k = wg % q.split, run = (int)(cluster % q.runs);
    Nhwc<E, V, kBatch, ONE, BWD, ACT> w(q, m, cluster / q.runs, run);
    w.place(k);
    collect(m.slots + cluster * q.split * groups, q.split * groups, 0, all, &missing);
    settle<BWD>(w, all, chan, run, groups, k == 0);
    w.map_from_memory([&](int e) { return chan[min(w.c + e, w.width - 1) / q.cg]; });
    __syncthreads();
  }
}

// ---- joins of three-launch runs, and the channels' gradients --------------------------------------
// By workgroups of 256, each of which takes every kJoins-th task (a launch may have 2^32 threads at the most).
// 4x64x512x512 in 16 groups: 6.7 us; one wave a task, without loads under way, 44.
constexpr size_t kJoins = 1 << 20;

// A task: a group of one image
__global__ __launch_bounds__(256) void k_gn_fwd_join(const Pair* __restrict__ part, float* __restrict__ mean,
                                                     float* __restrict__ rstd, float2* __restrict__ stat, Gn q, Parts where) {
  const int chans = where.nhwc ? q.cg : 1, count = chans * q.split;
  const double M = (double)q.cg * (double)q.P;
  auto size = [&](int i) {
    if (where.nhwc) {
      const size_t all = (size_t)q.rows * q.per;
      return (double)min(all, q.P - i * all);
    }
    const int teams = kThreads >> q.team_log;
    return q.pieces > 1 ? (double)min(q.step, q.P - (i % q.pieces) * q.step) : (double)min(teams, q.cg - i * teams) * (double)q.P;
  };
  for (size_t g = blockIdx.x; g < (size_t)q.N * q.G; g += gridDim.x) {
    const size_t n = g / q.G, c0 = g % q.G * chans;
    auto get = [&](int i) { return part[where.at(n, c0 + i % chans, i / chans)]; };
    double s = 0, s2 = 0;
#pragma unroll 4
    for (int i = threadIdx.x; i < count; i += 256) s += size(i / chans) * get(i).a;
    const double mu = block_sum(s) / M;
#pragma unroll 4
    for (int i = threadIdx.x; i < count; i += 256) {
      const Pair p = get(i);
      s2 += p.b + size(i / chans) * (p.a - mu) * (p.a - mu);
    }
    s2 = block_sum(s2);
    if (threadIdx.x) continue;
    const float r = (float)(1.0 / sqrt(s2 / M + (double)q.eps));
    stat[g] = make_float2((float)mu, r);
    if (mean) mean[g] = (float)mu;
    if (rstd) rstd[g] = r;
  }
}

// The first N * G tasks: a group's two means.  The next C: a channel's dbeta and dgamma.
__global__ __launch_bounds__(256) void k_gn_bwd_join(Gn q, Maps m, Parts where, float2* __restrict__ stat) {
  const size_t groups = (size_t)q.N * q.G;
  const double M = (double)q.cg * (double)q.P;
  for (size_t w = blockIdx.x; w < groups + q.C; w += gridDim.x) {
    double s1 = 0, s2 = 0;
    if (w >= groups) {
      const size_t c = w - groups;
#pragma unroll 4
      for (int i = threadIdx.x; i < q.N * where.per; i += 256) {
        const Pair p = m.part[where.at(i / where.per, c, i % where.per)];
        s1 += p.a;
        s2 += p.b;
      }
      s1 = block_sum(s1);
      s2 = block_sum(s2);
      if (threadIdx.x == 0 && m.dbeta) m.dbeta[c] = (float)s1;
      if (threadIdx.x == 0 && m.dgamma) m.dgamma[c] = (float)s2;
      continue;
    }
    const size_t c0 = w % q.G * q.cg;
#pragma unroll 4
    for (int i = threadIdx.x; i < q.cg * where.per; i += 256) {
      const size_t c = where.nhwc ? i % q.cg : i / where.per;
      const Pair p = m.part[where.at(w / q.G, c0 + c, where.nhwc ? i / q.cg : i % where.per)];
      const double ga = m.gamma ? m.gamma[c0 + c] : 1.f;
      s1 += p.a * ga;
      s2 += p.b * ga;
    }
    s1 = block_sum(s1);
    s2 = block_sum(s2);
    if (threadIdx.x == 0) stat[w] = make_float2((float)(s1 / M), (float)(s2 / M));
  }
}

// ---- host -----------------------------------------------------------------------------------------
std::atomic<int> g_wait{10000};        // 100 us

bool shaped(int N, int C, size_t P, int groups) {
  return N >= 1 && C >= 1 && P >= 1 && groups >= 1 && groups <= C && C % groups == 0 && P < (1ull << 31) && N < 65536 && groups < 65536 && C <= (1 << 20) &&
         (size_t)N * C < (1ull << 31) && (size_t)N * C * P < (1ull << 46);
}

size_t ceil_div(size_t a, size_t b) { return (a + b - 1) / b; }

size_t workgroups(const Gn& q, int layout) { return (size_t)q.N * (layout == TRAIN_NHWC ? q.runs : q.G) * q.split; }

Gn cut_nchw(Gn q, int elem, int per, bool held) {
  const int full = 16 / elem;
  q.vec = q.P >= (size_t)full ? full : 1;
  q.per = q.vec == 1 && held ? 2 : per;           // four lanes hold the up to seven pixels
  per = q.per;
  const size_t vectors = std::max<size_t>(1, q.P / q.vec);
  if (vectors <= 64u * per) {                     // a team of a wave or less holds a channel
    q.team_log = 2;
    while (((size_t)per << q.team_log) < vectors || 1 << q.team_log < q.vec) ++q.team_log;
    q.pieces = 1;
    q.step = q.P;
  } else {
    q.team_log = 9;
    static_assert(kThreads == 1 << 9, "");
    const size_t begun = ceil_div(q.P, q.vec);    // the last vector may be part of one
    q.pieces = (int)ceil_div(begun, (size_t)kThreads * per);
    q.step = ceil_div(begun, q.pieces) * q.vec;
    if (q.pieces == 1) q.step = q.P;
  }
  const int teams = kThreads >> q.team_log;
  q.split = (int)ceil_div((size_t)q.cg * q.pieces, teams);
  q.period = q.pieces > 1 ? q.pieces : q.split;
  q.size = q.pieces > 1 ? (float)q.step : (float)teams * (float)q.P;
  q.size_last = q.pieces > 1 ? (float)(q.P - (q.pieces - 1) * q.step) : (float)(q.cg - (q.split - 1) * teams) * (float)q.P;
  return q;
}

// held: a workgroup's vectors stay in registers
Gn cut_nhwc(Gn q, int elem, int per, bool held, bool bwd) {
  q.vec = 16 / elem;
  q.one = q.cg % q.vec == 0;
  if (!q.one) {
    // several groups' statistics in a lane: fewer vectors, and backward shorter ones, for the registers
    if (q.C % q.vec || bwd) q.vec = q.C % 4 == 0 ? 4 : 1;
    q.one = q.vec == 1;
    if (held) per = q.one ? 4 : std::min(per, 8);
  }
  q.per = per;
  // the shortest run of whole groups that fills a cache line of every pixel
  const size_t longest = std::min(kMaxRun, kThreads * q.vec);
  int take = 0;
  for (int g = 1; g <= q.G && (size_t)g * q.cg <= longest && !take; ++g)
    if (q.G % g == 0 && (size_t)g * q.cg % q.vec == 0 && ((size_t)g * q.cg * elem >= 128 || g == q.G)) take = g * q.cg;
  q.mode = take ? kFused : kSums;
  q.run = take ? take : (int)std::min<size_t>(q.C, longest);
  q.runs = (int)ceil_div(q.C, q.run);
  q.rows = kThreads / (q.run / q.vec);
  q.split = (int)ceil_div(q.P, (size_t)q.rows * per);
  q.period = q.split;
  q.size = (float)(q.rows * per);
  q.size_last = (float)(q.P - (size_t)(q.split - 1) * q.rows * per);
  return q;
}

// mode kSums: in three launches
Gn cut(int N, int C, size_t P, int groups, int layout, int elem, bool bwd) {
  Gn q = {};
  q.N = N, q.C = C, q.G = groups, q.cg = C / groups, q.P = P;
  Gn best = {};
  auto with = [&](int per) { return layout == TRAIN_NHWC ? cut_nhwc(q, elem, per, true, bwd) : cut_nchw(q, elem, per, true); };
  // A group (or run) in one workgroup needs no exchange and one launch: with as many lanes as that leaves.  Else the largest
  // parts that still give every CU a workgroup, so that fewer wait for one another: forward sixteen vectors a lane, backward
  // eight of each map.  (Forward by eight and by sixteen: bf16 4x128x256x256 channels last in 8 groups 41 and 31 us, NCHW in
  // 32 groups 26.2 and 24.6; fp32 4x64x256x256 NCHW in 2 groups 31 and 24.  Backward, the same two: 55 and 62 us, 39 and 43.)
  for (int per : {2, 4, 8}) {
    best = with(per);
    if (best.split == 1) break;
  }
  // Where two launches make it, every workgroup of the map joins the sums of its run's groups for itself: half as many
  // workgroups do where the parts would else leave more than 1024 sums (channels last bf16 3x60x101x75 in 12 groups, 672 sums
  // and 1344: 11.5 and 13.2 us; 4x256x32x32 fp32 in 32 groups, 128 and 256: 10.7 and 10.0; bf16 1x128x128x128 in 64, 2048 and
  // 4096, which three launches would join: forward 17.4 and 19.1, backward 22.2 and 20.0; of eight maps of 4 to 8 MB with fewer sums
  // all but one lose 0.3 to 4.5 us with half as many).
  const bool two = (size_t)N * C * P * elem <= kTwoBytes;
  auto sums_of = [&](const Gn& g) { return (size_t)g.split * (layout == TRAIN_NHWC ? g.run / g.cg : 1); };
  if (best.split > 1)
    for (int per : {16, 8, 4, 2}) {
      if (per == 16 && bwd) continue;
      best = with(per);
      if (workgroups(best, layout) >= (two && sums_of(best) > 512 ? 128 : 256)) break;
    }
  if (best.mode == kSums || best.split > kMaxSplit || sums_of(best) > (size_t)kMaxSlots) {
    // parts of any size, a few for each CU
    for (int per = 8;; per *= 2) {
      best = layout == TRAIN_NHWC ? cut_nhwc(q, elem, per, false, bwd) : cut_nchw(q, elem, per, false);
      if (workgroups(best, layout) <= 4096 || per == 256) break;
    }
    best.mode = kSums;
  }
  if (best.mode == kFused && best.split > 1 && two) best.mode = kTwo;
  best.over = (1 << kOver) / best.period + 1;
  return best;
}

// Room for sums: every channel's pieces or splits (the channels' gradients need them), and what three launches join
size_t parts_of(const Gn& q, int layout) {
  if (layout == TRAIN_NHWC) return (size_t)q.N * q.C * q.split;
  return std::max((size_t)q.N * q.C * q.pieces, (size_t)q.N * q.G * q.split);
}
size_t round256(size_t n) { return (n + 255) / 256 * 256; }
size_t slots_of(const Gn& q, int layout) {
  if (q.mode == kSums || q.split == 1) return 0;
  return workgroups(q, layout) * (layout == TRAIN_NHWC ? q.run / q.cg : 1);
}
size_t late_bytes(const Gn& q, int layout) { return slots_of(q, layout) ? round256((1 + workgroups(q, layout)) * 4) : 0; }
size_t need(const Gn& q, int layout) {
  return round256(parts_of(q, layout) * sizeof(Pair)) + round256(slots_of(q, layout) * 8) + round256((size_t)q.N * q.G * sizeof(float2)) +
         late_bytes(q, layout);
}
bool misaligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }
bool known(int act, int layout) {
  return (act == TRAIN_ACT_NONE || act == TRAIN_ACT_RELU || act == TRAIN_ACT_SILU) && (layout == TRAIN_NCHW || layout == TRAIN_NHWC);
}

typedef void (*Kernel)(Gn, Maps);
struct Kernels {
  Kernel main, map, sums;          // held in registers; read for the map, for the sums
};
template <typename E, bool BWD, int ACT>
Kernels pick_of(const Gn& q, int layout) {
  constexpr int full = 16 / sizeof(E);
  constexpr int SUM = BWD ? ACT : TRAIN_ACT_NONE;        // forward sums know no activation
  if (layout == TRAIN_NCHW) {
    if (q.vec == 1) return {k_gn_nchw<E, 1, 2, BWD, ACT>, k_gn_nchw_map<E, 1, BWD, ACT>, k_gn_nchw_sums<E, 1, BWD, SUM>};
    if constexpr (!BWD)
      if (q.per == 16) return {k_gn_nchw<E, full, 16, BWD, ACT>, k_gn_nchw_map<E, full, BWD, ACT>, k_gn_nchw_sums<E, full, BWD, SUM>};
    return {q.per == 8 ? k_gn_nchw<E, full, 8, BWD, ACT> : q.per == 4 ? k_gn_nchw<E, full, 4, BWD, ACT> : k_gn_nchw<E, full, 2, BWD, ACT>,
            k_gn_nchw_map<E, full, BWD, ACT>, k_gn_nchw_sums<E, full, BWD, SUM>};
  }
  if (q.vec == 1) return {k_gn_nhwc<E, 1, 4, true, BWD, ACT>, k_gn_nhwc_map<E, 1, true, BWD, ACT>, k_gn_nhwc_sums<E, 1, true, BWD, SUM>};
  if constexpr (!BWD && full == 8)
    if (!q.one && q.vec == 8)
      return {q.per == 8   ? k_gn_nhwc<E, 8, 8, false, BWD, ACT>
              : q.per == 4 ? k_gn_nhwc<E, 8, 4, false, BWD, ACT>
                           : k_gn_nhwc<E, 8, 2, false, BWD, ACT>,
              k_gn_nhwc_map<E, 8, false, BWD, ACT>,
              k_gn_nhwc_sums<E, 8, false, BWD, SUM>};
  if (!q.one)
    return {q.per == 8   ? k_gn_nhwc<E, 4, 8, false, BWD, ACT>
            : q.per == 4 ? k_gn_nhwc<E, 4, 4, false, BWD, ACT>
                         : k_gn_nhwc<E, 4, 2, false, BWD, ACT>,
            k_gn_nhwc_map<E, 4, false, BWD, ACT>,
            k_gn_nhwc_sums<E, 4, false, BWD, SUM>};
  if constexpr (!BWD)
    if (q.per == 16)
      return {k_gn_nhwc<E, full, 16, true, BWD, ACT>, k_gn_nhwc_map<E, full, true, BWD, ACT>, k_gn_nhwc_sums<E, full, true, BWD, SUM>};
  return {q.per == 8   ? k_gn_nhwc<E, full, 8, true, BWD, ACT>
          : q.per == 4 ? k_gn_nhwc<E, full, 4, true, BWD, ACT>
                       : k_gn_nhwc<E, full, 2, true, BWD, ACT>,
          k_gn_nhwc_map<E, full, true, BWD, ACT>, k_gn_nhwc_sums<E, full, true, BWD, SUM>};
}
template <typename E, bool BWD>
Kernels pick(const Gn& q, int layout) {
  if (q.act == TRAIN_ACT_RELU) return pick_of<E, BWD, TRAIN_ACT_RELU>(q, layout);
  if (q.act == TRAIN_ACT_SILU) return pick_of<E, BWD, TRAIN_ACT_SILU>(q, layout);
  return pick_of<E, BWD, TRAIN_ACT_NONE>(q, layout);
}

// the main kernel once (fused), or as sums and, after `join`, as the map
template <typename E, bool BWD, typename Join>
void launch(Gn q, Maps m, int layout, hipStream_t st, Join join) {
  const Kernels kernel = pick<E, BWD>(q, layout);
  const dim3 grid(q.split, layout == TRAIN_NHWC ? q.runs : q.G, q.N);
  if (q.mode == kFused) {
    const size_t n = slots_of(q, layout);
    if (n) k_gn_empty<<<(unsigned)std::min<size_t>(ceil_div(n, 256), 256), 256, 0, st>>>(m.slots, (int)n, m.late);
    kernel.main<<<grid, kThreads, 0, st>>>(q, m);
    if (n || (BWD && (m.dgamma || m.dbeta))) kernel.map<<<64, kThreads, 0, st>>>(q, m);
    return;
  }
  if (q.mode == kTwo) {
    kernel.main<<<grid, kThreads, 0, st>>>(q, m);
    kernel.map<<<(unsigned)workgroups(q, layout), kThreads, 0, st>>>(q, m);
    return;
  }
  kernel.sums<<<grid, kThreads, 0, st>>>(q, m);
  join();
  kernel.map<<<grid, kThreads, 0, st>>>(q, m);
}

struct Scratch {
  Pair* part;
  unsigned long long* slots;
  uint32_t* late;
  float2* stat;
  Scratch(const Gn& q, int layout, void* ws) {
    char* p = static_cast<char*>(ws);
    part = reinterpret_cast<Pair*>(p);
    p += round256(parts_of(q, layout) * sizeof(Pair));
    slots = reinterpret_cast<unsigned long long*>(p);
    p += round256(slots_of(q, layout) * 8);
    late = reinterpret_cast<uint32_t*>(p);
    p += late_bytes(q, layout);
    stat = reinterpret_cast<float2*>(p);
  }
};

template <typename E>
int fwd(const E* x, const float* gamma, const float* beta, E* y, float* mean, float* rstd, int N, int C, size_t P, int groups,
        float eps, int act, int layout, void* ws, size_t ws_bytes, void* stream) {
  if (!x || !y) return ROTCONV_ERR_NULL;
  if (!shaped(N, C, P, groups)) return ROTCONV_ERR_SHAPE;
  if (!known(act, layout) || !(eps >= 0.f) || misaligned(x, sizeof(E)) || misaligned(y, sizeof(E))) return ROTCONV_ERR_UNSUPPORTED;
  if (P == 1) layout = TRAIN_NHWC;                 // the two are the same
  Gn q = cut(N, C, P, groups, layout, sizeof(E), false);
  q.eps = eps, q.act = act, q.wait = g_wait.load(std::memory_order_relaxed);
  if (!ws || misaligned(ws, 16) || ws_bytes < need(q, layout)) return ROTCONV_ERR_WORKSPACE;
  if (q.split >= 1 << 22) return ROTCONV_ERR_SHAPE;
  hipStream_t st = static_cast<hipStream_t>(stream);
  const Scratch s(q, layout, ws);
  const Maps m{x, nullptr, y, gamma, beta, mean, rstd, nullptr, nullptr, s.part, s.slots, s.late, s.stat};
  launch<E, false>(q, m, layout, st, [&] {
    const Parts where{layout, q.split, (size_t)(layout == TRAIN_NHWC ? C : groups)};
    k_gn_fwd_join<<<(unsigned)std::min((size_t)N * groups, kJoins), 256, 0, st>>>(s.part, mean, rstd, s.stat, q, where);
  });
  return finish();
}

template <typename E>
int bwd(const E* x, const E* dy, const float* gamma, const float* beta, const float* mean, const float* rstd, E* dx,
        float* dgamma, float* dbeta, int N, int C, size_t P, int groups, int act, int layout, void* ws, size_t ws_bytes,
        void* stream) {
  if (!x || !dy || !mean || !rstd || !dx) return ROTCONV_ERR_NULL;
  if (!shaped(N, C, P, groups)) return ROTCONV_ERR_SHAPE;
  if (!known(act, layout) || misaligned(x, sizeof(E)) || misaligned(dy, sizeof(E)) || misaligned(dx, sizeof(E)))
    return ROTCONV_ERR_UNSUPPORTED;
  if (P == 1) layout = TRAIN_NHWC;
  Gn q = cut(N, C, P, groups, layout, sizeof(E), true);
  q.act = act, q.wait = g_wait.load(std::memory_order_relaxed);
  if (!ws || misaligned(ws, 16) || ws_bytes < need(q, layout)) return ROTCONV_ERR_WORKSPACE;
  if (q.split >= 1 << 22) return ROTCONV_ERR_SHAPE;
  hipStream_t st = static_cast<hipStream_t>(stream);
  const Scratch s(q, layout, ws);
  const Maps m{x, dy, dx, gamma, beta, const_cast<float*>(mean), const_cast<float*>(rstd), dgamma, dbeta, s.part, s.slots, s.late, s.stat};
  launch<E, true>(q, m, layout, st, [&] {
    const Parts where{layout, layout == TRAIN_NHWC ? q.split : q.pieces, (size_t)C};
    k_gn_bwd_join<<<(unsigned)std::min((size_t)N * groups + C, kJoins), 256, 0, st>>>(q, m, where, s.stat);
  });
  return finish();
}

}  // namespace
}  // namespace rotconv

extern "C" {

size_t train_groupnorm_workspace_bytes(int N, int C, size_t P, int groups) {
  if (!rotconv::shaped(N, C, P, groups)) return 0;
  size_t n = 0;
  for (int layout : {TRAIN_NCHW, TRAIN_NHWC})
    for (int elem : {4, 2})
      for (bool bwd : {false, true}) n = std::max(n, rotconv::need(rotconv::cut(N, C, P, groups, layout, elem, bwd), layout));
  return n;
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
int train_diag_groupnorm_wait(int ticks) { return rotconv::g_wait.exchange(ticks < 0 ? 0 : ticks, std::memory_order_relaxed); }

}  // extern "C"
