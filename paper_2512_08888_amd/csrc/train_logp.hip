// Log-probabilities of labels, forward and backward: their launches, and the entry points of these and of the policy loss (see
// include/unettrain.h).  The kernels are train_logp.h's.
#include <initializer_list>

#include "train_logp.h"

namespace rotconv {
namespace {

int finish() { return hipGetLastError() == hipSuccess ? ROTCONV_OK : ROTCONV_ERR_LAUNCH; }
bool refused(int N, int K, size_t P) {
  return N < 1 || K < 1 || P < 1 || K > (1 << 24) || P > 0x7fffffffull || (uint64_t)N * P > 0x7fffffffull;
}
// The sums of a launch's workgroups; behind them the shares of few long rows (fp32 rows have the most parts) and their labels' logits.
constexpr size_t kSums = (size_t)kMostBlocks * 4 * sizeof(double);
size_t workspace(size_t rows, int K) {
  const int parts = parts_of(rows, K / Vec<float>::V + 2);
  return kSums + (parts > 1 ? rows * parts * sizeof(float4) + kFewRows * sizeof(float) : 0);
}
void place(LossArgs& g, void* ws) {
  char* w = static_cast<char*>(ws);
  g.part = reinterpret_cast<double*>(w);
  g.taken = reinterpret_cast<float*>(w + kSums);
  g.shares = reinterpret_cast<float4*>(w + kSums + kFewRows * sizeof(float));
}

template <typename T>
int check(const LossArgs& g, int N, int K, size_t P, int layout) {
  if (refused(N, K, P)) return ROTCONV_ERR_SHAPE;
  if (layout != TRAIN_NCHW && layout != TRAIN_NHWC) return ROTCONV_ERR_UNSUPPORTED;
  if (misaligned(g.z, sizeof(T)) || misaligned(g.dz, sizeof(T)) || misaligned(g.labels, 4)) return ROTCONV_ERR_UNSUPPORTED;
  for (const float* p : {g.stat, g.ent, g.dlogp, g.dent, g.adv, g.old, g.ref, g.w, (const float*)g.logp, (const float*)g.ent_out, (const float*)g.stat_out})
    if (misaligned(p, 4)) return ROTCONV_ERR_UNSUPPORTED;
  return ROTCONV_OK;
}
struct Span {
  const void* p;                       // NULL: none
  size_t bytes;
};
// Whether something that a call writes lies in what it reads, or in another thing that it writes.
bool overlapping(std::initializer_list<Span> written, std::initializer_list<Span> read) {
  auto meet = [](const Span& a, const Span& b) {
    const uintptr_t p = reinterpret_cast<uintptr_t>(a.p), q = reinterpret_cast<uintptr_t>(b.p);
    return a.p && b.p && p < q + b.bytes && q < p + a.bytes;
  };
  for (const Span* a = written.begin(); a != written.end(); ++a) {
    for (const Span* b = written.begin(); b != a; ++b)
      if (meet(*a, *b)) return true;
    for (const Span& b : read)
      if (meet(*a, b)) return true;
  }
  return false;
}
LossArgs arguments(const void* z, void* dz, const int32_t* labels, int N, int K, size_t P) {
  LossArgs g = {};
  g.z = z, g.dz = dz, g.labels = labels, g.K = K, g.P = P, g.rows = (size_t)N * P;
  g.alike = (reinterpret_cast<uintptr_t>(z) - reinterpret_cast<uintptr_t>(dz)) % 16 == 0;
  return g;
}
bool in_rows(int layout, size_t P) { return layout == TRAIN_NHWC || P == 1; }

template <typename T>
int logp_fwd_t(const T* z, const int32_t* labels, float* logp, float* entropy, float* stat, int N, int K, size_t P, int layout, void* ws,
               size_t ws_bytes, void* stream) {
  if (!z || !labels || !logp) return ROTCONV_ERR_NULL;
  LossArgs g = arguments(z, nullptr, labels, N, K, P);
  g.logp = logp, g.ent_out = entropy, g.stat_out = stat;
  if (int e = check<T>(g, N, K, P, layout)) return e;
  if (!ws || misaligned(ws, 16) || ws_bytes < workspace(g.rows, K)) return ROTCONV_ERR_WORKSPACE;
  const size_t row = g.rows * 4, all = g.rows * K * sizeof(T);
  if (overlapping({{logp, row}, {entropy, row}, {stat, 2 * row}, {ws, workspace(g.rows, K)}}, {{z, all}, {labels, row}}))
    return ROTCONV_ERR_UNSUPPORTED;
  place(g, ws);
  unsigned blocks;
  launch_loss<T, kFwd>(g, in_rows(layout, P), &blocks, static_cast<hipStream_t>(stream));
  return finish();
}
template <typename T>
int logp_bwd_t(const T* z, const int32_t* labels, const float* stat, const float* entropy, const float* dlogp, const float* dentropy, T* dz,
               int N, int K, size_t P, int layout, void* stream) {
  if (!z || !labels || !stat || !dlogp || !dz || (dentropy && !entropy)) return ROTCONV_ERR_NULL;
  LossArgs g = arguments(z, dz, labels, N, K, P);
  g.stat = stat, g.ent = entropy, g.dlogp = dlogp, g.dent = dentropy;
  if (int e = check<T>(g, N, K, P, layout)) return e;
  const size_t row = g.rows * 4, all = g.rows * K * sizeof(T);
  if (overlapping({{dz, all}}, {{z == dz ? nullptr : z, all}, {labels, row}, {stat, 2 * row}, {dlogp, row}, {dentropy, row},
                                {dentropy ? entropy : nullptr, row}}))
    return ROTCONV_ERR_UNSUPPORTED;
  unsigned blocks;
  launch_loss<T, kBwd>(g, in_rows(layout, P), &blocks, static_cast<hipStream_t>(stream));
  return finish();
}
template <typename T>
int policy_loss_t(const T* z, const int32_t* labels, const float* advantage, const float* logp_old, const float* logp_ref, const float* weight,
                  float* out, T* dz, float* logp, int N, int K, size_t P, int layout, const train_policy* o, void* ws, size_t ws_bytes,
                  void* stream) {
  if (!z || !labels || !advantage || !out || !o || (o->kl != 0.f && !logp_ref)) return ROTCONV_ERR_NULL;
  LossArgs g = arguments(z, dz, labels, N, K, P);
  g.adv = advantage, g.old = logp_old, g.ref = logp_ref, g.w = weight, g.logp = logp;
  if (int e = check<T>(g, N, K, P, layout)) return e;
  if (!(o->clip_low >= 0.f && o->clip_low <= 1.f) || !(o->clip_high >= 0.f && o->clip_high <= FLT_MAX) || !(o->kl >= 0.f && o->kl <= FLT_MAX) ||
      !(o->entropy >= 0.f && o->entropy <= FLT_MAX) || (o->per_image != 0 && o->per_image != 1) || o->reserved != 0 ||
      misaligned(out, 4))
    return ROTCONV_ERR_UNSUPPORTED;
  if (!ws || misaligned(ws, 16) || ws_bytes < workspace(g.rows, K)) return ROTCONV_ERR_WORKSPACE;
  const size_t row = g.rows * 4, all = g.rows * K * sizeof(T);
  if (overlapping({{dz, all}, {logp, row}, {out, 4 * sizeof(float)}, {ws, workspace(g.rows, K)}},
                  {{z == dz ? nullptr : z, all}, {labels, row}, {advantage, o->per_image ? (size_t)N * 4 : row}, {logp_old, row}, {logp_ref, row},
                   {weight, row}}))
    return ROTCONV_ERR_UNSUPPORTED;
  g.per_image = o->per_image, g.low = 1.f - o->clip_low, g.high = 1.f + o->clip_high, g.kl = o->kl, g.entc = o->entropy;
  g.unit = (float)(1.0 / ((double)N * (double)P));
  place(g, ws);
  launch_policy(g, sizeof(T) == 2, in_rows(layout, P), out, static_cast<hipStream_t>(stream));
  return finish();
}

}  // namespace
}  // namespace rotconv

using namespace rotconv;

extern "C" {

size_t train_logp_workspace_bytes(int N, int K, size_t P) { return refused(N, K, P) ? 0 : workspace((size_t)N * P, K); }

int train_logp_fwd(const float* logits, const int32_t* labels, float* logp, float* entropy, float* stat, int N, int K, size_t P, int layout,
                   void* ws, size_t ws_bytes, void* stream) {
  return logp_fwd_t(logits, labels, logp, entropy, stat, N, K, P, layout, ws, ws_bytes, stream);
}
int train_logp_fwd_bf16(const uint16_t* logits, const int32_t* labels, float* logp, float* entropy, float* stat, int N, int K, size_t P,
                        int layout, void* ws, size_t ws_bytes, void* stream) {
  return logp_fwd_t(logits, labels, logp, entropy, stat, N, K, P, layout, ws, ws_bytes, stream);
}
int train_logp_bwd(const float* logits, const int32_t* labels, const float* stat, const float* entropy, const float* dlogp,
                   const float* dentropy, float* dlogits, int N, int K, size_t P, int layout, void* stream) {
  return logp_bwd_t(logits, labels, stat, entropy, dlogp, dentropy, dlogits, N, K, P, layout, stream);
}
int train_logp_bwd_bf16(const uint16_t* logits, const int32_t* labels, const float* stat, const float* entropy, const float* dlogp,
                        const float* dentropy, uint16_t* dlogits, int N, int K, size_t P, int layout, void* stream) {
  return logp_bwd_t(logits, labels, stat, entropy, dlogp, dentropy, dlogits, N, K, P, layout, stream);
}
int train_policy_loss(const float* logits, const int32_t* labels, const float* advantage, const float* logp_old, const float* logp_ref,
                      const float* weight, float* out, float* dlogits, float* logp, int N, int K, size_t P, int layout,
                      const train_policy* options, void* ws, size_t ws_bytes, void* stream) {
  return policy_loss_t(logits, labels, advantage, logp_old, logp_ref, weight, out, dlogits, logp, N, K, P, layout, options, ws, ws_bytes,
                       stream);
}
int train_policy_loss_bf16(const uint16_t* logits, const int32_t* labels, const float* advantage, const float* logp_old, const float* logp_ref,
                           const float* weight, float* out, uint16_t* dlogits, float* logp, int N, int K, size_t P, int layout,
                           const train_policy* options, void* ws, size_t ws_bytes, void* stream) {
  return policy_loss_t(logits, labels, advantage, logp_old, logp_ref, weight, out, dlogits, logp, N, K, P, layout, options, ws, ws_bytes,
                       stream);
}

}  // extern "C"
