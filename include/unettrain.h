/*
 * unettrain.h - C ABI of the training operators around the stack: group normalisation with an
 * activation (forward and backward), log-probabilities of labels (forward and backward) and the
 * clipped policy loss with its gradient, the norm of many gradients at once, the AdamW step over
 * many parameter tensors at once, and Muon's step over many matrices at once.
 *
 * Same conventions as rotconv.h and unetglue.h: plain C; every tensor pointer is DEVICE memory owned
 * by the caller; `stream` is a hipStream_t passed as void*; calls only enqueue (train_list_create
 * and train_matrices_create excepted: they upload tables and return when these are there); results are bitwise
 * reproducible.  Return value: a rotconv_status (ROTCONV_ERR_NULL, ROTCONV_ERR_SHAPE,
 * ROTCONV_ERR_UNSUPPORTED, ROTCONV_ERR_WORKSPACE, ROTCONV_ERR_LAUNCH).
 */
#ifndef UNETTRAIN_H
#define UNETTRAIN_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* ---- group normalisation with an activation ------------------------------------------------------
 * x holds N images of C channels of P pixels, C a multiple of `groups`.  Over each group of C / groups
 * channels of an image (M = C / groups * P values)
 *     mean = sum x / M      rstd = 1 / sqrt(sum (x - mean)^2 / M + eps)
 *     z = (x - mean) * rstd * gamma[c] + beta[c]      y = act(z)
 * z is formed in exactly this order, each operation rounded to fp32 by itself, in both directions: the
 * backward pass sees every element on the side of a ReLU's kink on which the forward pass left it.
 * gamma / beta: fp32 [C], or NULL for ones / zeros.  mean, rstd: fp32 [N, groups].
 * A NaN or an infinity makes its group's results NaN and touches no other group; an activation
 * passes a NaN on, backward too: dgamma and dbeta of the group's channels are NaN (dbeta without an activation is the sum of
 * dy whatever x holds).
 * Refused (ROTCONV_ERR_SHAPE): N or groups of 65536 or more, C above 2^20, P of 2^31 or more, N * C of 2^31 or more. */
typedef enum { TRAIN_ACT_NONE = 0, TRAIN_ACT_RELU = 1, TRAIN_ACT_SILU = 2 } train_act;
/* order of x, y, dy and dx in memory: [N][C][P] or, channels last, [N][P][C] */
typedef enum { TRAIN_NCHW = 0, TRAIN_NHWC = 1 } train_layout;

/* scratch that either direction needs, whatever the layout and storage type; 0 for extents that are refused */
size_t train_groupnorm_workspace_bytes(int N, int C, size_t P, int groups);
/* y must not overlap x; mean and rstd may be NULL where nobody needs them (inference) */
int train_groupnorm_fwd(const float* x, const float* gamma, const float* beta, float* y, float* mean, float* rstd,
                        int N, int C, size_t P, int groups, float eps, int act, int layout, void* ws, size_t ws_bytes,
                        void* stream);
/* With dz = dy * act'(z), xh = (x - mean) * rstd and t = dz * gamma[c]:
 *     dx = rstd * (t - sum t / M - xh * sum (t * xh) / M)
 *     dgamma[c] = sum over n, p of dz * xh      dbeta[c] = sum over n, p of dz
 * mean, rstd: what the forward call wrote.
 * dgamma / dbeta may be NULL.  dx may be dy itself (same address), but overlap nothing else. */
int train_groupnorm_bwd(const float* x, const float* dy, const float* gamma, const float* beta, const float* mean,
                        const float* rstd, float* dx, float* dgamma, float* dbeta, int N, int C, size_t P, int groups,
                        int act, int layout, void* ws, size_t ws_bytes, void* stream);
/* bfloat16 twins: x, y, dy, dx as bfloat16 (uint16_t holding the upper half of the fp32 bit pattern), everything
 * else fp32; arithmetic in fp32, results rounded once. */
int train_groupnorm_fwd_bf16(const uint16_t* x, const float* gamma, const float* beta, uint16_t* y, float* mean,
                             float* rstd, int N, int C, size_t P, int groups, float eps, int act, int layout, void* ws,
                             size_t ws_bytes, void* stream);
int train_groupnorm_bwd_bf16(const uint16_t* x, const uint16_t* dy, const float* gamma, const float* beta,
                             const float* mean, const float* rstd, uint16_t* dx, float* dgamma, float* dbeta, int N,
                             int C, size_t P, int groups, int act, int layout, void* ws, size_t ws_bytes,
                             void* stream);

/* Workgroups that share a group wait for one another's sums, at most this many ticks of 10 ns (10000 at first) from then
 * on, and leave their part to a second launch where that is too short: same bits, more reads.  Returns the number
 * before.  For the whole process; results do not depend on it. */
int train_diag_groupnorm_wait(int ticks);

/* ---- log-probabilities of labels, and the clipped policy loss ----------------------------------------
 * logits z hold N images of K classes of P pixels (TRAIN_NCHW: [N][K][P]; TRAIN_NHWC: [N][P][K]; tokens are images of one
 * pixel); labels int32 [N, P].  A row is a pixel's K logits.  With t the largest of a row and l = ln sum_j exp(z_j - t):
 *     logp = z_label - t - l      p_j = exp(z_j - t - l)      entropy = l - sum_j p_j (z_j - t)
 * Logits of -infinity are classes that cannot be taken: p_j = 0, and p_j ln p_j counts as 0.  A row is left out (its outputs 0,
 * its logits' gradient 0, nothing in any sum, whatever it holds) where its label lies outside 0..K-1; the notes at the calls
 * name the further ones.  A NaN or a +infinity makes its own row's results NaN.
 * What a call writes (its scratch too) overlaps nothing that it reads and nothing else that it writes, but for gradients in the place of
 * their logits, at the same address: anything else is refused (ROTCONV_ERR_UNSUPPORTED).
 * Refused (ROTCONV_ERR_SHAPE): N or K below 1, P of 0, K above 2^24, N * P of 2^31 or more. */

/* scratch that train_logp_fwd and train_policy_loss need, whatever the layout and storage type; 0 for extents that are refused.  One serves
 * calls of one stream at a time. */
size_t train_logp_workspace_bytes(int N, int K, size_t P);
/* logp, entropy: fp32 [N, P]; stat: fp32 [N, P, 2], t and l, which the backward call reads.  entropy and stat may be NULL.
 * Left out beside those without a label: rows whose logits are all -infinity (their t is kept as it is, -infinity, with l = 0; beside a NaN
 * l is NaN). */
int train_logp_fwd(const float* logits, const int32_t* labels, float* logp, float* entropy, float* stat, int N, int K,
                   size_t P, int layout, void* ws, size_t ws_bytes, void* stream);
/* dlogits_j = dlogp (1[j = label] - p_j) - dentropy p_j (ln p_j + entropy)
 * stat, entropy: what the forward call wrote.  dentropy may be NULL (none), and entropy is read only beside it.
 * dlogits may be the logits themselves (same address).  Left out too: rows whose t is -infinity with l = 0, and
 * rows whose dlogp and dentropy are 0. */
int train_logp_bwd(const float* logits, const int32_t* labels, const float* stat, const float* entropy,
                   const float* dlogp, const float* dentropy, float* dlogits, int N, int K, size_t P, int layout,
                   void* stream);

typedef struct {
  float clip_low, clip_high;   /* 0 <= clip_low <= 1, clip_high >= 0: the ratio counts from 1 - clip_low to 1 + clip_high */
  float kl;                    /* factor of the distance to the reference, >= 0; 0 without one */
  float entropy;               /* factor of the entropy (a bonus), >= 0 */
  int32_t per_image;           /* 1: advantage holds a value for each image; 0: for each row */
  int32_t reserved;            /* 0 */
} train_policy;

/* Loss and gradient in one call, for labels that were taken with log-probability logp_old.  Of a row with advantage A and weight w:
 *     r = exp(logp - logp_old)                       (1, with its gradient, where logp_old is NULL)
 *     s = min(r A, clip(r, 1 - clip_low, 1 + clip_high) A)                       (0 for A = 0)
 *     d = exp(q) - q - 1 with q = logp_ref - logp    (0 where logp_ref is NULL)
 *     out[0] = sum w (-s + kl d - entropy H)      out[1] = sum w d      out[2] = sum w H      out[3] = sum of w where s is cut
 * (H, the entropy, counts as 0 where its factor is 0, and d where kl is 0.)  s is cut where A > 0 and r > 1 + clip_high, or A < 0 and
 * r < 1 - clip_low: it has no gradient there.
 *     dlogits_j = w (G (1[j = label] - p_j) + entropy p_j (ln p_j + H)),      G = (cut ? 0 : -A r) + kl (1 - exp(q))
 * weight: fp32 [N, P], or NULL for 1 / (N P); the caller's own normalisation and mask.  Left out too: rows of weight 0, and rows
 * whose logits are all -infinity.  logp: fp32 [N, P] or NULL.  advantage: fp32 [N, P] or [N].  out: fp32 [4], sums in 64 bits.
 * dlogits may be the logits themselves; NULL where only the loss is wanted. */
int train_policy_loss(const float* logits, const int32_t* labels, const float* advantage, const float* logp_old,
                      const float* logp_ref, const float* weight, float* out, float* dlogits, float* logp, int N, int K,
                      size_t P, int layout, const train_policy* options, void* ws, size_t ws_bytes, void* stream);
/* bfloat16 twins: logits and dlogits as bfloat16, everything else fp32; arithmetic in fp32, results rounded once. */
int train_logp_fwd_bf16(const uint16_t* logits, const int32_t* labels, float* logp, float* entropy, float* stat, int N,
                        int K, size_t P, int layout, void* ws, size_t ws_bytes, void* stream);
int train_logp_bwd_bf16(const uint16_t* logits, const int32_t* labels, const float* stat, const float* entropy,
                        const float* dlogp, const float* dentropy, uint16_t* dlogits, int N, int K, size_t P, int layout,
                        void* stream);
int train_policy_loss_bf16(const uint16_t* logits, const int32_t* labels, const float* advantage, const float* logp_old,
                           const float* logp_ref, const float* weight, float* out, uint16_t* dlogits, float* logp, int N,
                           int K, size_t P, int layout, const train_policy* options, void* ws, size_t ws_bytes,
                           void* stream);

/* ---- many tensors at once -----------------------------------------------------------------------
 * A list names parameter tensors with their gradients.  It holds their addresses, not their values: the
 * caller keeps the memory in place for as long as the list is used and creates another list where it moves.  The list
 * holds the counters by which a launch's workgroups find the last of them: one list serves one stream at a time. */
typedef struct {
  float* param;            /* fp32; NULL in lists that are only measured */
  const void* grad;        /* of the list's gradient type */
  uint16_t* copy;          /* NULL, or a bfloat16 copy of param that every step refreshes (rounded to nearest even) */
  uint64_t n;              /* elements, >= 1 */
  float weight_decay;      /* of this tensor, >= 0 */
  int32_t reserved;        /* 0 */
} train_tensor;

typedef struct train_list train_list;

/* grad_dtype: ROTCONV_F32 or ROTCONV_BF16.  The list belongs to the device that is current here.  Refused (ROTCONV_ERR_SHAPE):
 * tensors of more than 2^40 elements, and lists whose norm would take 2^24 workgroups or more (16 million tensors). */
int train_list_create(const train_tensor* tensors, int count, int grad_dtype, train_list** out);
int train_list_destroy(train_list* list);
/* Elements that the states of a list span: tensor k's start at the sum of the sizes before it, each size rounded
 * up to a multiple of 32. */
uint64_t train_list_elements(const train_list* list);
size_t train_list_workspace_bytes(const train_list* list);

/* What the calls on a list read and write on the device, 64 bytes owned by the caller; train_control_init() fills
 * them.  One block serves calls of one stream at a time. */
typedef struct {
  int32_t step;            /* steps taken */
  float lr;                /* learning rate of the next step */
  float coef;              /* factor of every gradient in the next step: train_grad_norm()'s serves that step alone and can be
                            * read until the next (in further steps it counts as 1, and a skipped step sets it to 1); one that
                            * the caller writes serves until another is written */
  float norm;              /* norm of all gradients, of the last train_grad_norm() */
  int32_t nonfinite;       /* 1: that norm was not finite; the next step then changes nothing here but `skipped`, coef and this */
  int32_t skipped;         /* steps skipped so */
  int32_t reserved[2];     /* 0 */
  int32_t clip;            /* 1: coef is train_grad_norm()'s and waits for its step; 2: spent is one that a step has used */
  float spent;             /* coef is that one as long as the two have the same bits */
  int32_t reserved2[6];    /* 0 */
} train_control;

/* step (0 to 2^31 - 2) as given, lr as given, coef 1, everything else 0 */
int train_control_init(train_control* control, int step, float lr, void* stream);

/* norms[k] = sqrt(sum of grad_k^2) (fp32 [count], or NULL), control->norm = sqrt(sum of all squares), summed in 64 bits;
 * control->coef = min(1, max_norm / norm), 1 for a norm of 0; control->nonfinite (judged in 64 bits: a norm above fp32's range is
 * finite, and norm then shows an infinity).  max_norm > 0, infinity: no clipping. */
int train_grad_norm(const train_list* list, float max_norm, float* norms, train_control* control, void* ws,
                    size_t ws_bytes, void* stream);

/* One AdamW step of every tensor.  With t = control->step + 1 and g = control->coef * grad:
 *     m = beta1 * m + (1 - beta1) * g          v = beta2 * v + (1 - beta2) * g^2
 *     param -= lr * weight_decay * param + lr / (1 - beta1^t) * m / (sqrt(v) / sqrt(1 - beta2^t) + eps)
 * then control->step = t.  With control->nonfinite set it changes nothing but the control block: one more skipped, the flag cleared.
 * States, train_list_elements() elements each and zero before the first step:
 *   TRAIN_STATE_F32: m, v fp32; the scales are NULL.
 *   TRAIN_STATE_MX8: m and s = sqrt(v) (in v's place) in OCP e4m3, with one power-of-two scale (e8m0: 2^(byte - 127)) for
 *     each block of 32 elements in m_scale / v_scale [elements / 32].  A block's scale is the smallest with every value
 *     at most 448 times it.  param is updated from the unrounded m and v.  m is formed in fp32 and rounded to
 *     nearest even.  s is rounded
 *     stochastically, so that a change far smaller than the step between two codes still moves it on average: up with the
 *     probability of the part cut off, from 16 bits of a hash of (seed, t, position), and a positive s to no less than
 *     the smallest code, so that no denominator vanishes beside an m.  A NaN or an infinity makes its block NaN. */
typedef enum { TRAIN_STATE_F32 = 0, TRAIN_STATE_MX8 = 1 } train_state;
typedef struct {
  double beta1, beta2;     /* 0 <= beta < 1 */
  float eps;               /* a normal number > 0 */
  int32_t state;           /* a train_state */
  uint32_t seed;
  int32_t reserved;        /* 0 */
} train_adamw;
int train_adamw_step(const train_list* list, const train_adamw* options, void* m, void* v, uint8_t* m_scale,
                     uint8_t* v_scale, train_control* control, void* stream);

/* ---- Muon: orthogonalised updates of many matrices ---------------------------------------------------
 * Matrices with their gradients, as train_list names tensors.  A stack of `count` matrices of one shape lies in one piece,
 * each row-major; a filter bank is a matrix of output channels x taps. */
typedef struct {
  float* param;            /* fp32 [count][rows][cols] */
  const void* grad;        /* of the handle's gradient type */
  uint16_t* copy;          /* NULL, or a bfloat16 copy of param that every step refreshes (rounded to nearest even) */
  int32_t count, rows, cols;
  float weight_decay;      /* >= 0 */
  float scale;             /* factor of the orthogonal matrix beside the learning rate, finite */
  int32_t reserved;        /* 0 */
} train_matrix;

typedef struct train_matrices train_matrices;

/* As train_list_create; one handle and one workspace serve calls of one stream at a time.  Gradients, momentum and scratch lie apart from
 * params and copies.  Refused (ROTCONV_ERR_UNSUPPORTED): params and copies that overlap one another.  Refused (ROTCONV_ERR_SHAPE): extents
 * below 1, the shorter side of a matrix above 32768, the longer above 2^24, stacks of more than 2^40 elements, more matrices than 65535
 * or more work than 2^24 - 1 workgroups do (of 128 x 128 elements; sixteen to each of A's). */
int train_matrices_create(const train_matrix* matrices, int count, int grad_dtype, train_matrices** out);
int train_matrices_destroy(train_matrices* matrices);
/* Elements that the momentum spans: stack k's start at the sum of the sizes before it, each size rounded up to a
 * multiple of 32. */
uint64_t train_matrices_elements(const train_matrices* matrices);
size_t train_matrices_workspace_bytes(const train_matrices* matrices);

/* One step of every matrix.  With g = control->coef * grad:
 *     momentum = mu * momentum + g
 *     u = g + mu * momentum (nesterov), or momentum      X = u / (|u| + eps), |u| the root of the sum of u's squares
 *     `steps` times: A = X X^T, X = a X + (b A + c A^2) X with a = 3.4445, b = -4.7750, c = 2.0315 (transposed where rows > cols)
 *     param -= lr * weight_decay * param + lr * scale * X
 * five steps bring every singular value of u that is not vanishing beside the others to between 0.7 and 1.2.
 * momentum: fp32, train_matrices_elements(), zero before the first step.  Products multiply fp16 values (all of them bounded: see
 * the kernels) and add in fp32; X is held in 22 bits between them, and the diagonals of A and of the polynomial in 32.  X's result is off by
 * 2e-4 to 8e-4 of its norm for gradients of full rank, by up to 6e-3 where a few singular values are all there is (rank 1, or noise a hundredth
 * of the rest and below).  A NaN or an infinity makes its own matrix NaN.
 * Then the control block is advanced as by train_adamw_step, unless `keep` is set: a further step that shares the block (AdamW over the
 * network's other tensors) does it.  With control->nonfinite set nothing else is changed. */
typedef struct {
  float momentum;          /* 0 <= momentum < 1 */
  float eps;               /* a normal number > 0 */
  int32_t nesterov, steps; /* steps: 1 to 16 */
  int32_t keep;            /* 1: leaves the control block as it is */
  int32_t reserved;        /* 0 */
} train_muon;
int train_muon_step(const train_matrices* matrices, const train_muon* options, float* momentum, train_control* control,
                    void* ws, size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* UNETTRAIN_H */
