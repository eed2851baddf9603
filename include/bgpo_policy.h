/*
 * bgpo_policy.h - token log-probabilities of logits (libbgpo).
 *
 * What stands beside the ELBO head of bgpo.h when a policy is trained or
 * scored: the log-probability of a given token in each row of logits that a
 * model has returned (an old policy, a reference model, a head with terms of
 * its own) with its backward pass.
 *
 * Conventions as in bgpo.h: array arguments are device pointers owned by the
 * caller, the problem structs host pointers; work is enqueued on `stream`
 * without synchronising, allocating or copying, so that every call can be
 * captured into a HIP graph; host-detectable errors return a negative
 * bgpo_status before anything is enqueued; a workspace (256-byte aligned)
 * carries nothing from one call to the next, and calls that may overlap in
 * time (other streams, captured graphs) must not share one.  Matrices have
 * contiguous rows whose starts are ld elements apart; any alignment that the
 * element type allows is taken (16 bytes and even strides are fastest).
 * Elements between the rows are neither read nor written.  An output must not
 * overlap an input or another output unless the call says so
 * (BGPO_ERR_INVALID_ARG).  All sums run in a fixed order: identical inputs
 * give identical bits.
 */
#ifndef BGPO_POLICY_H_
#define BGPO_POLICY_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* ---------------------------------------------------------------- logits */

/* Rows of logits x[rows, V].  With z = scale x (scale = 1 / temperature) and
 * p = softmax(z), a row whose target token is y has
 *   lse = log sum_v e^{z_v},  logp = z_y - lse,  H = lse - sum_v p_v z_v
 * A logit of -inf is a token that cannot be drawn (p = 0, no contribution to
 * H); a row with a NaN or +inf, or with nothing but -inf, gives NaN.  A row is
 * masked if row_mask is given and 0 there, or if its target is negative: its
 * logits are not read, whatever they hold.  A target of V or more gives
 * NaN (logp, and the row's gradient); nothing is read out of range. */
typedef struct bgpo_logits {
  int64_t rows;       /* 0 <= rows < 2^31 */
  int64_t ld;         /* elements between rows, >= V (any value for one row) */
  int32_t V;          /* 1 <= V <= 2^24 */
  int32_t in_dtype;   /* BGPO_BF16 or BGPO_F32 */
  float scale;        /* > 0, finite */
  int32_t reserved;   /* 0 */
} bgpo_logits;

/* Bytes of device workspace of bgpo_logits_logp (0 where it needs none; then
 * workspace may be NULL).  Depends on rows and V only.  Host only. */
int bgpo_logits_workspace_size(const bgpo_logits* prob, size_t* bytes);

/* Log-probabilities of the targets.
 *   logits    bf16 or fp32 [rows, V] (in_dtype, ld)
 *   targets   int32 [rows]
 *   row_mask  uint8 [rows] or NULL (every row counts)
 *   logp      float [rows]   out; 0 on masked rows
 *   entropy   float [rows]   out, 0 on masked rows; may be NULL
 *   lse       float [rows]   out, 0 on masked rows; may be NULL (the backward
 *                            takes it)
 * Sums and statistics are held in fp32, a few hundred terms each, and joined
 * over the row. */
int bgpo_logits_logp(const bgpo_logits* prob, const void* logits, const int32_t* targets,
                     const uint8_t* row_mask, float* logp, float* entropy, float* lse,
                     void* workspace, size_t ws_bytes, void* stream);

/* Gradient of a scalar w.r.t. the logits, from its gradients w.r.t. logp (a)
 * and the entropy (b):
 *   dlogits_v = scale (a (1[v = y] - p_v) - b p_v (log p_v + H))
 *   lse       float [rows]   of bgpo_logits_logp with the same scale
 *   entropy   float [rows]   of the same call; may be NULL without dentropy
 *   dlogp     float [rows]   a
 *   dentropy  float [rows]   b; NULL = 0
 *   dlogits   [rows, V] of in_dtype, rows ld_out elements apart: out, every
 *             entry written (not accumulated), rounded once (nearest even).
 *             May be `logits` itself (the same pointer and stride).
 * Rows that are masked, or whose a and b are both 0 (a token that a clip has
 * cut off), become 0 without their logits being read. */
int bgpo_logits_logp_bwd(const bgpo_logits* prob, const void* logits, const int32_t* targets,
                         const uint8_t* row_mask, const float* lse, const float* entropy,
                         const float* dlogp, const float* dentropy, void* dlogits,
                         int64_t ld_out, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* BGPO_POLICY_H_ */
