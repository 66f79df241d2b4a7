/*
 * topoep_moe.h -- C ABI of the operators beside the planner on one MI355X
 * (gfx950): the router that makes the planner's top-k ids, the router's
 * gradient, a whole mixture-of-experts layer for a few tokens (decoding:
 * nothing to balance, the weights' bytes are all that counts), and the
 * global gradient norm with its clip, which ends a training step over
 * main experts, replicas and dense parameters.
 *
 * Conventions are topoep.h's: "device" pointers are HIP device memory of the
 * current device and owned by the caller; `stream` is a hipStream_t as
 * void*; work is only enqueued, with no allocation, no host-device
 * synchronisation and no copy, so every call may be captured in a HIP graph;
 * return codes are TOPOEP_OK, TOPOEP_EINVAL, TOPOEP_EWORKSPACE, TOPOEP_EHIP
 * and TOPOEP_ELIMIT, and nothing is enqueued where one other than TOPOEP_OK
 * or TOPOEP_EHIP is returned.
 */
#ifndef TOPOEP_MOE_H
#define TOPOEP_MOE_H

#include <stddef.h>
#include <stdint.h>

#include "topoep.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types. */
#define TOPOEP_F32 0
#define TOPOEP_BF16 1
#define TOPOEP_F16 2

/* Scores of a router. */
#define TOPOEP_SOFTMAX 0
#define TOPOEP_SIGMOID 1

/* Norms. */
#define TOPOEP_NORM_2 0
#define TOPOEP_NORM_INF 1

typedef struct topoep_router {
  int32_t num_experts; /* E, 1 .. TOPOEP_ROUTER_MAX_EXPERTS                          */
  int32_t topk;        /* k, 1 .. min(E, TOPOEP_ROUTER_MAX_TOPK)                     */
  int32_t groups;      /* n groups of E / n consecutive experts (the nodes that hold */
                       /* them), n divides E, n <= 64; 1 = no groups                 */
  int32_t top_groups;  /* g of them are open to a token, 1 <= g <= n, g E / n >= k   */
  int32_t scoring;     /* TOPOEP_SOFTMAX or TOPOEP_SIGMOID                           */
  int32_t renorm;      /* nonzero: the chosen scores are divided by their sum        */
  int32_t dtype;       /* of the logits and of their gradient                        */
  float scale;         /* factor c of the weights, finite                            */
} topoep_router;

#define TOPOEP_ROUTER_MAX_EXPERTS 1024
#define TOPOEP_ROUTER_MAX_TOPK 64

/*
 * Enqueue the router: ids and weights of every token's k experts.
 *
 *   logits   device [T, E] of r->dtype, row t at logits + t * ld elements
 *            (ld >= E, any alignment of the element's size).  NaN and -inf
 *            are masked: chosen last, score 0.  +inf counts as the largest
 *            finite number.
 *   bias     device float [E] or NULL: added to the LOGITS where experts are
 *            chosen, not in their weights.  A bias that was trained to be added
 *            to sigmoid scores is another rule and chooses other experts.
 *   ids      device int32 out [T, k]: the experts of the k largest keys,
 *            key = logit + bias rounded to 32 bits (a NaN key is -inf),
 *            descending, equal keys by the lower id.  With groups, only the
 *            experts of the g groups of the largest maximum key (equal ones
 *            by the lower group; not of the largest sum of two keys).  Always k distinct valid ids, as
 *            topoep_plan takes them.
 *   weights  device float out [T, k]: c times the score.  Softmax scores are
 *            over all E logits, or with renorm over the chosen ones; sigmoid
 *            scores with renorm are divided by the chosen scores' sum (where the
 *            largest is below e^-709, which ends 64 bits, it counts as zero).
 *            Where a sum is zero (every logit masked) the weights are zero.
 *            A row's ids and weights do not depend on the rows beside it.
 *
 * T = 0 enqueues nothing.  TOPOEP_EINVAL: null pointers (bias excepted),
 * sizes outside the ranges of topoep_router, T < 0 or T * k > INT32_MAX, ld <
 * E.  TOPOEP_ELIMIT: E or k or the groups beyond their maximum.
 */
int topoep_route(const topoep_router *r, const void *logits, int64_t ld, int32_t T, const float *bias, int32_t *ids,
                 float *weights, void *stream);

/*
 * Enqueue the router's gradient: from that of the weights to that of the
 * logits (the choice itself has none, and a bias enters only the choice).
 *
 *   logits, ld    as topoep_route was given them
 *   ids           device int32 [T, k]: topoep_route's (distinct in a row; one
 *                 outside [0, E) is taken for a masked expert)
 *   grad_weights  device float [T, k]; a masked choice's is not used, whatever
 *                 it holds
 *   grad_logits   device out [T, E] of r->dtype, row t at t * ldg elements
 *                 (ldg >= E); every element of a row is written, columns
 *                 beyond E are not.  Masked logits get zero.
 *
 * Return codes as topoep_route.
 */
int topoep_route_backward(const topoep_router *r, const void *logits, int64_t ld, int32_t T, const int32_t *ids,
                          const float *grad_weights, void *grad_logits, int64_t ldg, void *stream);

typedef struct topoep_moe {
  int32_t hidden;        /* H, a multiple of 8, at most 2^17                         */
  int32_t inter;         /* I, a multiple of 8, at most 2^17; H I <= 2^30            */
  int32_t local_experts; /* L >= 1 experts whose weights are here                    */
  int32_t dtype;         /* of x, the weights and out: TOPOEP_BF16 or TOPOEP_F16     */
} topoep_moe;

#define TOPOEP_MOE_MAX_TOKENS 128

/* Bytes of device workspace topoep_moe_few needs for T tokens or fewer. */
int topoep_moe_workspace_bytes(const topoep_moe *m, const topoep_router *r, int32_t T, size_t *bytes_out);

/*
 * Enqueue a whole mixture-of-experts layer (SwiGLU experts) for 0 .. 128
 * tokens.  With t's experts e_j and weights w_j from the router on the logits
 * x_t gate^T (held in 32 bits; r->dtype is not read), and s_j = slot[e_j]:
 *
 *   h_j   = silu(up[s_j][0:I] x_t) * (up[s_j][I:2I] x_t),  silu(z) = z / (1 + exp(-z))
 *   out_t = sum_{j: s_j >= 0} w_j down[s_j] h_j
 *
 *   x            device [T, H], row t at x + t * ldx elements (H <= ldx < 2^24,
 *                a multiple of 8), 16-byte aligned, as are the weights and out
 *   gate         device [E, H]
 *   bias         device float [E] or NULL, as topoep_route
 *   expert_slot  device int32 [E] or NULL: where each expert's weights lie in
 *                up and down; outside [0, L) = not here: it adds nothing, and
 *                a token without any expert here gets zeros.  NULL: expert e at
 *                slot e
 *   up           device [L, 2I, H]: I gate rows, then I up rows, per expert
 *   down         device [L, H, I]
 *   out          device out [T, H], dense
 *   ids, weights device out [T, k]: the router's
 *   workspace    topoep_moe_workspace_bytes bytes, 256-byte aligned; nothing
 *                in it is kept between calls or has to be cleared.  Calls that
 *                share one are ordered on one stream.
 *
 * Products are accumulated in 32 bits; h is held in two words of the weights'
 * type: to 2^-16 of it (bf16), 2^-22 (f16, at least 2^-25; saturated at 2^27).
 * Outputs are rounded once.  TOPOEP_EINVAL: null
 * pointers, sizes outside their ranges, misaligned buffers; TOPOEP_ELIMIT:
 * T above TOPOEP_MOE_MAX_TOKENS or the router's limits;
 * TOPOEP_EWORKSPACE: workspace too small or misaligned.
 */
int topoep_moe_few(const topoep_moe *m, const topoep_router *r, const void *x, int64_t ldx, int32_t T,
                   const void *gate, const float *bias, const int32_t *expert_slot, const void *up, const void *down,
                   void *out, int32_t *ids, float *weights, void *workspace, size_t workspace_bytes, void *stream);

/* One tensor of a gradient set (host memory; read during the call). */
typedef struct topoep_grad {
  const void *grad;  /* device, n elements of dtype, any alignment of their size     */
  void *out;         /* device, n elements of out_dtype: where the clipped gradient  */
                     /* goes.  May be grad itself (dtype == out_dtype); otherwise no */
                     /* out overlaps another out or any grad of the set.  Not read   */
                     /* by topoep_grad_norm                                          */
  int64_t n;         /* >= 0; a set has at most 2^40 elements                        */
  int32_t dtype;
  int32_t out_dtype;
} topoep_grad;

/* Bytes of device workspace for a set of `count` tensors or fewer. */
int topoep_grads_workspace_bytes(int32_t count, size_t *bytes_out);

/*
 * Enqueue the global norm of a set of tensors: *norm (device float) = scale *
 * the 2-norm, or the largest magnitude, over all of their elements.  Squares
 * are summed in 64 bits in an order that depends only on the sizes and on which
 * tensors follow each other in memory, so equal calls give equal bits.  NaN
 * where an element is NaN.  scale: finite, >= 0 (1 / the loss scale).
 * TOPOEP_EINVAL: null pointers, negative sizes or more than 2^40 elements, unknown
 * types or norms, pointers not aligned to their elements; TOPOEP_EWORKSPACE:
 * workspace too small or not 256-byte aligned.
 */
int topoep_grad_norm(const topoep_grad *grads, int32_t count, float scale, int32_t ord, float *norm, void *workspace,
                     size_t workspace_bytes, void *stream);

/*
 * Enqueue the clip: out = grad * (scale * min(1, max_norm / (norm + 1e-6))) for
 * every element.  given_norm: device float, the norm to clip by (a group's, say,
 * already scaled), or NULL: that of topoep_grad_norm over this set, which is
 * also written to *norm (may be NULL).  Where the norm is not finite nothing
 * is written but *norm, so that the caller can drop the step.  Where the
 * factor is 1, tensors clipped in place are left alone.  max_norm > 0, finite or
 * infinite.  Return codes as topoep_grad_norm; TOPOEP_EINVAL also for outputs
 * that overlap (a tensor clipped in place that is in the set twice, say),
 * TOPOEP_ELIMIT where the host has no memory to look.
 */
int topoep_clip_grads(const topoep_grad *grads, int32_t count, float scale, int32_t ord, float max_norm,
                      const float *given_norm, float *norm, void *workspace, size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* TOPOEP_MOE_H */
