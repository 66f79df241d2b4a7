/*
 * topoep_ffn.h -- C ABI of the experts' products on one MI355X (gfx950): the
 * gated feed-forward block with its gradients, dense (a shared expert) or for
 * the experts a router chose (topoep_route's ids and weights); the rows of such
 * a layer sorted by expert; and for serving, the product in 8-bit integers with
 * a scale for each token and channel, and the quantisation that makes them.
 *
 * Conventions are topoep.h's: "device" pointers are HIP device memory of the
 * current device and owned by the caller; `stream` is a hipStream_t as
 * void*; work is only enqueued, with no allocation, no host-device
 * synchronisation and no copy, so every call may be captured in a HIP graph;
 * return codes are TOPOEP_OK, TOPOEP_EINVAL, TOPOEP_EWORKSPACE, TOPOEP_EHIP
 * and TOPOEP_ELIMIT, and nothing is enqueued where one other than TOPOEP_OK
 * or TOPOEP_EHIP is returned.  Types are topoep_moe.h's.  A workspace is 256-byte
 * aligned; nothing in it is kept between calls or has to be cleared, and calls
 * that share one are ordered on one stream.  No result depends on the
 * order in which workgroups run: equal calls give equal bits.
 */
#ifndef TOPOEP_FFN_H
#define TOPOEP_FFN_H

#include <stddef.h>
#include <stdint.h>

#include "topoep_moe.h"

#ifdef __cplusplus
extern "C" {
#endif

#define TOPOEP_FFN_MAX_EXPERTS 1024

/* Bytes of device workspace topoep_expert_rows needs for T tokens or fewer. */
int topoep_expert_rows_workspace_bytes(int32_t T, int32_t k, int32_t L, size_t *bytes_out);

/*
 * Enqueue the order of a router's choices by expert: choice (t, j) is pair
 * t * k + j, and those of one expert keep their order.
 *
 *   ids          device int32 [T, k]; what is outside [0, E) is nowhere
 *   expert_slot  device int32 [E] or NULL: where each expert lies among the L
 *                here (outside [0, L): elsewhere).  NULL: expert e at slot e
 *   offsets      device int32 out [L + 1]: slot s has the rows
 *                offsets[s] .. offsets[s + 1] - 1; offsets[0] = 0
 *   pairs        device int32 out [T * k]: the pair of each row; -1 behind
 *                the last
 *   places       device int32 out [T, k]: the row of each pair; -1 where its
 *                expert is not here
 *   workspace    topoep_expert_rows_workspace_bytes bytes
 *
 * T = 0 writes offsets alone.  TOPOEP_EINVAL: null pointers (expert_slot
 * excepted), T < 0, k < 1, T * k > INT32_MAX, E < 1, L < 1.  TOPOEP_ELIMIT: L above
 * TOPOEP_FFN_MAX_EXPERTS.  TOPOEP_EWORKSPACE: too small or misaligned.
 */
int topoep_expert_rows(const int32_t *ids, int32_t T, int32_t k, const int32_t *expert_slot, int32_t E, int32_t L,
                       int32_t *offsets, int32_t *pairs, int32_t *places, void *workspace, size_t workspace_bytes,
                       void *stream);

typedef struct topoep_ffn {
  int32_t hidden;  /* H, a multiple of 8, at most 2^17                               */
  int32_t inter;   /* I, a multiple of 8, at most 2^17; H I <= 2^30                  */
  int32_t experts; /* L >= 1 blocks of weights                                       */
  int32_t dtype;   /* of x, weights, outputs, gradients: TOPOEP_BF16 or TOPOEP_F16   */
} topoep_ffn;

/* The rows of the experts, as topoep_expert_rows leaves them (all device). */
typedef struct topoep_ffn_rows {
  const int32_t *offsets; /* [L + 1]                                                 */
  const int32_t *pairs;   /* [T * k]                                                 */
  const int32_t *places;  /* [T, k]                                                  */
  const float *weights;   /* [T, k]: the router's                                    */
  int32_t topk;           /* k, 1 .. TOPOEP_ROUTER_MAX_TOPK                          */
  int32_t num_experts;    /* E >= 1, of which the router chose: the rows an expert   */
                          /* gets, about, are T k / E (for the kernels' tiles alone) */
} topoep_ffn_rows;

/*
 * Bytes of a forward pass's workspace (the same with saved and without), of what it keeps for a backward pass
 * (saved), and of the backward pass's workspace, for T tokens; rows: whether
 * the layer is a routed one, and its k and E (these alone are read).  All three hold T k rows, however many
 * of them have their expert here.  NULL outputs are not written.
 */
int topoep_ffn_bytes(const topoep_ffn *f, int32_t T, const topoep_ffn_rows *rows, size_t *forward, size_t *saved,
                     size_t *backward);

/*
 * Enqueue the gated feed-forward block (SwiGLU):
 *
 *   f(x) = down (silu(up[0:I] x) * (up[I:2I] x)),  silu(z) = z / (1 + exp(-z))
 *
 * rows NULL (L = 1): out_t = f(x_t).  Otherwise with t's experts e_j at slots s_j
 * and weights w_j: out_t = sum over its choices that are here, in their order, of w_j f_{s_j}(x_t);
 * a token without any gets zeros.
 *
 *   x        device [T, H], row t at x + t * ldx elements (ldx >= H, a multiple
 *            of 8), 16-byte aligned, as are the weights, out and saved
 *   up       device [L, 2I, H]: I gate rows, then I up rows, per expert
 *   down     device [L, H, I]
 *   out      device out [T, H], dense
 *   saved    device out or NULL (no backward pass follows)
 *
 * Products are accumulated in 32 bits.  The hidden values, times their row's
 * weight, are rounded once to the weights' type, the second product's
 * operand (f16: beyond 65504 infinite, below 2^-14 to multiples of 2^-24, so that a small weight costs
 * bits); a routed token's sum is kept in 32 bits and rounded once.  Gate
 * and up values are kept for the backward pass in 32 bits.  T = 0 enqueues
 * nothing.  TOPOEP_EINVAL: null pointers, sizes outside their ranges, T * k
 * above 2^30, rows NULL with L > 1, misaligned buffers; TOPOEP_ELIMIT:
 * L or k above its maximum; TOPOEP_EWORKSPACE: workspace too small or misaligned.
 */
int topoep_ffn_forward(const topoep_ffn *f, const void *x, int64_t ldx, int32_t T, const topoep_ffn_rows *rows,
                       const void *up, const void *down, void *out, void *saved, void *workspace,
                       size_t workspace_bytes, void *stream);

/*
 * Enqueue its gradients, from that of out (device [T, H], dense, 16-byte
 * aligned).  x, rows, up, down as the forward pass was given them, saved as
 * it left it.  With h and a = (g, u) of a row, w its weight:
 *
 *   dh = down^T dout,  grad_w = <dh, h>,  da = w (dh u silu'(g), dh silu(g))
 *   grad_x = sum up^T da,  grad_up = sum da x^T,  grad_down = sum w dout h^T
 *
 *   grad_x        device out [T, H], dense
 *   grad_weights  device float out [T, k] (rows NULL: not read); 0 where a
 *                 choice's expert is not here
 *   grad_up, grad_down  device out [L, 2I, H] and [L, H, I]; zeros for an expert without rows
 *
 * NULL: a gradient that is not wanted.  da is rounded once to the weights'
 * type.  Return codes as topoep_ffn_forward; with T = 0 grad_up and grad_down
 * are zeros.
 */
int topoep_ffn_backward(const topoep_ffn *f, const void *x, int64_t ldx, int32_t T, const topoep_ffn_rows *rows,
                        const void *up, const void *down, const void *saved, const void *grad_out, void *grad_x,
                        float *grad_weights, void *grad_up, void *grad_down, void *workspace, size_t workspace_bytes,
                        void *stream);

/*
 * Enqueue the quantisation of rows to 8 bits:
 *
 *   scale_m = max_k |x_mk| / 127 (to the nearest of 32 bits),  q_mk = x_mk / scale_m to the nearest integer, ties to even
 *
 * at most 127 in magnitude; a row of zeros has scale 0 and zeros.  A row with an
 * infinity or NaN gets that as its scale (NaN before infinity), and zeros.
 *
 *   x      device [M, K] of dtype (32, 16 bits), row m at x + m * ldx elements
 *          (ldx >= K; any alignment of the element's size)
 *   q      device int8 out [M, K], dense
 *   scale  device float out [M]
 *
 * M = 0 enqueues nothing.  TOPOEP_EINVAL: null pointers, M < 0, K < 1, K > 2^30, ldx < K, an unknown type.
 */
int topoep_quantize(const void *x, int32_t dtype, int64_t ldx, int32_t M, int32_t K, int8_t *q, float *scale,
                    void *stream);

typedef struct topoep_int8 {
  int32_t n;         /* N, rows (channels) of a weight matrix, 1 .. 2^20; even where gated */
  int32_t k;         /* K, a multiple of 16, at most 2^17 (sums are at most 2^31)    */
  int32_t groups;    /* G weight matrices, 1 .. TOPOEP_FFN_MAX_EXPERTS               */
  int32_t gated;     /* nonzero: out = silu(a[0:N/2]) * a[N/2:N]                     */
  int32_t out_dtype;
} topoep_int8;

/* Bytes of device workspace topoep_matmul_int8 needs for M rows (0: none). */
int topoep_matmul_int8_workspace_bytes(const topoep_int8 *p, int32_t M, size_t *bytes_out);

/*
 * Enqueue the product of rows and weights in 8 bits:
 *
 *   a_mn = (sum_k q_mk w_nk) * scale_m * w_scale_n,  the sum exact
 *
 *   q        device int8 [M, K], row m at q + m * ldq (ldq >= K, a multiple of
 *            16), 16-byte aligned, as is w
 *   scale    device float [M]
 *   offsets  device int32 [G + 1] or NULL (G = 1: all rows): matrix g takes the
 *            rows offsets[g] .. offsets[g + 1] - 1; ascending, from 0 to at most M.
 *            Rows behind the last are zeros in out, or left as they were where
 *            keep_rest is nonzero
 *   w        device int8 [G, N, K], w_scale device float [G, N]
 *   out      device out [M, N] (gated: [M, N / 2]) of out_dtype, dense
 *   workspace  topoep_matmul_int8_workspace_bytes bytes
 *
 * Any of the 256 values may be in q and w.  The product with the scales and the
 * activation are in 32 bits, rounded once.
 * M = 0 enqueues nothing.  TOPOEP_EINVAL: null pointers, M above 2^30, sizes outside their
 * ranges, misaligned buffers, offsets NULL with G > 1; TOPOEP_ELIMIT: G above its
 * maximum; TOPOEP_EWORKSPACE: too small or misaligned.
 */
int topoep_matmul_int8(const topoep_int8 *p, const int8_t *q, int64_t ldq, const float *scale, int32_t M,
                       const int32_t *offsets, int32_t keep_rest, const int8_t *w, const float *w_scale, void *out,
                       void *workspace, size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* TOPOEP_FFN_H */
