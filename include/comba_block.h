/*
 * comba_block.h -- a recurrent model's block beside comba.h's mixer: linear
 * attention with a decay for each head, and the norms after and before a block
 * fused with its gate, residual scale and residual stream.  For training (forward
 * and backward), prompts (fixed rows or packed sequences, states that enter and
 * leave) and single tokens (states in slots, in place).
 *
 * The conventions of comba_layer.h hold: ownership, streams, status codes, packed
 * sequences, types (activations, their gradients and the outputs bf16 or fp32;
 * parameters, their gradients and states fp32), rows named by `*_row` fields,
 * alignment, token-free calls, slots of single-token calls.
 */
#ifndef COMBA_BLOCK_H
#define COMBA_BLOCK_H

#include "comba_layer.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- linear attention with a decay for each head ------------------------- */
typedef struct {
  int32_t B, T;               /* rows and tokens per row (packed: 1, total; step: B, 1)   */
  int32_t H;                  /* heads: of the states, o and the decays; up to 65535      */
  int32_t Hq, Hk, Hv;         /* heads of q, k and v; each divides H: head h reads head   */
                              /* h / (H / Hq) of q, and so on                             */
  int32_t dk, dv;             /* head sizes, 1..256                                       */
  int32_t num_seqs;           /* as in comba_shape                                        */
  const int32_t *cu_seqlens;
  const int32_t *cu_seqlens_host;
  comba_dtype in_dtype;       /* of q, k, v, o and their gradients                        */
  comba_dtype g_dtype;        /* of g and dg: in_dtype, or fp32 (per head: fp32)          */
  int32_t g_per_head;         /* g is [H], the same for every token                       */
  float scale;
  int64_t q_row, k_row, v_row, g_row; /* elements between token rows (0: contiguous);     */
                              /* up to 2^22 but for the step                              */
} comba_decay_shape;

/*
 * Per head, with the state S [dk,dv] in fp32:
 *     S_t = exp(g_t) S_{t-1} + k_t v_t^T,      o_t = scale S_t^T q_t.
 *   q [B,T,Hq,dk], k [B,T,Hk,dk], v [B,T,Hv,dv], o [B,T,H,dv] in_dtype; g [B,T,H] or
 *   [H] log-decays; h0, ht [num_seqs,H,dk,dv] fp32 or NULL.
 * g = -inf starts a state anew from a finite one (zero times Inf or NaN is NaN: fill the
 * memory of a new state); log-decays below -128 count as -128, whose decay is zero in
 * fp32.  A NaN or Inf in an input makes outputs of its own sequence and
 * head non-finite, up to 63 tokens before its own among them (gradients: behind it).
 * bf16: products of operands rounded to bf16, summed in fp32 (o within about two
 * roundings to bf16); the states keep fp32.  The states kept for chunks have one scale for
 * 16 value by 16 or 32 key columns: what is below 2^-29 of the largest there loses
 * bits, below 2^-39 it counts as zero in o and the gradients (not in ht and dh0).
 * The workspace holds comba_decay_fwd_workspace_bytes, the state at every 64th token
 * among them (bf16: 16 bits a value, fp16 and its scale; else fp32).  The saving form's
 * holds comba_decay_save_bytes and keeps those: comba_decay_bwd takes it as `saved`,
 * unmodified, together with the same shape and inputs (either call may know the offsets on
 * the host) and a workspace of its own (comba_decay_bwd_workspace_bytes).
 * Limits: H max(dk, dv) up to 2^22; pieces of 64 tokens (a sequence's last one may be
 * partial) times H, and sequences times H times dv / 32, below 2^31 / 512; a step's
 * rows below 2^24.
 * Long sequences are cut into segments that run side by side where that is faster; the
 * choice follows from the shape, the host offsets and the device (COMBA_SCAN_SEGMENTS is
 * not read), and changes results by roundings only.  Every sum runs in an order fixed by
 * that choice.
 * Log-decays above zero are taken too: a growth of more than 2^127 over a chunk of 64
 * tokens, or over the segments of a sequence, overflows, also before a state that is zero.
 */
size_t comba_decay_fwd_workspace_bytes(const comba_decay_shape *shape);
size_t comba_decay_save_bytes(const comba_decay_shape *shape);
size_t comba_decay_bwd_workspace_bytes(const comba_decay_shape *shape);
comba_status comba_decay_fwd(const comba_decay_shape *shape, const void *q, const void *k,
                             const void *v, const void *g, const float *h0, void *o, float *ht,
                             void *ws, size_t ws_bytes, void *stream);
comba_status comba_decay_fwd_save(const comba_decay_shape *shape, const void *q, const void *k,
                                  const void *v, const void *g, const float *h0, void *o,
                                  float *ht, void *ws, size_t ws_bytes, void *stream);
/*
 * From dO [B,T,H,dv] in_dtype and dht [num_seqs,H,dk,dv] fp32 (or NULL): dq, dk, dv
 * (layouts of q, k, v, contiguous), dg [B,T,H] g_dtype (NULL: not wanted; per-head
 * decays are constants and have none), dh0 fp32 (or NULL).  Gradients of shared
 * heads are summed in fp32 in the order of the heads.  bf16: dg is formed from
 * products of operands rounded to bf16 whatever its own type.
 */
comba_status comba_decay_bwd(const comba_decay_shape *shape, const void *q, const void *k,
                             const void *v, const void *g, const float *h0, const void *dO,
                             const float *dht, void *dq, void *dk, void *dv, void *dg, float *dh0,
                             const void *saved, size_t saved_bytes, void *ws, size_t ws_bytes,
                             void *stream);
/* One token per row (T = 1): o [B,H,dv]; state [num_slots,H,dk,dv] fp32, in place. */
comba_status comba_decay_step(const comba_decay_shape *shape, const void *q, const void *k,
                              const void *v, const void *g, float *state, const int32_t *slots,
                              int32_t num_slots, void *o, void *stream);

/* ---- norms after and before a block, gate, residual scale, stream --------- */
typedef struct {
  int64_t rows;               /* tokens                                                   */
  int32_t C;                  /* channels                                                 */
  comba_dtype dtype;          /* of y, z, n and their gradients                           */
  comba_dtype x_dtype;        /* of the stream x, r and their gradients: dtype, or fp32   */
  comba_activation activation; /* of the gate                                             */
  float eps;                  /* >= 0, added to the mean squares                          */
  int64_t y_row, z_row, x_row; /* elements between rows (0: C)                            */
} comba_block_norm_shape;

/*
 * A block's output y joins the residual stream x, and the next block's input n
 * leaves it.  Per token, rms(u) = sqrt(mean(u^2) + eps) over its C channels:
 *     p = y / rms(y) * post_weight   (p = y without post_weight),
 *     t = p act(z)                   (t = p without the gate z),
 *     r = x + scale t                (without x: r = scale t; without scale: 1),
 *     n = r / rms(r) * weight        (not formed when weight is NULL).
 *   y, z [rows,C]; x, r [rows,C]; n [rows,C]; post_weight, scale, weight [C] fp32 or
 *   NULL.  n is formed from r before its rounding.
 */
comba_status comba_block_norm_fwd(const comba_block_norm_shape *shape, const void *y,
                                  const void *x, const void *z, const float *post_weight,
                                  const float *scale, const float *weight, void *r, void *n,
                                  void *stream);
/*
 * From dr [rows,C] (x_dtype) and dn [rows,C] (either may be NULL: zeros): dy, dz
 * (with z), dx (with x; NULL: not wanted), and dpost_weight, dscale, dweight [C] fp32
 * where their parameter is given (each may be NULL).  Recomputes p, r and both
 * norms; sums in a fixed order.  Without weight or without dn the norm of r takes no
 * part (dweight is zero): what x holds, Inf among it, reaches no gradient.
 * Without post_weight y enters dy through the norm of r alone.
 */
size_t comba_block_norm_workspace_bytes(const comba_block_norm_shape *shape);
comba_status comba_block_norm_bwd(const comba_block_norm_shape *shape, const void *y,
                                  const void *x, const void *z, const float *post_weight,
                                  const float *scale, const float *weight, const void *dr,
                                  const void *dn, void *dy, void *dx, void *dz,
                                  float *dpost_weight, float *dscale, float *dweight, void *ws,
                                  size_t ws_bytes, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* COMBA_BLOCK_H */
