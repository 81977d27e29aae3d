/*
 * comba_layer.h -- operators around and beside the token mixer of comba.h in a
 * recurrent layer: the short causal convolution with its history, the selective
 * state space scan, and the group norm per token with an activation or a gate.
 * For training (forward and backward), prompts (fixed rows or packed sequences,
 * states that enter and leave) and single tokens (states in slots, in place).
 *
 * The conventions of comba.h hold (ownership, streams, status codes, offsets of
 * packed sequences), with these differences:
 *  - Activations have dtype in_dtype (bf16 or fp32), and so have their
 *    gradients and the outputs; parameters, their gradients and the scan's
 *    states are fp32; the convolution's states have in_dtype.
 *  - Rows: the inputs named with a `*_row` field are [tokens] rows that lie
 *    `*_row` elements apart (0: contiguous), so that a column slice of a wider
 *    projection is taken as it lies; a row's own elements are contiguous.
 *    comba_select_fwd, _fwd_save and _bwd take rows up to 2^22 elements apart,
 *    the other calls any distance.  Every other tensor is C-contiguous.
 *  - Alignment: every pointer needs its element's size only, a workspace 256
 *    bytes.  Calls are fastest where rows start at multiples of 16 bytes.
 *  - Token-free calls are valid as in comba.h: states pass through.
 *  - Step calls (one token per sequence) update the states in place: row b uses
 *    slot slots[b] of the pool, or slot b when slots is NULL.  A row whose slot
 *    lies outside [0, num_slots) is padding: its y is zero and no state is
 *    touched.  Two rows with the same slot race.
 */
#ifndef COMBA_LAYER_H
#define COMBA_LAYER_H

#include "comba.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { COMBA_ACT_NONE = 0, COMBA_ACT_SILU = 1, COMBA_ACT_SIGMOID = 2 } comba_activation;

/* ---- short causal convolution ------------------------------------------- */
typedef struct {
  int32_t B, T;               /* rows and tokens per row (packed: 1, total; step: B, 1)   */
  int32_t D;                  /* channels                                                 */
  int32_t K;                  /* taps, 2..4                                               */
  int32_t num_seqs;           /* as in comba_shape                                        */
  const int32_t *cu_seqlens;  /* as in comba_shape                                        */
  const int32_t *cu_seqlens_host;
  comba_dtype in_dtype;
  comba_activation activation; /* NONE or SILU                                            */
  int64_t x_row;              /* elements between token rows of x (0: D)                  */
} comba_conv_shape;

/*
 * Depthwise causal convolution of a sequence's extended input xt = [h0; x] (its
 * K - 1 inputs before the first token, zeros when h0 is NULL):
 *     u_t = bias + sum_{j<K} w[c][j] xt_{t+j},   y_t = act(u_t),
 * the newest token under the last tap.  ht: the last K - 1 rows of xt.
 *   x, y [B,T,D] in_dtype; w [D,K] fp32; bias [D] fp32 or NULL;
 *   h0, ht [num_seqs,K-1,D] in_dtype or NULL (oldest first).
 */
comba_status comba_conv_fwd(const comba_conv_shape *shape, const void *x, const float *w,
                            const float *bias, const void *h0, void *y, void *ht, void *stream);
/*
 * Backward: from dy [B,T,D] in_dtype and dht (layout of ht, or NULL) the
 * gradients dx [B,T,D] in_dtype, dw [D,K] and dbias [D] fp32 (dbias NULL when
 * bias is), dh0 in_dtype (or NULL).  Recomputes u.  Sums run in a fixed order.
 */
size_t comba_conv_workspace_bytes(const comba_conv_shape *shape);
comba_status comba_conv_bwd(const comba_conv_shape *shape, const void *x, const float *w,
                            const float *bias, const void *h0, const void *dy, const void *dht,
                            void *dx, float *dw, float *dbias, void *dh0, void *ws,
                            size_t ws_bytes, void *stream);
/* One token per row (T = 1): y [B,D]; state [num_slots,K-1,D] in_dtype, in place. */
comba_status comba_conv_step(const comba_conv_shape *shape, const void *x, const float *w,
                             const float *bias, void *state, const int32_t *slots,
                             int32_t num_slots, void *y, void *stream);

/* ---- selective state space scan ------------------------------------------ */
typedef struct {
  int32_t B, T, D;            /* rows, tokens per row, channels                           */
  int32_t N;                  /* states per channel: 8, 16 or 32                          */
  int32_t G;                  /* groups of B and C rows; divides D                        */
  int32_t num_seqs;           /* as in comba_shape                                        */
  const int32_t *cu_seqlens;
  const int32_t *cu_seqlens_host;
  comba_dtype in_dtype;
  int32_t delta_softplus;     /* dt = softplus(delta + bias) (else delta + bias)          */
  int64_t u_row, delta_row, z_row; /* elements between token rows (0: D)                  */
  int64_t b_row, c_row;       /* the same for B and C (0: G * N)                          */
} comba_select_shape;

/*
 * Per channel c and state n (group g = c / (D / G)), fp32 states:
 *     dt_t = softplus(delta_t + delta_bias),  h_t = exp(dt_t A) h_{t-1} + dt_t u_t B_t[g],
 *     s_t = <C_t[g], h_t> + Dskip u_t,        y_t = s_t silu(z_t)   (y_t = s_t without z).
 *   u, delta, z, y [B,T,D] in_dtype (z or NULL); A [D,N] fp32 (negative for a
 *   decaying state); Bm, Cm [B,T,G,N] in_dtype; Dskip, delta_bias [D] fp32 or
 *   NULL; h0, ht [num_seqs,D,N] fp32 or NULL.
 * Sequences times blocks of 512 / N channels (per group) may be up to 2^32 / 768
 * (N = 8: 512) in a call.
 * The decays of several tokens (of a segment: all of its tokens) are multiplied in
 * fp32 before they meet a state: where dt A > 0, a growth of more than 2^127 over
 * them overflows, also before a state that is zero.
 * Few long rows (packed ones only with cu_seqlens_host) are cut into segments
 * that run side by side; the choice follows from the shape and the device.
 * The workspace holds comba_select_fwd_workspace_bytes.  The saving form's holds
 * comba_select_save_bytes and keeps the states that the backward needs:
 * comba_select_bwd takes it as `saved`, unmodified, together with the same shape
 * and inputs and a workspace of its own (comba_select_bwd_workspace_bytes, which
 * need not live between the two).
 */
size_t comba_select_fwd_workspace_bytes(const comba_select_shape *shape);
size_t comba_select_save_bytes(const comba_select_shape *shape);
size_t comba_select_bwd_workspace_bytes(const comba_select_shape *shape);
comba_status comba_select_fwd(const comba_select_shape *shape, const void *u, const void *delta,
                              const float *A, const void *Bm, const void *Cm, const float *Dskip,
                              const void *z, const float *delta_bias, const float *h0, void *y,
                              float *ht, void *ws, size_t ws_bytes, void *stream);
comba_status comba_select_fwd_save(const comba_select_shape *shape, const void *u,
                                   const void *delta, const float *A, const void *Bm,
                                   const void *Cm, const float *Dskip, const void *z,
                                   const float *delta_bias, const float *h0, void *y, float *ht,
                                   void *ws, size_t ws_bytes, void *stream);
/*
 * From dy [B,T,D] in_dtype and dht [num_seqs,D,N] fp32 (or NULL): du, ddelta, dz
 * [B,T,D] and dB, dC [B,T,G,N] in_dtype; dA [D,N], dD [D], ddelta_bias [D] fp32;
 * dh0 [num_seqs,D,N] fp32 (or NULL).  dz, dD and ddelta_bias are required
 * where their input is given, and not written otherwise.  Every sum runs in a
 * fixed order.
 */
comba_status comba_select_bwd(const comba_select_shape *shape, const void *u, const void *delta,
                              const float *A, const void *Bm, const void *Cm, const float *Dskip,
                              const void *z, const float *delta_bias, const float *h0,
                              const void *dy, const float *dht, void *du, void *ddelta, float *dA,
                              void *dB, void *dC, float *dD, void *dz, float *ddelta_bias,
                              float *dh0, const void *saved, size_t saved_bytes, void *ws,
                              size_t ws_bytes, void *stream);
/* One token per row (T = 1): y [B,D]; state [num_slots,D,N] fp32, in place. */
comba_status comba_select_step(const comba_select_shape *shape, const void *u, const void *delta,
                               const float *A, const void *Bm, const void *Cm, const float *Dskip,
                               const void *z, const float *delta_bias, float *state,
                               const int32_t *slots, int32_t num_slots, void *y, void *stream);

/* ---- group norm per token ------------------------------------------------ */
typedef struct {
  int64_t rows;               /* tokens                                                   */
  int32_t C;                  /* channels                                                 */
  int32_t G;                  /* groups of C / G consecutive channels; divides C          */
  comba_dtype x_dtype;        /* of x and dx: out_dtype, or fp32                          */
  comba_dtype out_dtype;      /* of y, z, dy and dz                                       */
  comba_activation activation;
  float eps;                  /* >= 0, added to the variance                              */
  int64_t x_row, z_row;       /* elements between rows (0: C)                             */
} comba_group_norm_shape;

/*
 * Per token and group of m = C / G channels: mean and (biased) variance over the
 * group's channels, n = (x - mean) / sqrt(var + eps) * weight + bias, and
 *     y = act(n)     without z,        y = n act(z)     with the gate z.
 *   x [rows,C]; weight, bias [C] fp32 or NULL (1 and 0); z [rows,C] or NULL.
 */
comba_status comba_group_norm_fwd(const comba_group_norm_shape *shape, const void *x,
                                  const float *weight, const float *bias, const void *z, void *y,
                                  void *stream);
/*
 * From dy [rows,C]: dx (x_dtype), dz (required with z), dweight and dbias [C]
 * fp32 (each may be NULL).  Recomputes the statistics; sums in a fixed order.
 */
size_t comba_group_norm_workspace_bytes(const comba_group_norm_shape *shape);
comba_status comba_group_norm_bwd(const comba_group_norm_shape *shape, const void *x,
                                  const float *weight, const float *bias, const void *z,
                                  const void *dy, void *dx, void *dz, float *dweight, float *dbias,
                                  void *ws, size_t ws_bytes, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* COMBA_LAYER_H */
