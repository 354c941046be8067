/*
 * ucd -- linear attention and gated projection: sequence operators of the models' larger parts, with
 * their gradients and, for decoding, their forms for single tokens.
 *
 * The conventions are those of ucd_seq.h, but for two:
 *   - The products' operands are bfloat16 where dtype is 1 (what is computed on the way is rounded to
 *     it once; what is added to a state is not), with sums in fp32: where another operand is rounded
 *     beside the output itself, errors are 2.4e-3 in the 2-norm instead of 1.7e-3.  fp32 operands are
 *     multiplied as matrix instructions of fp32 or as parts of three bfloat16: some 5e-7 (attention)
 *     and 1e-6 (gated projection).
 *   - The gated projection's weights and their gradients are of the activations' type.
 */
#ifndef UCD_MIX_H
#define UCD_MIX_H

#include "ucd_seq.h"

#ifdef __cplusplus
extern "C" {
#endif

/* A further activation, of the gated projection alone: GELU in its tanh form,
 * v (1 + tanh(sqrt(2/pi) (v + 0.044715 v^3))) / 2. */
enum { UCD_ACT_GELU = 2 };

/* ---- linear attention with a decay for each head -------------------------------------------------
 * q, k (B, L, Hk, Dk), v, y (B, L, H, Dv), g (B, L, H): each of the Hk heads of q and k serves H/Hk
 * neighbouring heads of v.  Every head has a state of Dk by Dv, rows of Dv:
 *   l_t = decay + g_t,   S_t = exp(l_t) S_{t-1} + k_t^T v_t,   S_{-1} = state_in or 0,
 *   y_t = scale q_t S_t.
 * decay (H) are constants of the heads, g the decays' own part for every token, both logarithms and
 * at most 0 together; without either (NULL) its term is left out.  What is below -80 counts as -80,
 * exp of which is as good as 0: -infinity forgets what was before the token, and has no gradient.
 * Tokens are taken 64 at a time, from a sequence's first on: a value that is not finite may reach all
 * 64 outputs and gradients around it, beside those of the formulas.  1 <= Dk, Dv <= 128 (wider heads of v are more heads of v to
 * one of q and k); Hk divides H; B, L >= 0.  Rows of q, k, v, g and y, and a token's stride of
 * theirs, are at most 2^23 elements. */
typedef struct {
    int32_t B, L, H, Hk, Dk, Dv, dtype;
    int32_t n_slots;
    float scale;
    int64_t q_b, q_l, k_b, k_l, v_b, v_l, g_b, g_l, y_b, y_l;
} ucd_linear_attention_t;

typedef struct {
    const void *q, *k, *v;
    const void *g;            /* may be NULL */
    const float *decay;       /* may be NULL */
    const int32_t *lengths;   /* may be NULL */
    const int32_t *slots;     /* may be NULL */
} ucd_linear_attention_in_t;

/* Receivers of the gradients: g (where the input has it) and state (the gradient of state_in,
 * (B, H, Dk, Dv)) may be NULL. */
typedef struct {
    void *q, *k, *v, *g;
    float *state;
} ucd_linear_attention_grad_t;

/* Bytes of workspace of a direction, and of what Forward keeps for Backward.  Host only. */
size_t ucd_linear_attention_workspace_size(const ucd_linear_attention_t *attention, int dir);
size_t ucd_linear_attention_saved_size(const ucd_linear_attention_t *attention);

/* state_in (NULL: zeros), state_out (NULL: not wanted): (n_slots or B, H, Dk, Dv) floats.  saved (NULL:
 * no Backward will follow): ucd_linear_attention_saved_size bytes. */
int ucd_linear_attention_fwd(const ucd_linear_attention_t *attention, const ucd_linear_attention_in_t *in,
                             const float *state_in, float *state_out, void *y, void *saved, size_t saved_bytes,
                             void *ws, size_t ws_bytes, void *stream);

/* Backward, without slots; saved is what Forward wrote for the same inputs.  dstate_out (NULL: zeros):
 * gradient of state_out, (B, H, Dk, Dv) floats.  Sums for g's gradient run in another order: q's and k's may
 * round to another last bit than without it.  Nothing else that is left out changes what is written. */
int ucd_linear_attention_bwd(const ucd_linear_attention_t *attention, const ucd_linear_attention_in_t *in,
                             const void *dy, const float *dstate_out, const void *saved, size_t saved_bytes,
                             const ucd_linear_attention_grad_t *grad, void *ws, size_t ws_bytes, void *stream);

/* One token of each sequence (L = 1; lengths is not read): as Forward with state_in = state_out = state. */
int ucd_linear_attention_step(const ucd_linear_attention_t *attention, const ucd_linear_attention_in_t *in,
                              float *state, void *y, void *stream);

/* ---- gated projection ---------------------------------------------------------------------------
 * Both projections of a gated feed-forward block, its activation and its product: x (M, D), one row a
 * token, w_gate, w_up (F, D) with dense rows of x's type, y (M, F):
 *   y = act(x w_gate^T) * (x w_up^T).
 * The weights' gradients are of the weights' type: in bfloat16 they are rounded once, and parts of a
 * mini-batch (beta = 1) once each.  dgate and dup, the gradients of both projections, are rounded once
 * to bfloat16 before they are multiplied where dtype is 1.  fp32 operands are multiplied as three
 * bfloat16 parts each, to about 2^-22 of a product; sums of one that is not finite are not finite.
 * 1 <= D, F <= 2^20, a row's stride 2^21 at most; M >= 0. */
typedef struct {
    int32_t M, D, F, act, dtype;
    int64_t x_m, y_m;             /* strides of x, dx and of y, dy */
} ucd_gated_projection_t;

/* Bytes of workspace of a direction, and of what Forward keeps for Backward (both projections, fp32).
 * Host only. */
size_t ucd_gated_projection_workspace_size(const ucd_gated_projection_t *gated, int dir);
size_t ucd_gated_projection_saved_size(const ucd_gated_projection_t *gated);

/* saved (NULL: no Backward will follow): ucd_gated_projection_saved_size bytes. */
int ucd_gated_projection_fwd(const ucd_gated_projection_t *gated, const void *x, const void *w_gate, const void *w_up,
                             void *y, void *saved, size_t saved_bytes, void *ws, size_t ws_bytes, void *stream);

/* dx, dw_gate, dw_up (weights' type) from dy and what Forward kept for the same inputs. */
int ucd_gated_projection_bwd(const ucd_gated_projection_t *gated, const void *x, const void *w_gate, const void *w_up,
                             const void *dy, const void *saved, size_t saved_bytes, void *dx, void *dw_gate,
                             void *dw_up, float beta, void *ws, size_t ws_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* UCD_MIX_H */
