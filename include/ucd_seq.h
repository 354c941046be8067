/*
 * ucd -- sequence operators: group norm with an activation, short causal convolution and
 * selective state space scan, with their gradients and, for decoding, their single-token forms.
 *
 * Conventions beside those of ucd.h (device pointers, caller-owned buffers and stream, status
 * codes, no allocation, no synchronisation, nothing launched by a call that fails)
 *   - Channels are the last extent and contiguous.  Every activation tensor has two strides, in
 *     elements, of its sequence (sample) and of its token (position); 0 stands for the dense one.
 *     An extent is at most 2^30, a row 2^25 elements, a tensor 2^40; rows must not overlap, a
 *     token's stride is at most 2^25 and a sequence's 2^40 (UCD_E_INVALID otherwise), but for
 *     those of an extent of one, which are not taken; a gradient has the strides of its tensor.
 *     Calls that would be 2^31 workgroups (the scan's 2^30) are UCD_E_UNSUPPORTED.
 *   - dtype 0: activations (and their gradients, filters and convolution states) fp32; dtype 1:
 *     bfloat16, rounded to nearest-even once.  Everything else is fp32: norm weights, biases, A,
 *     skip, scan states, statistics, gradients of all weights; and so is all arithmetic.
 *   - Any alignment of an element's own size is accepted, of workspaces and saved states 16 bytes.
 *   - Outputs overlap no input and no other output, but for state_out == state_in.
 *   - Gradients of weights are beta * old + sum, beta in {0, 1}, as in ucd_conv_bwd_filter: a
 *     mini-batch may be run in parts.  beta = 0 ignores old contents.
 *   - Sums are taken in a fixed order: outputs are bit-identical from run to run, whether or not
 *     ucd_set_deterministic is on.
 *   - lengths (may be NULL): device, int32 per sequence, taken between 0 and L.  Tokens from a
 *     sequence's length on are padding: their inputs are not read (they may hold NaN), their
 *     outputs and gradients are 0.
 *   - slots (may be NULL): device, int32 per sequence, its place in a pool of n_slots states.  A
 *     place outside 0 .. n_slots-1 marks an idle sequence: no state is read or written and its
 *     outputs are 0.  Sequences of one call have places of their own.  Without slots the states
 *     are one per sequence (n_slots = 0); a pool without slots goes with no sequences alone.
 */
#ifndef UCD_SEQ_H
#define UCD_SEQ_H

#include "ucd.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Activations; SiLU(v) = v / (1 + exp(-v)). */
enum { UCD_ACT_NONE = 0, UCD_ACT_SILU = 1 };

/* The directions of an operator, for workspace queries. */
enum { UCD_SEQ_FWD = 0, UCD_SEQ_BWD = 1 };

/* ---- group norm with an activation ------------------------------------------------------------
 * x (N, S, C): N samples of S positions; the C channels are G groups of C/G neighbours.  Mean and
 * variance (divided by the number of elements) are over the S positions and C/G channels of a
 * sample's group:
 *   y = act(gamma * (x - mean) * rstd + beta),  rstd = 1 / sqrt(var + eps).
 * S = 1 normalises single tokens; G = 1 all channels together.  N, S, C, G >= 1, G divides C. */
typedef struct {
    int32_t N, S, C, G, act, dtype;
    float eps;
    int64_t x_n, x_s, y_n, y_s;   /* strides of x, dx and of y, dy */
} ucd_group_norm_t;

/* Bytes of workspace of a direction; UCD_WS_NA for an invalid descriptor.  Host only. */
size_t ucd_group_norm_workspace_size(const ucd_group_norm_t *norm, int dir);

/* stats (may be NULL): device, 2*N*G floats, receives mean[N][G] and rstd[N][G] for Backward. */
int ucd_group_norm_fwd(const ucd_group_norm_t *norm, const void *x, const float *gamma, const float *beta_w,
                       void *y, float *stats, void *ws, size_t ws_bytes, void *stream);

/* dx, dgamma[C], dbeta[C] from dy and Forward's x and stats. */
int ucd_group_norm_bwd(const ucd_group_norm_t *norm, const void *x, const float *gamma, const float *beta_w,
                       const float *stats, const void *dy, void *dx, float *dgamma, float *dbeta, float beta,
                       void *ws, size_t ws_bytes, void *stream);

/* ---- short causal convolution -----------------------------------------------------------------
 * x (B, L, D), w (D, K), every channel by itself:
 *   y_t = act(bias + sum_k w[k] x_{t-K+1+k}),
 * tokens before the first come from the state (K-1, D), oldest first, or are 0.  1 <= K <= 8;
 * B, L >= 0. */
typedef struct {
    int32_t B, L, D, K, act, dtype;
    int32_t n_slots;
    int64_t x_b, x_l, y_b, y_l;   /* strides of x, dx and of y, dy */
} ucd_causal_conv_t;

/* Bytes of workspace of Backward (Forward and the step need none). */
size_t ucd_causal_conv_workspace_size(const ucd_causal_conv_t *conv);

/* state_in (NULL: zeros), state_out (NULL: not wanted): (n_slots or B, K-1, D); state_out receives
 * the last K-1 tokens of state_in and the sequence.  bias may be NULL. */
int ucd_causal_conv_fwd(const ucd_causal_conv_t *conv, const void *x, const void *w, const float *bias,
                        const int32_t *lengths, const int32_t *slots, const void *state_in, void *state_out,
                        void *y, void *stream);

/* Backward, without slots.  dstate_out (NULL: zeros) is the gradient of state_out, dstate_in (NULL:
 * not wanted) receives that of state_in, both (B, K-1, D); dbias (NULL: not wanted). */
int ucd_causal_conv_bwd(const ucd_causal_conv_t *conv, const void *x, const void *w, const float *bias,
                        const int32_t *lengths, const void *state_in, const void *dy, const void *dstate_out,
                        void *dx, float *dw, float *dbias, void *dstate_in, float beta,
                        void *ws, size_t ws_bytes, void *stream);

/* One token of each sequence (L = 1): as Forward with state_in = state_out = state. */
int ucd_causal_conv_step(const ucd_causal_conv_t *conv, const void *x, const void *w, const float *bias,
                         const int32_t *slots, void *state, void *y, void *stream);

/* ---- selective state space scan ---------------------------------------------------------------
 * u, dt, z, y (B, L, D); A (D, N); Bm, Cm (B, L, G, N): the D channels are G groups of neighbours
 * that share Bm and Cm; skip, dt_bias (D).  Every channel has N states:
 *   d_t = dt_t + dt_bias, with softplus: d_t = log(1 + exp(dt_t + dt_bias)),
 *   h_t = exp(d_t A) h_{t-1} + d_t u_t Bm_t,      h_{-1} = state_in or 0,
 *   y_t = (sum_n Cm_t h_t + skip u_t) * SiLU(z_t).
 * Without skip, z, dt_bias (NULL) their terms are left out.  1 <= N <= 64; G divides D. */
typedef struct {
    int32_t B, L, D, N, G, dtype, softplus;
    int32_t n_slots;
    int64_t u_b, u_l, dt_b, dt_l, Bm_b, Bm_l, Cm_b, Cm_l, z_b, z_l, y_b, y_l;
} ucd_scan_t;

typedef struct {
    const void *u, *dt;
    const float *A;
    const void *Bm, *Cm;
    const float *skip;        /* may be NULL */
    const void *z;            /* may be NULL */
    const float *dt_bias;     /* may be NULL */
    const int32_t *lengths;   /* may be NULL */
    const int32_t *slots;     /* may be NULL */
} ucd_scan_in_t;

/* Receivers of the gradients: skip, z and dt_bias as in the inputs; state (the gradient of
 * state_in, (B, D, N)) may be NULL. */
typedef struct {
    void *u, *dt;
    float *A;
    void *Bm, *Cm;
    float *skip;
    void *z;
    float *dt_bias;
    float *state;
} ucd_scan_grad_t;

/* Bytes of workspace of a direction, and of what Forward keeps for Backward (states at regular
 * distances).  Host only. */
size_t ucd_scan_workspace_size(const ucd_scan_t *scan, int dir);
size_t ucd_scan_saved_size(const ucd_scan_t *scan);

/* state_in (NULL: zeros), state_out (NULL: not wanted): (n_slots or B, D, N) floats.  saved (NULL:
 * no Backward will follow): ucd_scan_saved_size bytes. */
int ucd_scan_fwd(const ucd_scan_t *scan, const ucd_scan_in_t *in, const float *state_in, float *state_out,
                 void *y, void *saved, size_t saved_bytes, void *ws, size_t ws_bytes, void *stream);

/* Backward, without slots; saved is what Forward wrote for the same inputs.  dstate_out (NULL:
 * zeros): gradient of state_out, (B, D, N) floats. */
int ucd_scan_bwd(const ucd_scan_t *scan, const ucd_scan_in_t *in, const void *dy, const float *dstate_out,
                 const void *saved, size_t saved_bytes, const ucd_scan_grad_t *grad, float beta,
                 void *ws, size_t ws_bytes, void *stream);

/* One token of each sequence (L = 1; lengths is not read): as Forward with state_in = state_out = state. */
int ucd_scan_step(const ucd_scan_t *scan, const ucd_scan_in_t *in, float *state, void *y, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* UCD_SEQ_H */
