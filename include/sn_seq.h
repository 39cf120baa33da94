/*
 * sn_seq.h -- layers along token sequences: the short causal convolution, the norm of heads with the position
 * rotation, and the selective state space scan; forward, backward and for single tokens.
 *
 * They are the layer level of a memory-budgeted training step (SuperNeurons, arXiv 1801.04380) like the CONV, BN and
 * LRN calls of sn.h, and its conventions hold: device pointers owned by the caller, work enqueued on `stream`, no
 * allocation, no synchronisation, outputs overwritten, sn_status returned before anything is launched.  What differs:
 *  - A token tensor is rows x channels, one token a row, channels contiguous, rows `ld` elements apart (a column
 *    slice of a wider tensor is fine).  Token tensors, filters and 16-bit states are of `dtype` and aligned to one
 *    element; everything else is fp32 (or int32) and aligned to 4 bytes; workspaces are 256-byte aligned.
 *  - Sequences lie packed one behind the other.  seq_offsets == NULL: `seqs` sequences of rows / seqs rows each
 *    (seqs must divide rows).  Otherwise int32[seqs + 1] in device memory, ascending: sequence s is the rows
 *    seq_offsets[s] .. seq_offsets[s+1] - 1.  Empty sequences are allowed.  Rows that no sequence holds (behind the last, in
 *    front of the first) are neither read for any result nor written.  Offsets that descend, or leave 0 .. rows, give undefined results, but no access
 *    outside the tensors.
 *  - Sizes, SN_ERR_UNSUPPORTED beyond: rows 2^30 (of a step call 2^24 - 1), sequences 2^24 - 1, channels of the convolution 65535 * 256,
 *    channels of the scan 65535 blocks of 16 of one group, heads of queries and keys together 2^20.  Addresses are 64-bit.  rows = 0 is a valid call.
 *  - Outputs must not overlap inputs or each other, except where a call says so.
 *  - Arithmetic, states and sums are fp32; a result of `dtype` is rounded once.  Sums are in a fixed order: results are
 *    run-to-run identical.  Those over rows are as exact as sums of about 256 terms, however many rows there are.
 */
#ifndef SN_SEQ_H
#define SN_SEQ_H

#include "sn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- short causal convolution along the tokens, one filter per channel -------------------------------------------
 *   p[t,d] = bias[d] + sum_{j < width} w[d][j] * x[t - (width-1) + j, d],      y = silu ? p * sigmoid(p) : p
 * The rows before a sequence's first are its initial state: state_in[s][width-1][channels], oldest first, or zeros
 * where state_in is NULL.  The final state, the sequence's last width-1 inputs (rows of the initial state among them where the
 * sequence is shorter), goes to state_out, if given, in the same layout. */
#define SN_CONV1D_MAX_WIDTH 8

typedef struct {
    int64_t rows;
    int32_t seqs, channels;
    int32_t width;             /* 1 .. SN_CONV1D_MAX_WIDTH */
    int32_t silu;              /* 0 / 1 */
    int32_t dtype;             /* of x, w, y, dy, dx and the states */
    int64_t ld_x, ld_y, ld_dx; /* row strides: of x, of y or dy, of dx (backward only) */
} sn_conv1d_shape;

/* bias (fp32 [channels]) may be NULL. */
sn_status sn_causal_conv1d_fwd(const void *x, const void *w, const float *bias, void *y, const sn_conv1d_shape *shape,
                               const int32_t *seq_offsets, const void *state_in, void *state_out, sn_stream stream);

/* Backward: from dy (and dstate_out, the gradient of the final state, or NULL) dx, dw (fp32 [channels][width]), dbias (fp32, may be
 * NULL) and dstate_in (the gradient of the initial state, or NULL); p is recomputed from x.  scratch: at least
 * sn_causal_conv1d_scratch_bytes(rows, channels, width), 256-byte aligned (SN_ERR_WORKSPACE_TOO_SMALL if smaller). */
size_t sn_causal_conv1d_scratch_bytes(int64_t rows, int32_t channels, int32_t width);
sn_status sn_causal_conv1d_bwd(const void *x, const void *w, const float *bias, const void *dy, void *dx, float *dw, float *dbias,
                               const sn_conv1d_shape *shape, const int32_t *seq_offsets, const void *state_in,
                               const void *dstate_out, void *dstate_in, void *scratch, size_t scratch_bytes,
                               sn_stream stream);

/* One token for each of shape->rows streams (shape->seqs is ignored): y from the stream's state and x, the new state into state_out.
 * state, state_out: [num_slots][width-1][channels]; row i works on slot slots[i], or on slot i where slots is NULL
 * (then rows <= num_slots).  A row whose slot is negative or >= num_slots is skipped, its y not written: the padding of a batch.
 * No slot may occur twice.  state_out may be state; in another buffer only the slots that occur are written. */
sn_status sn_causal_conv1d_step(const void *x, const void *w, const float *bias, void *y, const void *state, void *state_out,
                                const int32_t *slots, int32_t num_slots, const sn_conv1d_shape *shape, sn_stream stream);

/* ---- norm of queries and keys for each head, with the position rotation in the same pass -------------------------
 * Every head (head_dim neighbouring channels) of q and k:
 *   r = 1 / sqrt(mean(x^2) + eps),  n = x * r * weight,
 *   y: (n1, n2) -> (n1 cos a - n2 sin a, n2 cos a + n1 sin a),  a = positions[t] * inv_freq[i]
 * for the pairs i < rot_dim / 2, which are channels (i, i + rot_dim/2) of the head, or (2i, 2i+1) where interleaved; channels
 * from rot_dim on stay n.  An angle's fraction of a turn is formed in twice 64 bits: it is as good at position 2^31 as at 1.
 * positions: int32 [rows], any sign, or NULL for 0, 1, 2 ...; inv_freq: fp32 [rot_dim / 2] (NULL iff rot_dim = 0); wq, wk: fp32 [head_dim], or NULL for ones.
 * k may be absent (k_heads = 0, its pointers NULL).  yq may be q and yk k with the same row stride; so may dq be dyq and dk dyk. */
#define SN_HEADNORM_MAX_DIM 512

typedef struct {
    int64_t rows;
    int32_t q_heads, k_heads;   /* q_heads >= 1 */
    int32_t head_dim, rot_dim;  /* both even, rot_dim <= head_dim <= SN_HEADNORM_MAX_DIM */
    int32_t interleaved;
    int32_t dtype;
    float eps;                  /* > 0 */
    int64_t ld_q, ld_k;         /* row strides of q and k */
    int64_t ld_yq, ld_yk;       /* of yq and yk, or of dyq and dyk */
    int64_t ld_dq, ld_dk;       /* of dq and dk (backward only) */
} sn_headnorm_shape;

sn_status sn_headnorm_rot_fwd(const void *q, const void *k, const float *wq, const float *wk, const int32_t *positions,
                              const float *inv_freq, void *yq, void *yk, const sn_headnorm_shape *shape, sn_stream stream);

/* Backward: dq, dk, and the weights' gradients dwq, dwk (fp32 [head_dim], the sum over rows and heads; either may be NULL). */
size_t sn_headnorm_rot_scratch_bytes(int64_t rows, int32_t q_heads, int32_t k_heads, int32_t head_dim);
sn_status sn_headnorm_rot_bwd(const void *q, const void *k, const float *wq, const float *wk, const int32_t *positions,
                              const float *inv_freq, const void *dyq, const void *dyk, void *dq, void *dk, float *dwq, float *dwk,
                              const sn_headnorm_shape *shape, void *scratch, size_t scratch_bytes, sn_stream stream);

/* ---- selective state space scan ----------------------------------------------------------------------------------
 * Per channel d (of group g = d / (channels / groups)) and state n, along each sequence:
 *   delta = softplus ? log(1 + exp(dt + dt_bias)) : dt + dt_bias
 *   h[d,n] = exp(delta * A[d][n]) * h[d,n] + delta * u * B[t,g,n]
 *   y = (sum_n C[t,g,n] * h[d,n] + D[d] * u) * (z ? z * sigmoid(z) : 1)
 * u, dt, z, y: rows x channels; B, C: rows x (groups * states); A: fp32 [channels][states]; D, dt_bias: fp32 [channels].  D, dt_bias
 * and z may be NULL.  h0, hT: fp32 [seqs][channels][states], the initial (NULL: zeros) and the final state; hT may be NULL, and must
 * not overlap h0.  Row strides of the scan are 2^24 elements at most (SN_ERR_UNSUPPORTED).
 * Workspace and speed: a call needs parallel work beyond channels x sequences only where these are few; then it cuts the
 * tokens into chunks whose states are joined through the workspace.  With less than preferred_bytes it cuts into fewer chunks, with
 * the least into none; the result differs by the rounding of the joins only. */
#define SN_SCAN_MAX_STATES 64
typedef enum { SN_SCAN_FWD = 0, SN_SCAN_BWD = 1 } sn_scan_dir;

typedef struct {
    int64_t rows;
    int32_t seqs, channels, states, groups; /* states <= SN_SCAN_MAX_STATES; groups divides channels */
    int32_t dtype;                          /* of u, dt, B, C, z, y and of their gradients */
    int32_t softplus;
    int32_t ragged;                         /* seq_offsets is given */
    int64_t ld_u, ld_dt, ld_b, ld_c, ld_z;  /* row strides of the inputs, */
    int64_t ld_y;                           /* of y or dy, */
    int64_t ld_du, ld_ddt, ld_db, ld_dc, ld_dz; /* and of the gradients (backward only) */
} sn_scan_shape;

/* The strides of shape are not looked at here.  For SN_SCAN_BWD both sizes are those of a call that is given `states`; a call that is not
 * needs sn_scan_states_bytes(shape) more.  Sequences of equal length ask for what ragged ones ask for where they are many and short (to 16 tokens, and
 * beyond as long as it saves more than an eighth); a few are walked side by side, with kept states and sums for whole tiles each. */
sn_status sn_scan_workspace_query(const sn_scan_shape *shape, sn_scan_dir dir, size_t *min_bytes, size_t *preferred_bytes);

/* What the backward pass needs of the forward pass: the state before every 16th token.  Kept (sn_scan_fwd's `states`) or left out and
 * replayed from the inputs by sn_scan_bwd (Sec. 3.4: recomputation); the results differ by the rounding of the joins only, as a replay may
 * cut the tokens elsewhere.  256-byte aligned. */
size_t sn_scan_states_bytes(const sn_scan_shape *shape);

sn_status sn_scan_fwd(const void *u, const void *dt, const float *A, const void *B, const void *C, const float *D, const void *z,
                      const float *dt_bias, void *y, const sn_scan_shape *shape, const int32_t *seq_offsets, const float *h0,
                      float *hT, float *states, void *workspace, size_t workspace_bytes, sn_stream stream);

/* Backward from dy and dhT (the gradient of the final state, or NULL).  du, ddt, dz (iff z), dB, dC of dtype; dA fp32 [channels][states];
 * dD (iff D), ddt_bias (iff dt_bias) fp32 [channels]; dh0 fp32 [seqs][channels][states] or NULL.  h0 as in the forward call.
 * states: as sn_scan_fwd left them for the same shape and inputs, or NULL.  A shape with rows = 0 gives zero sums and dh0 = dhT. */
sn_status sn_scan_bwd(const void *u, const void *dt, const float *A, const void *B, const void *C, const float *D, const void *z,
                      const float *dt_bias, const void *dy, void *du, void *ddt, float *dA, void *dB, void *dC, float *dD, void *dz,
                      float *ddt_bias, const sn_scan_shape *shape, const int32_t *seq_offsets, const float *h0, const float *states,
                      const float *dhT, float *dh0, void *workspace, size_t workspace_bytes, sn_stream stream);

/* One token for each of shape->rows streams (shape->seqs is ignored): state, state_out fp32 [num_slots][channels][states]; slots as for
 * sn_causal_conv1d_step.  state_out may be state. */
sn_status sn_scan_step(const void *u, const void *dt, const float *A, const void *B, const void *C, const float *D, const void *z,
                       const float *dt_bias, void *y, const float *state, float *state_out, const int32_t *slots, int32_t num_slots,
                       const sn_scan_shape *shape, sn_stream stream);

#ifdef __cplusplus
}
#endif
#endif /* SN_SEQ_H */
