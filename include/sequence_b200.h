/*
 * sequence_b200 -- operators along a sequence that stand next to the convolutions of conv2d_b200.h, for models that
 * convolve, scan and normalise tensors whose channels lie together ("channels last"): the short causal convolution
 * of every channel, the selective state space scan that reads its output, and group norm with an activation.
 * Each has a forward and a backward pass; the first two also a form for one token of every sequence.
 *
 * Conventions (beyond those of conv2d_b200.h, which hold except where this says otherwise)
 *   - `type` names the element type of all `void` tensors of a call: CONV2D_OPERAND_BF16, _FP16 or _FP32.  `float` tensors are
 *     fp32 whatever the type.  Arithmetic, sums, statistics and states are fp32; a result of a shorter type is
 *     rounded once, to nearest.
 *   - Tensors are dense but for the distance between rows: row r of a tensor begins r * ld elements after its first
 *     element, ld at least the length of a row (a slice of a wider tensor's columns has the wider tensor's ld).  Row of
 *     sequence b and token t: b * L + t.
 *     There are at most 2^30 rows and 2^22 channels, ld is below 2^31; offsets may exceed 32 bits.
 *   - Addresses need the alignment of their elements only; rows on 16-byte boundaries are faster.
 *   - `lengths`: NULL, or B device integers (values outside 0 .. L are taken as the nearest of these): sequence b has
 *     lengths[b] tokens and the rows behind them are padding.  Padding is not read, whatever it holds, and the rows of outputs that
 *     belong to it are written as zeros.
 *   - Pointers described as optional may be NULL.  Outputs must not overlap inputs or each other, except where noted.
 *   - Workspaces: the size comes from the query of the same name; any alignment of 16 bytes.  They hold nothing between calls,
 *     so calls in a row on one stream may share one, calls that can overlap must not.
 *   - Results do not depend on timing: the same call gives the same bits (no atomic additions).
 *   - Errors: CONV2D_ERR_NULL, _SHAPE (extents beyond these, a row distance below the row's length), _ALIGN, _UNSUPPORTED (an unknown type, activation or
 *     flag, more taps or states than stated), _WORKSPACE, as argument errors before anything is enqueued; _ARCH, _CUDA.
 */
#ifndef SEQUENCE_B200_H
#define SEQUENCE_B200_H

#include "conv2d_b200.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    CONV2D_ACT_NONE = 0,
    CONV2D_ACT_RELU = 1,
    CONV2D_ACT_SILU = 2,  /* v / (1 + e^-v) */
    CONV2D_ACT_GELU = 3   /* v (1 + erf(v / sqrt 2)) / 2, its digits kept where it is small */
} conv2d_activation_t;

/*
 * Causal convolution of every channel with its own K taps, 1 <= K <= 8:
 *   a[b,t,d] = bias[d] + sum_k w[d,k] * xe[b,t-(K-1)+k,d],   y = act(a),
 * xe being x with the K-1 rows of state_in before its first row (zeros where state_in is NULL).
 *   x, y [B*L][D] (ldx, ldy); w [D][K]; bias [D], optional; state_in, state_out [B][K-1][D], dense, optional.
 * state_out: the last K-1 rows of xe in front of the padding (what the next piece of the sequence, or its next token, continues from);
 * it may be the same buffer as state_in.
 */
conv2d_status_t conv1d_fwd_causal(const void* x, const void* w, const void* bias, const void* state_in, const int* lengths,
                                  void* y, void* state_out, int B, int L, int D, int K, long long ldx, long long ldy,
                                  conv2d_operand_t type, conv2d_activation_t act, void* cuda_stream);

/* One token of every sequence: x, y [B][D]; state_in and state_out (required for K > 1; may be the same buffer) as above. */
conv2d_status_t conv1d_step_causal(const void* x, const void* w, const void* bias, const void* state_in, void* y, void* state_out,
                                   int B, int D, int K, long long ldx, long long ldy,
                                   conv2d_operand_t type, conv2d_activation_t act, void* cuda_stream);

/*
 * Backward: from dy [B*L][D] (lddy) and, optional, dstate_out [B][K-1][D] (the gradient of state_out) the gradients
 *   dx [B*L][D] (lddx), dw [D][K] and dbias [D] (fp32; each optional), dstate_in [B][K-1][D] (optional).
 * x, w, bias, state_in, lengths as given to the forward pass.  workspace is required unless both dw and dbias are NULL.
 */
conv2d_status_t conv1d_bwd_causal_workspace_size(int B, int L, int D, int K, size_t* bytes);
conv2d_status_t conv1d_bwd_causal(const void* x, const void* w, const void* bias, const void* state_in, const int* lengths,
                                  const void* dy, const void* dstate_out, void* dx, float* dw, float* dbias, void* dstate_in,
                                  int B, int L, int D, int K, long long ldx, long long lddy, long long lddx,
                                  conv2d_operand_t type, conv2d_activation_t act,
                                  void* workspace, size_t workspace_bytes, void* cuda_stream);

/* `flags` of the scan */
enum {
    CONV2D_FLAG_SCAN_SOFTPLUS = 1u   /* step sizes are log(1 + e^v) of v = delta + delta_bias, else v itself */
};

/*
 * Selective state space scan.  With s = delta + delta_bias (softplus of it with CONV2D_FLAG_SCAN_SOFTPLUS):
 *   h_t[d,n] = exp(s_t[d] A[d,n]) h_{t-1}[d,n] + s_t[d] u_t[d] Bm_t[g,n]
 *   v_t[d]   = sum_n Cm_t[g,n] h_t[d,n] + Dskip[d] u_t[d],     y = v * silu(z)   (y = v where z is NULL)
 * for channels d < D in G groups of D / G channels that share Bm and Cm (g = d / (D / G); G divides D), 1 <= N <= 128 states.
 *   u, delta, z (optional), y [B*L][D]; Bm, Cm [B*L][G*N] (rows of ldB, ldC elements);
 *   A [D][N], Dskip [D] (optional), delta_bias [D] (optional), state_in, state_out [B][D][N] (optional): fp32.
 * state_out is h after the last token (state_in, or zeros, for a sequence without tokens); it may be the same buffer as state_in.
 * states (optional): what the backward pass continues from, scan_states_size bytes; the caller keeps it until then.
 */
conv2d_status_t scan_states_size(int B, int L, int D, int N, size_t* bytes);
conv2d_status_t scan_fwd_selective_workspace_size(int B, int L, int D, int N, int G, size_t* bytes);
conv2d_status_t scan_fwd_selective(const void* u, const void* delta, const float* A, const void* Bm, const void* Cm,
                                   const float* Dskip, const void* z, const float* delta_bias,
                                   const float* state_in, const int* lengths, void* y, float* state_out, void* states,
                                   int B, int L, int D, int N, int G, long long ldu, long long lddelta,
                                   long long ldB, long long ldC, long long ldz, long long ldy,
                                   conv2d_operand_t type, unsigned flags,
                                   void* workspace, size_t workspace_bytes, void* cuda_stream);

/* One token of every sequence: u, delta, z, y [B][D]; Bm, Cm [B][G*N]; state_in, state_out required, may be the same buffer. */
conv2d_status_t scan_step_selective(const void* u, const void* delta, const float* A, const void* Bm, const void* Cm,
                                    const float* Dskip, const void* z, const float* delta_bias,
                                    const float* state_in, void* y, float* state_out,
                                    int B, int D, int N, int G, long long ldu, long long lddelta,
                                    long long ldB, long long ldC, long long ldz, long long ldy,
                                    conv2d_operand_t type, unsigned flags, void* cuda_stream);

/*
 * Backward: from dy [B*L][D] and, optional, dstate_out [B][D][N] (the gradient of state_out) the gradients of every input, du, ddelta,
 * dz (required exactly where z is given) [B*L][D], dB, dC [B*L][G*N] of `type`, and in fp32 dA [D][N], dDskip [D] (optional),
 * ddelta_bias [D] (optional), dstate_in [B][D][N] (optional).  `states` as the forward pass of the same inputs left it.
 * The workspace grows with the tensors: 4 bytes for every element of u with up to 16 states, 16 with 64, 64 with 128 (more where channels are few), so
 * that training with many states wants it larger than all tensors together; `states` takes N / 4 bytes for every element.  A batch can be taken in pieces.
 */
conv2d_status_t scan_bwd_selective_workspace_size(int B, int L, int D, int N, int G, size_t* bytes);
conv2d_status_t scan_bwd_selective(const void* u, const void* delta, const float* A, const void* Bm, const void* Cm,
                                   const float* Dskip, const void* z, const float* delta_bias, const int* lengths,
                                   const void* states, const void* dy, const float* dstate_out,
                                   void* du, void* ddelta, float* dA, void* dB, void* dC, float* dDskip, void* dz,
                                   float* ddelta_bias, float* dstate_in,
                                   int B, int L, int D, int N, int G, long long ldu, long long lddelta,
                                   long long ldB, long long ldC, long long ldz, long long lddy,
                                   long long lddu, long long ldddelta, long long lddB, long long lddC, long long lddz,
                                   conv2d_operand_t type, unsigned flags,
                                   void* workspace, size_t workspace_bytes, void* cuda_stream);

/*
 * Group norm with an activation: N samples of S positions (rows) of C channels in G groups (G divides C),
 *   m, q = mean and variance over the S * C/G elements of sample n and group g,   rstd = 1 / sqrt(q + eps),
 *   y = act(gamma[c] (x - m) rstd + beta[c]).
 * With S = 1 every row is normalised by itself (the heads of a token).
 *   x, y [N*S][C] (ldx, ldy); gamma, beta [C] fp32, each optional (1 and 0); mean, rstd [N][G] fp32, optional; eps >= 0.
 */
conv2d_status_t norm_fwd_groups_workspace_size(int N, int S, int C, int G, size_t* bytes);
conv2d_status_t norm_fwd_groups(const void* x, const float* gamma, const float* beta, void* y, float* mean, float* rstd,
                                int N, int S, int C, int G, long long ldx, long long ldy, float eps,
                                conv2d_operand_t type, conv2d_activation_t act,
                                void* workspace, size_t workspace_bytes, void* cuda_stream);

/* Backward: mean and rstd as the forward pass left them; dx [N*S][C] (lddx), dgamma, dbeta [C] fp32 (each optional). */
conv2d_status_t norm_bwd_groups_workspace_size(int N, int S, int C, int G, size_t* bytes);
conv2d_status_t norm_bwd_groups(const void* x, const float* gamma, const float* beta, const float* mean, const float* rstd,
                                const void* dy, void* dx, float* dgamma, float* dbeta,
                                int N, int S, int C, int G, long long ldx, long long lddy, long long lddx,
                                conv2d_operand_t type, conv2d_activation_t act,
                                void* workspace, size_t workspace_bytes, void* cuda_stream);

#ifdef __cplusplus
}
#endif
#endif /* SEQUENCE_B200_H */
