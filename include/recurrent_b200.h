/*
 * recurrent_b200 -- what a layer of a recurrent language model needs next to the operators of sequence_b200.h: the gated delta
 * rule (a state that forgets, corrects what it holds for a key and answers a query), over prompts, single tokens and training steps, and
 * the RMS norm at the layer's entry (with the residual's addition, in 8 bits for its projections), of its heads, and at its exit (with a gate).
 *
 * The conventions of sequence_b200.h hold: types, rows and their distances, alignment, lengths, workspaces, errors, results that do not
 * depend on timing.
 */
#ifndef RECURRENT_B200_H
#define RECURRENT_B200_H

#include "sequence_b200.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Gated delta rule.  Every head h < H has a state S, K rows of V numbers.  With the query and the key of head h / (H / Hk) (Hk divides H):
 *   S' = e^g S_{t-1},   u = beta (v - S'^T k),   S_t = S' + k u^T,   o = scale S_t^T q.
 *   q, k [B*L][Hk*K] (ldq, ldk); v, o [B*L][H*V] (ldv, ldo); g, beta [B*L][H] fp32 (ldg, ldbeta); 1 <= K <= 128, 1 <= V <= 65536.
 *   state_in, state_out [B][H][K][V] fp32, dense, optional (zeros); state_out is S after the last token (state_in, or zeros, for a sequence
 *   without tokens) and may be the same buffer as state_in.
 * g is a log decay: 0 keeps, -infinity forgets (below -10000 is taken as that).  Sequences are computed in pieces of 64 tokens: a key, value,
 * query, beta or other decay that is not finite spoils the whole piece that it is in and all that follows in its head and sequence (and, backward, what comes before
 * it there), and nothing else.
 * Products run on the tensor cores, sums and states as operands in three bf16 numbers each (24 bits).
 * states (optional): what the backward pass continues from, delta_states_size bytes, aligned to 16; the caller keeps it until then.  For every 64 tokens of a head
 * 49 KB and 4 (K' + 64) V' bytes, K' = 64 or 128, V' = V rounded up to 16 (8192 tokens of 16 heads of 128 x 128: 305 MB, nine times v in bf16).
 * A batch can be taken in pieces.
 * B * H * ceil(L / 64) * ceil(V / 16) is below 2^31.
 * Waits on the device are bounded; should one expire, the results are not defined and conv2d_get_status(NULL, cuda_stream) says so (CONV2D_ERR_DEVICE_TIMEOUT).
 */
conv2d_status_t delta_states_size(int B, int L, int Hk, int H, int K, int V, conv2d_operand_t type, size_t* bytes);
conv2d_status_t delta_fwd_gated_workspace_size(int B, int L, int Hk, int H, int K, int V, conv2d_operand_t type, size_t* bytes);
conv2d_status_t delta_fwd_gated(const void* q, const void* k, const void* v, const float* g, const float* beta,
                                const float* state_in, const int* lengths, void* o, float* state_out, void* states,
                                int B, int L, int Hk, int H, int K, int V, long long ldq, long long ldk, long long ldv,
                                long long ldg, long long ldbeta, long long ldo, float scale, conv2d_operand_t type,
                                void* workspace, size_t workspace_bytes, void* cuda_stream);

/* One token of every sequence: q, k [B][Hk*K]; v, o [B][H*V]; g, beta [B][H]; state_in, state_out required, may be the same buffer. */
conv2d_status_t delta_step_gated(const void* q, const void* k, const void* v, const float* g, const float* beta,
                                 const float* state_in, void* o, float* state_out,
                                 int B, int Hk, int H, int K, int V, long long ldq, long long ldk, long long ldv,
                                 long long ldg, long long ldbeta, long long ldo, float scale, conv2d_operand_t type, void* cuda_stream);

/*
 * Backward: from the gradient dout of o [B*L][H*V] (lddo) and, optional, dstate_out [B][H][K][V] (the gradient of state_out) the gradients
 * dq, dk [B*L][Hk*K], dv [B*L][H*V] of `type`, and in fp32 dg, dbeta [B*L][H] and, optional, dstate_in [B][H][K][V].
 * q, k, lengths, scale as given to the forward pass; `states` as that left it (it holds all else).
 */
conv2d_status_t delta_bwd_gated_workspace_size(int B, int L, int Hk, int H, int K, int V, conv2d_operand_t type, size_t* bytes);
conv2d_status_t delta_bwd_gated(const void* q, const void* k, const int* lengths, const void* states, const void* dout, const float* dstate_out,
                                void* dq, void* dk, void* dv, float* dg, float* dbeta, float* dstate_in,
                                int B, int L, int Hk, int H, int K, int V, long long ldq, long long ldk, long long lddo,
                                long long lddq, long long lddk, long long lddv, long long lddg, long long lddbeta,
                                float scale, conv2d_operand_t type, void* workspace, size_t workspace_bytes, void* cuda_stream);

/*
 * RMS norm of M rows of C <= 16384 channels in G groups (G divides C), each normalised by itself:
 *   h = x + residual, rounded to `type` (h = x where residual is NULL),   r = 1 / sqrt(mean(h^2) + eps),   n = gamma[c % (C/G)] h r,
 *   y = n * silu(z)   (y = n where z is NULL).   With eps of zero a group of zeros becomes NaN.
 *   The mean is of squares in fp32: numbers up to 2^63 are normalised; from 2^64 on it is infinite and the group becomes zeros.  Squares of numbers below 2^-63 lose
 *   digits, and vanish below 2^-75, which only an eps as small shows.
 *   x, residual (optional), z (optional), y [M][C] (ldx, ldr, ldz, ldy); gamma [C/G] fp32, optional (1); eps >= 0.
 *   h [M][C] (ldh): required exactly where residual is given; the residual of the next layer.  It may be the same tensor as residual, or x.
 *   rstd [M][G] fp32, optional: r, for the backward pass.
 *   y8 [M][C] bytes (ld8), scales [M][ceil(C/block)] fp32: y in 8 bits (e4m3), both or neither; at least one of y and y8.  Every `block` adjacent columns of
 *   a row (the last ones may be fewer) share a scale s = max |y| / 448, at least 2^-126, and y8 = y / s, rounded to nearest, even.
 *   A block of more than C columns is the row.  block is not looked at without y8.  What is rounded is y before it is rounded to `type`.
 *   A NaN keeps its place and does not count for the scale; a block with an infinity has an infinite scale, its finite numbers become zeros, its infinities NaN.
 */
conv2d_status_t norm_fwd_rms(const void* x, const void* residual, const void* z, const float* gamma, void* y, void* h,
                             void* y8, float* scales, float* rstd, int M, int C, int G, int block,
                             long long ldx, long long ldr, long long ldz, long long ldy, long long ldh, long long ld8,
                             float eps, conv2d_operand_t type, void* cuda_stream);

/*
 * Backward: from dy [M][C] and, optional, dh [M][C] (the gradient that reaches h on its way past this layer) the gradients
 *   dx [M][C], of x and of residual alike (may be the same tensor as dy or dh); dz [M][C], required exactly where z is given;
 *   dgamma [C/G] fp32, optional.   h as the forward pass left it (x without a residual), rstd likewise.
 * workspace is required unless dgamma is NULL.
 */
conv2d_status_t norm_bwd_rms_workspace_size(int M, int C, int G, size_t* bytes);
conv2d_status_t norm_bwd_rms(const void* h, const void* z, const float* gamma, const float* rstd, const void* dy, const void* dh,
                             void* dx, void* dz, float* dgamma, int M, int C, int G,
                             long long ldh, long long ldz, long long lddy, long long lddh, long long lddx, long long lddz,
                             conv2d_operand_t type, void* workspace, size_t workspace_bytes, void* cuda_stream);

#ifdef __cplusplus
}
#endif
#endif /* RECURRENT_B200_H */
