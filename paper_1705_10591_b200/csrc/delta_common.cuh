// What the kernels of the gated delta rule share: pieces of 64 tokens, numbers as sums of bf16 parts, matrix products of those, layouts.
//
// A head's state S (K x V) runs through pieces of 64 tokens.  Within one, with G_i the sum of the log decays up to token i, S the state before it,
//   A_ij = e^(G_i - G_j) k_i.k_j (j < i),   P_ij = e^(G_i - G_j) q_i.k_j (j <= i),   t = (1 + A diag(beta))^-1 A   (strictly lower),
//   R = V - diag(e^G) K S,   E = R - t diag(beta) R,   O = scale (diag(e^G) Q S + P diag(beta) E),
//   S <- e^(G_63) S + K^T diag(e^(G_63 - G) beta) E.
// t holds neither the identity nor betas: both stay in fp32, and the backward pass uses the same t (beta may be zero).
// Every warp of the kernels that walk the pieces owns 16 columns of V for all of K and computes transposed, S^T [16][K] in the accumulators of its
// MMAs: accumulators have the layout of the next product's left operand, so R, E and S go from product to product in registers, and warps
// only share what comes from memory (K, Q, t, P).
#pragma once

#include "seq_common.cuh"
#include "recurrent_b200.h"

namespace conv2d_b200 {

constexpr int kPiece = 64;
constexpr int kFactors = 5;                                     // of a piece: e^G, e^(G_63 - G), beta, G in two floats
constexpr int kMost = 128;                                      // numbers of a key

// Numbers of bf16 that hold a tensor's element, and of those that hold sums and states: 16 bits with two (a rounding of 2^-8, of the rest of it again).
template <typename T> struct Parts;
template <> struct Parts<bf16> { static constexpr int in = 1, sum = 2, out = 1; };   // out: of what only goes to outputs of 8 bits
template <> struct Parts<fp16> { static constexpr int in = 2, sum = 2, out = 2; };
template <> struct Parts<float> { static constexpr int in = 3, sum = 3, out = 3; };
inline int parts_in(conv2d_operand_t t) { return t == CONV2D_OPERAND_BF16 ? 1 : t == CONV2D_OPERAND_FP16 ? 2 : 3; }
inline int parts_sum(conv2d_operand_t t) { return t == CONV2D_OPERAND_FP32 ? 3 : 2; }

// a, b as N parts each, the two of a part side by side.
template <int N>
__device__ __forceinline__ void split(float a, float b, uint32_t (&out)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i) {
        out[i] = from_pair(make_float2(a, b), bf16());
        if (i + 1 < N) {
            const float2 f = to_pair(out[i], bf16());
            a -= f.x, b -= f.y;
        }
    }
}

__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void ldsm(uint32_t (&r)[4], uint32_t at)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at));
}
__device__ __forceinline__ void ldsm_t(uint32_t (&r)[4], uint32_t at)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at));
}

// A tile of rows of W bf16 numbers in shared memory, its 16-byte units spread over the banks: unit u of row r lies at u ^ (r & 7), of the four of a
// row of 32 at u ^ (r / 2 & 3), so that eight rows' units of one number meet in no bank.
template <int W>
__device__ __forceinline__ uint32_t unit_at(uint32_t base, int row, int unit)
{
    return base + row * (W * 2) + ((unit ^ (W >= 64 ? row & 7 : (row >> 1) & 3)) << 4);
}

// Fragments of 16 x 16 blocks, by what lies along the tile's rows (m = lane / 8 picks one of four 8 x 8 blocks):
//   rows of the product's right operand along n, k inside them   -> two tiles of 8 columns: {b0, b1}, {b0, b1}
template <int W> __device__ __forceinline__ void right_nk(uint32_t (&r)[4], uint32_t base, int n0, int k0, int lane)
{
    ldsm(r, unit_at<W>(base, n0 + ((lane >> 4) << 3) + (lane & 7), (k0 >> 3) + ((lane >> 3) & 1)));
}
//   rows along k, n inside them
template <int W> __device__ __forceinline__ void right_kn(uint32_t (&r)[4], uint32_t base, int k0, int n0, int lane)
{
    ldsm_t(r, unit_at<W>(base, k0 + (lane & 15), (n0 >> 3) + (lane >> 4)));
}
//   the left operand, rows along m, k inside them
template <int W> __device__ __forceinline__ void left_mk(uint32_t (&r)[4], uint32_t base, int m0, int k0, int lane)
{
    ldsm(r, unit_at<W>(base, m0 + (lane & 15), (k0 >> 3) + (lane >> 4)));
}
//   rows along k, m inside them
template <int W> __device__ __forceinline__ void left_km(uint32_t (&r)[4], uint32_t base, int k0, int m0, int lane)
{
    ldsm_t(r, unit_at<W>(base, k0 + ((lane >> 4) << 3) + (lane & 7), (m0 >> 3) + ((lane >> 3) & 1)));
}

// The left operand of 16 columns from accumulators of two tiles of 8, as N parts.
template <int N>
__device__ __forceinline__ void left_of(uint32_t (&a)[N][4], const float (&c0)[4], const float (&c1)[4])
{
    uint32_t p[N];
    split<N>(c0[0], c0[1], p);
#pragma unroll
    for (int i = 0; i < N; ++i) a[i][0] = p[i];
    split<N>(c0[2], c0[3], p);
#pragma unroll
    for (int i = 0; i < N; ++i) a[i][1] = p[i];
    split<N>(c1[0], c1[1], p);
#pragma unroll
    for (int i = 0; i < N; ++i) a[i][2] = p[i];
    split<N>(c1[2], c1[3], p);
#pragma unroll
    for (int i = 0; i < N; ++i) a[i][3] = p[i];
}

// c0, c1 += the products of N parts of a left operand with part j of a right one, but for those that lie below the last part.
template <int N>
__device__ __forceinline__ void mma_parts(float (&c0)[4], float (&c1)[4], const uint32_t (&a)[N][4], const uint32_t (&b)[4], int j)
{
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (i + j < N) {
            mma(c0, a[i], b[0], b[1]);
            mma(c1, a[i], b[2], b[3]);
        }
}

// Where things lie in what the forward pass leaves (`states`) and in workspaces.  A "unit" is one piece of one head of one sequence, number
// (b * H + h) * pieces + c.  Sections in this order, sizes in bytes for each unit:
struct DeltaLayout {
    int B, L, Hk, H, K, V, KD, VP, pieces, in, sum;              // KD: K rounded up to 32, 64 or 128; VP: V to 16
    size_t units, keys;                                          // pieces of all value heads, of all key heads
    DeltaLayout(int B_, int L_, int Hk_, int H_, int K_, int V_, conv2d_operand_t type)
        : B(B_), L(L_), Hk(Hk_), H(H_), K(K_), V(V_), KD(K_ <= 32 ? 32 : K_ <= 64 ? 64 : 128), VP((V_ + 15) / 16 * 16), pieces((int)(((long long)L_ + kPiece - 1) / kPiece)),
          in(parts_in(type)), sum(parts_sum(type)), units((size_t)B_ * H_ * pieces), keys((size_t)B_ * Hk_ * pieces)
    {
    }
    size_t square() const { return (size_t)sum * kPiece * kPiece * 2; }              // t, or P
    size_t prepared_bytes() const { return units * (2 * square() + kFactors * kPiece * 4); }
    size_t state_plane() const { return (size_t)sum * VP * KD * 2; }                 // S or its gradient, [part][V][K]
    size_t update_plane() const { return (size_t)sum * VP * kPiece * 2; }            // E or dV, [part][V][token]
    size_t saved_bytes() const { return units * (state_plane() + update_plane()); }
    size_t key_plane() const { return (size_t)in * kPiece * KD * 2; }                // K, or Q, [part][token][K]
    size_t keys_bytes() const { return keys * 2 * key_plane(); }
};

// What the kernels read and write; the typed pointers of T are cast by them.
struct DeltaArgs {
    const void *q, *k, *v, *dout;
    const float *g, *beta, *state_in, *dstate_out;
    const int* lengths;
    void *o, *dq, *dk, *dv;
    float *state_out, *dg, *dbeta, *dstate_in;
    int B, L, Hk, H, K, V, share, pieces, VP;
    long long ldq, ldk, ldv, ldg, ldbeta, ldo, lddo, lddq, lddk, lddv, lddg, lddbeta;
    float scale;
    bf16 *t, *p;                  // [unit][part][64][64]
    float* factors;               // [unit][kFactors][64]
    bf16* planes;                 // [key unit][K, Q][part][64][KD]; NULL: the tensors themselves serve (bf16, K = KD, rows on 16 bytes)
    bf16 *states, *updates;       // saved by the forward pass: [unit][part][VP][KD], [unit][part][VP][64]; NULL: not wanted
    bf16 *dstates, *dupdates;     // the same of their gradients (dS after the piece, dV)
    float* dbeta_parts;           // [unit][VP / 16][64]
    float *dq_parts, *dk_parts;   // [B*L][H*K] fp32: gradients of heads that share a key, before they are summed
};

// Pieces in flight are counted in 31 bits.
inline bool delta_extents_ok(int B, int L, int H, int V)
{
    const long long pieces = ((long long)L + kPiece - 1) / kPiece;
    return (long long)B * H <= 0x7fffffffLL / pieces && (long long)B * H * pieces <= 0x7fffffffLL / ((V + 15) / 16);
}

conv2d_status_t launch_delta_fwd(DeltaArgs a, conv2d_operand_t type, void* states, void* workspace, cudaStream_t stream);
conv2d_status_t launch_delta_bwd(DeltaArgs a, conv2d_operand_t type, const void* states, void* workspace, cudaStream_t stream);
conv2d_status_t launch_delta_step(const DeltaArgs& a, conv2d_operand_t type, cudaStream_t stream);
// The first kernel of both passes: t, P and factors of every piece (backward: only the planes of keys and queries).
conv2d_status_t launch_delta_prepare(const DeltaArgs& a, conv2d_operand_t type, bool squares, cudaStream_t stream);
size_t delta_states_bytes(const DeltaLayout& l);
size_t delta_fwd_workspace_bytes(const DeltaLayout& l);
size_t delta_bwd_workspace_bytes(const DeltaLayout& l);
// Whether K and Q can be copied as they lie.
inline bool delta_direct(const DeltaArgs& a, conv2d_operand_t type, int KD)
{
    return type == CONV2D_OPERAND_BF16 && a.K == KD && rows_aligned(a.q, a.ldq, 2, 16) && rows_aligned(a.k, a.ldk, 2, 16);
}

#ifdef __CUDACC__
// Copies of K or Q (which = 0, 1) of a piece into a swizzled tile [part][64][KD], by `threads` threads of which this is number `id`; rows from `live` on
// are zeros.  Complete after the caller's wait for its copies.
template <int KD, int IN>
__device__ __forceinline__ void copy_keys(const DeltaArgs& a, uint32_t to, int which, int b, int hk, int piece, int live, int id, int threads)
{
    constexpr int UNITS = KD / 8;
    const char* from;
    long long row_bytes;
    if (a.planes) {
        from = reinterpret_cast<const char*>(a.planes) + ((((size_t)b * a.Hk + hk) * a.pieces + piece) * 2 + which) * ((size_t)IN * kPiece * KD * 2);
        row_bytes = KD * 2;
    } else {
        const long long ld = which ? a.ldq : a.ldk;
        from = static_cast<const char*>(which ? a.q : a.k) + (((long long)b * a.L + (long long)piece * kPiece) * ld + (long long)hk * KD) * 2;
        row_bytes = ld * 2;
    }
    for (int i = id; i < IN * kPiece * UNITS; i += threads) {
        const int row = i / UNITS, unit = i % UNITS, token = row % kPiece;
        const bool real = token < live;
        const char* src = real ? from + row * row_bytes + unit * 16 : from;
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(unit_at<KD>(to, row, unit)), "l"(src), "r"(real ? 16 : 0) : "memory");
    }
}
// Copies of `rows` dense rows of W bf16 numbers, those from `live` on as zeros.
template <int W>
__device__ __forceinline__ void copy_rows(const bf16* from, uint32_t to, int rows, int live, int id, int threads)
{
    constexpr int UNITS = W / 8;
    for (int i = id; i < rows * UNITS; i += threads) {
        const int row = i / UNITS, unit = i % UNITS;
        const bool real = row < live;
        const bf16* src = real ? from + (size_t)row * W + unit * 8 : from;
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(unit_at<W>(to, row, unit)), "l"(src), "r"(real ? 16 : 0) : "memory");
    }
}
// A tile of tokens x columns of a tensor, as it lies, rows `pitch` elements apart in shared memory; zeros beyond `live` tokens and `cols` columns.  By copies of
// 16 bytes where the rows allow it.
template <typename T>
__device__ __forceinline__ void copy_values(const T* from, long long ld, T* to, int pitch, int width, int live, int cols, bool wide, int id, int threads)
{
    constexpr int PER = 16 / (int)sizeof(T);
    if (wide) {                   // cols and width are multiples of PER then
        const int units = width / PER;
        for (int i = id; i < kPiece * units; i += threads) {
            const int row = i / units, c = i % units * PER;
            const bool real = row < live && c < cols;
            copy_async<16>(to + row * pitch + c, real ? from + row * ld + c : from, real);
        }
    } else {
        for (int i = id; i < kPiece * width; i += threads) {
            const int row = i / width, c = i % width;
            to[row * pitch + c] = row < live && c < cols ? from[row * ld + c] : from_float<T>(0.f);
        }
    }
}
#endif

}  // namespace conv2d_b200
