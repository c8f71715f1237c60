// What the kernels of the gated delta rule share: pieces of 64 tokens, numbers as sums of bf16 parts, matrix products of those, layouts.
//
// A head's state S (K x V) runs through pieces of 64 tokens.  Within one, with G_i the sum of the log decays up to token i, S the state before it,
//   A_ij = e^(G_i - G_j) k_i.k_j (j < i),   P_ij = e^(G_i - G_j) q_i.k_j (j <= i),   t = (1 + A diag(beta))^-1 A   (strictly lower),   P' = P (1 - diag(beta) t),
//   R = V - diag(e^G) K S,   E = R - t diag(beta) R,   O = scale (diag(e^G) Q S + P' diag(beta) R),
//   S <- e^(G_63) S + K^T diag(e^(G_63 - G) beta) E.
// t and P' hold neither the identity nor the betas to their right: both stay in fp32, and the backward pass uses the same two (beta may be zero).
// A piece is three products of 128 rows:  [K; Q] S,  [-t; P'] (beta R),  K^T (e^(G_63 - G) beta E).
#pragma once

#include "masked_load.cuh"
#include "recurrent_b200.h"

namespace conv2d_b200 {

constexpr int kPiece = 64;
constexpr int kFactors = 5;                                     // of a piece: e^G, e^(G_63 - G), beta, G in two floats
constexpr int kMost = 128;                                      // numbers of a key

// Numbers of bf16 that hold a tensor's element, and kSum of those that hold sums and states as
// operands: all of their 24 bits.  Two would be 16: half the products of two sums, but results in fp32 (states, gradients of gates) were off by 3e-6 to
// 9e-6 then, by about 1e-6 so.
template <typename T> struct Parts;
template <> struct Parts<bf16> { static constexpr int in = 1; };
template <> struct Parts<fp16> { static constexpr int in = 2; };
template <> struct Parts<float> { static constexpr int in = 3; };
constexpr int kSum = 3;
inline int parts_in(conv2d_operand_t t) { return t == CONV2D_OPERAND_BF16 ? 1 : t == CONV2D_OPERAND_FP16 ? 2 : 3; }

// a, b as N parts each, the two of a part side by side.  Rounded, not cut: the parts that are left out of products are smaller by half so, twice over, and of
// either sign.
template <int N>
__device__ __forceinline__ void split(float a, float b, uint32_t (&out)[N])
{
    float2 v = make_float2(a, b);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        out[i] = from_pair(v, bf16());
        if (i + 1 < N) v = __ffma2_rn(to_pair(out[i], bf16()), both(-1.f), v);
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

// A tile of rows of W = 64 or 32 bf16 numbers, its 16-byte units spread over the banks as the tensor core's 128- and 64-byte swizzles have them: unit u of row r
// lies at u ^ (r & 7), of the four of a row of 32 at u ^ (r / 2 & 3), so that eight rows' units of one number meet in no bank.
template <int W>
__device__ __forceinline__ uint32_t unit_at(uint32_t base, int row, int unit)
{
    return base + row * (W * 2) + ((unit ^ (W >= 64 ? row & 7 : (row >> 1) & 3)) << 4);
}

// N elements of a row of a tensor as they lie, zeros beyond `there`: to be converted when they are used, since a conversion waits for the load.  WIDE: by accesses of
// 16 bytes, `there` a multiple of those; a template's matter, since a branch between loads waits for them, too.
template <typename T, int N>
struct Row {
    static constexpr int PER = 16 / (int)sizeof(T) < N ? 16 / (int)sizeof(T) : N;
    Pack<T, PER> p[N / PER];
    template <bool WIDE>
    __device__ __forceinline__ void load(const T* from, int there)
    {
        if (WIDE) {
#pragma unroll
            for (int i = 0; i < N / PER; ++i) p[i] = load_masked<T, PER>(from + i * PER, i * PER < there);
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) p[i / PER].e[i % PER] = load_masked<T, 1>(from + i, i < there).e[0];
        }
    }
    __device__ __forceinline__ void get(float (&f)[N]) const
    {
#pragma unroll
        for (int i = 0; i < N / PER; ++i) {
            float x[PER];
            unpack(p[i], x);
#pragma unroll
            for (int j = 0; j < PER; ++j) f[i * PER + j] = x[j];
        }
    }
};

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

// c0, c1 += the products of N parts of a left operand with part j of a right one, but for those that lie below the last part of a sum.
template <int N>
__device__ __forceinline__ void mma_parts(float (&c0)[4], float (&c1)[4], const uint32_t (&a)[N][4], const uint32_t (&b)[4], int j)
{
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (i + j < kSum) {
            mma(c0, a[i], b[0], b[1]);
            mma(c1, a[i], b[2], b[3]);
        }
}

// Where things lie in what the forward pass leaves (`states`) and in workspaces.  A "unit" is one piece of one head of one sequence, number
// (b * H + h) * pieces + c; a "key unit" the same of a key head.  Sections in this order, sizes in bytes for each unit:
constexpr size_t kSquares = (size_t)kSum * 2 * kPiece * kPiece * 2;      // [-t^T | P'^T], [part][two][64][64], units of 16 bytes swizzled as unit_at does;
constexpr size_t kPrepared = kSquares + kFactors * kPiece * 4;           // and the factors behind them
struct DeltaLayout {
    int B, L, Hk, H, K, V, KD, VP, pieces, in;                   // KD: K rounded up to 64 or 128; VP: V to 16
    size_t units, keys;                                          // pieces of all value heads, of all key heads
    DeltaLayout(int B_, int L_, int Hk_, int H_, int K_, int V_, conv2d_operand_t type)
        : B(B_), L(L_), Hk(Hk_), H(H_), K(K_), V(V_), KD(K_ <= 64 ? 64 : 128), VP((V_ + 15) / 16 * 16), pieces((int)(((long long)L_ + kPiece - 1) / kPiece)),
          in(parts_in(type)), units((size_t)B_ * H_ * pieces), keys((size_t)B_ * Hk_ * pieces)
    {
    }
    size_t prepared_bytes() const { return units * kPrepared; }
    size_t state() const { return (size_t)KD * VP * 4; }                             // S or its gradient, [V/4][K][4]
    size_t update() const { return (size_t)kPiece * VP * 4; }                        // E or dV, [V/4][token][4]
    size_t saved_bytes() const { return units * (state() + update()); }
    size_t key_tile() const { return (size_t)in * 2 * kPiece * KD * 2; }             // [K; Q], [part][64 numbers][128][64], swizzled likewise
    size_t keys_bytes() const { return keys * key_tile(); }
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
    unsigned char *prepared, *keys;   // of units, and tiles of key units
    float *states, *updates;      // saved by the forward pass: [unit][VP/4][KD][4], [unit][VP/4][64][4]; NULL: not wanted
    float *dstates, *dupdates;    // the same of their gradients (dS after the piece, dV)
    float* dbeta_parts;           // [unit][VP / 16][64]
    float *dq_parts, *dk_parts;   // [B*L][H*K] fp32: gradients of heads that share a key, before they are summed
    unsigned *timeout, max_polls; // raised when a wait within a kernel runs out
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
// The first kernel of both passes: tiles and factors of every piece (backward: only the tiles of keys and queries).
conv2d_status_t launch_delta_prepare(const DeltaArgs& a, conv2d_operand_t type, bool squares, cudaStream_t stream);
size_t delta_states_bytes(const DeltaLayout& l);
size_t delta_fwd_workspace_bytes(const DeltaLayout& l);
size_t delta_bwd_workspace_bytes(const DeltaLayout& l);
}  // namespace conv2d_b200
