// Gated delta rule, backward.  With dS the gradient of the state behind a piece (D_ij = e^(G_i - G_j), E and t as in the forward pass):
//   dU = scale P^T dO + diag(e^(G_63 - G)) K dS,   W = dU - t^T (beta dU),   dV = beta W,   dbeta = rows of W . E,
//   dS <- e^(G_63) dS + Q^T (scale e^G dO) - K^T (e^G dV)
// walks the pieces from the last one back, 16 columns of V a warp, as the forward pass does; then every piece by itself:
//   p = D o (scale dO (beta E)^T), j <= i;   y = -D o (dV (beta E)^T), j < i;
//   dq = scale e^G dO S^T + p K;   dk = a + c,  a = y K - e^G dV S^T,  c = p^T Q + y^T K + e^(G_63 - G) beta E dS^T,
//   dG_i = q_i.dq_i + k_i.a_i - k_i.c_i,   dg_t = sum of dG_i, i >= t, + <S after the piece, dS>
// (every exponential of G stands beside a query or key: what scales them says what the exponent would have done).
#include "delta_walk.cuh"

namespace conv2d_b200 {
namespace {

template <typename T, int KD>
__global__ void __launch_bounds__((kComputing + kLoaders) * 32, 1) delta_bwd_walk_kernel(const DeltaArgs a, int warps, int across, bool wide_do, bool wide_dv)
{
    using W = Walk<T, KD>;
    constexpr int IN = Parts<T>::in, SUM = Parts<T>::sum, STAGES = W::stages;
    extern __shared__ __align__(1024) unsigned char raw[];
    ptx::grid_dep_wait();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, c = 2 * (lane & 3);
    const int v0 = (int)(blockIdx.x % across) * warps * 16, bh = blockIdx.x / across, h = bh % a.H, b = bh / a.H;
    const int len = sequence_length(a.lengths, b, a.L), pieces = (len + kPiece - 1) / kPiece;
    const bool computes = warp < warps;
    const int v = v0 + warp * 16;
    const T* values = static_cast<const T*>(a.dout);
    const int cols = min(warps * 16, a.V - v0);
    auto stage = [&](int i) { return Stage<T, KD>{raw + (STAGES == 2 ? (i & 1) * W::stage(warps) : 0), warps}; };
    auto load = [&](int i, int id, int threads) {
        load_piece<T, KD>(a, stage(i), values, a.lddo, wide_do, b, h, i, len - i * kPiece, v0, id, threads);
        copies_commit();
    };

    float S[KD / 8][4];                                        // dS^T
    const size_t state0 = ((size_t)b * a.H + h) * a.K * a.V;
#pragma unroll
    for (int n = 0; n < KD / 8; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int k = n * 8 + c + (e & 1), col = v + g + 8 * (e >> 1);
            S[n][e] = a.dstate_out && computes && k < a.K && col < a.V ? a.dstate_out[state0 + (size_t)k * a.V + col] : 0.f;
        }

    if (pieces > 0 && STAGES == 2) {
        load(pieces - 1, tid, blockDim.x);
        copies_wait<0>();
    }
    __syncthreads();
    for (int i = pieces - 1; i >= 0; --i) {
        if (STAGES == 1) {
            load(i, tid, blockDim.x);
            copies_wait<0>();
            __syncthreads();
        } else if (!computes) {
            if (i > 0) load(i - 1, tid - warps * 32, blockDim.x - warps * 32);
            copies_wait<0>();
        }
        if (computes && v < a.V) {
            const Stage<T, KD> s = stage(i);
            const float* f = s.factors();
            const size_t unit = ((size_t)b * a.H + h) * a.pieces + i;
            float U[8][4] = {}, X[8][4] = {};
            // dS^T K^T
#pragma unroll
            for (int n = 0; n < KD / 8; n += 2) {
                uint32_t x[SUM][4];
                left_of<SUM>(x, S[n], S[n + 1]);
                bf16* to = a.dstates + (unit * SUM * a.VP + v + g) * KD + n * 8 + c;
#pragma unroll
                for (int p = 0; p < SUM; ++p, to += (size_t)a.VP * KD) {
                    *reinterpret_cast<uint32_t*>(to) = x[p][0], *reinterpret_cast<uint32_t*>(to + 8 * KD) = x[p][1];
                    *reinterpret_cast<uint32_t*>(to + 8) = x[p][2], *reinterpret_cast<uint32_t*>(to + 8 * KD + 8) = x[p][3];
                }
#pragma unroll
                for (int m = 0; m < 8; m += 2) {
#pragma unroll
                    for (int p = 0; p < IN; ++p) {
                        uint32_t r[4];
                        right_nk<KD>(r, s.k() + p * (kPiece * KD * 2), m * 8, n * 8, lane);
                        mma_parts<SUM>(U[m], U[m + 1], x, r, p);
                    }
                }
            }
            // dO^T P
            const T* ds = s.values() + warp * 16 + g;
            auto dout = [&](int j, float (&d)[4]) {            // a tile of dO^T, 8 tokens from 8 j on
#pragma unroll
                for (int e = 0; e < 4; ++e) d[e] = to_float(ds[(j * 8 + c + (e & 1)) * s.pitch() + 8 * (e >> 1)]);
            };
#pragma unroll
            for (int j = 0; j < 8; j += 2) {
                uint32_t x[IN][4];
                float d0[4], d1[4];
                dout(j, d0), dout(j + 1, d1);
                left_of<IN>(x, d0, d1);
#pragma unroll
                for (int m = 0; m <= j; m += 2) {
#pragma unroll
                    for (int p = 0; p < SUM; ++p) {
                        uint32_t r[4];
                        right_kn<kPiece>(r, s.p() + p * (kPiece * kPiece * 2), j * 8, m * 8, lane);
#pragma unroll
                        for (int q = 0; q < IN; ++q)
                            if (p + q < SUM) mma(X[m], x[q], r[0], r[1]), mma(X[m + 1], x[q], r[2], r[3]);
                    }
                }
            }
#pragma unroll
            for (int m = 0; m < 8; ++m) {
                const float2 d = *reinterpret_cast<const float2*>(f + kPiece + m * 8 + c);
                const float2 be = *reinterpret_cast<const float2*>(f + 2 * kPiece + m * 8 + c);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    U[m][e] = fmaf(a.scale, X[m][e], (e & 1 ? d.y : d.x) * U[m][e]);
                    X[m][e] = -(e & 1 ? be.y : be.x) * U[m][e];
                }
            }
            // W = dU - t^T (beta dU): tokens j * 8 .. + 15 on those up to there
#pragma unroll
            for (int j = 0; j < 8; j += 2) {
                uint32_t x[SUM][4];
                left_of<SUM>(x, X[j], X[j + 1]);
#pragma unroll
                for (int m = 0; m <= j; m += 2) {
#pragma unroll
                    for (int p = 0; p < SUM; ++p) {
                        uint32_t r[4];
                        right_kn<kPiece>(r, s.t() + p * (kPiece * kPiece * 2), j * 8, m * 8, lane);
                        mma_parts<SUM>(U[m], U[m + 1], x, r, p);
                    }
                }
            }
            // dbeta: this warp's share of W . E; dV
            const bf16* es = a.updates + (unit * SUM * a.VP + v + g) * kPiece + c;
            bf16* dvs = a.dupdates + (unit * SUM * a.VP + v + g) * kPiece + c;
            float* parts = a.dbeta_parts + (unit * (a.VP / 16) + v / 16) * kPiece;
#pragma unroll
            for (int m = 0; m < 8; ++m) {
                float2 e0 = make_float2(0.f, 0.f), e1 = e0;
#pragma unroll
                for (int p = SUM - 1; p >= 0; --p) {
                    const bf16* at = es + (size_t)p * a.VP * kPiece + m * 8;
                    const float2 lo = to_pair(*reinterpret_cast<const uint32_t*>(at), bf16()), hi = to_pair(*reinterpret_cast<const uint32_t*>(at + 8 * kPiece), bf16());
                    e0.x += lo.x, e0.y += lo.y, e1.x += hi.x, e1.y += hi.y;
                }
                float2 sum = make_float2(fmaf(U[m][0], e0.x, U[m][2] * e1.x), fmaf(U[m][1], e0.y, U[m][3] * e1.y));
#pragma unroll
                for (int d = 4; d < 32; d *= 2) sum.x += __shfl_xor_sync(0xffffffffu, sum.x, d), sum.y += __shfl_xor_sync(0xffffffffu, sum.y, d);
                if (g == 0) *reinterpret_cast<float2*>(parts + m * 8 + c) = sum;
                const float2 be = *reinterpret_cast<const float2*>(f + 2 * kPiece + m * 8 + c);
                U[m][0] *= be.x, U[m][1] *= be.y, U[m][2] *= be.x, U[m][3] *= be.y;
                uint32_t x[SUM], y[SUM];
                split<SUM>(U[m][0], U[m][1], x);
                split<SUM>(U[m][2], U[m][3], y);
#pragma unroll
                for (int p = 0; p < SUM; ++p) {
                    bf16* to = dvs + (size_t)p * a.VP * kPiece + m * 8;
                    *reinterpret_cast<uint32_t*>(to) = x[p], *reinterpret_cast<uint32_t*>(to + 8 * kPiece) = y[p];
                }
            }
            T* mine = reinterpret_cast<T*>(raw + STAGES * W::stage(warps)) + warp * kPiece * (16 + W::kPad);
            store_columns(U, mine, static_cast<T*>(a.dv) + ((long long)b * a.L + (long long)i * kPiece) * a.lddv + (long long)h * a.V + v, a.lddv, len - i * kPiece,
                          a.V - v, wide_dv, lane);
            // dS <- e^G_63 dS + (scale e^G dO)^T Q - (e^G dV)^T K
            const float whole = f[kPiece - 1];
#pragma unroll
            for (int n = 0; n < KD / 8; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) S[n][e] *= whole;
#pragma unroll
            for (int j = 0; j < 8; j += 2) {
                uint32_t x[SUM][4], y[SUM][4];
                float d0[4], d1[4];
                dout(j, d0), dout(j + 1, d1);
                const float2 g0 = *reinterpret_cast<const float2*>(f + j * 8 + c), g1 = *reinterpret_cast<const float2*>(f + j * 8 + 8 + c);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float x0 = e & 1 ? g0.y : g0.x, x1 = e & 1 ? g1.y : g1.x;
                    d0[e] *= a.scale * x0, d1[e] *= a.scale * x1;
                    U[j][e] *= -x0, U[j + 1][e] *= -x1;
                }
                left_of<SUM>(x, d0, d1);
                left_of<SUM>(y, U[j], U[j + 1]);
#pragma unroll
                for (int n = 0; n < KD / 8; n += 2) {
#pragma unroll
                    for (int p = 0; p < IN; ++p) {
                        uint32_t r[4];
                        right_kn<KD>(r, s.q() + p * (kPiece * KD * 2), j * 8, n * 8, lane);
                        mma_parts<SUM>(S[n], S[n + 1], x, r, p);
                        right_kn<KD>(r, s.k() + p * (kPiece * KD * 2), j * 8, n * 8, lane);
                        mma_parts<SUM>(S[n], S[n + 1], y, r, p);
                    }
                }
            }
        }
        __syncthreads();
    }
    if (a.dstate_in && computes) {
#pragma unroll
        for (int n = 0; n < KD / 8; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int k = n * 8 + c + (e & 1), col = v + g + 8 * (e >> 1);
                if (k < a.K && col < a.V) a.dstate_in[state0 + (size_t)k * a.V + col] = S[n][e];
            }
    }
    zero_rows(static_cast<T*>(a.dv) + (long long)b * a.L * a.lddv + (long long)h * a.V + v0, a.lddv, len, a.L, cols, tid, blockDim.x);
}

// One block for one piece of one value head.  Four warps by 16 tokens times two by halves of K; products over V in blocks of 64 columns.
template <typename T, int KD>
struct Piecewise {
    static constexpr int IN = Parts<T>::in, SUM = Parts<T>::sum, BLOCK = 64;
    static constexpr size_t dout = (size_t)IN * kPiece * BLOCK * 2, update = (size_t)SUM * BLOCK * kPiece * 2, state = (size_t)SUM * BLOCK * KD * 2;
    static constexpr size_t over_v = dout + 2 * update + 2 * state;
    static constexpr size_t keys = (size_t)IN * kPiece * KD * 2, square = (size_t)SUM * kPiece * kPiece * 2;
    static constexpr size_t over_tokens = 2 * keys + 2 * square;
    static constexpr size_t smem = over_v > over_tokens ? over_v : over_tokens;
};

template <typename T, int KD>
__global__ void __launch_bounds__(256) delta_bwd_pieces_kernel(const DeltaArgs a)
{
    using S = Piecewise<T, KD>;
    constexpr int IN = S::IN, SUM = S::SUM, BLOCK = S::BLOCK, HALF = KD / 2, NT = HALF / 8;
    extern __shared__ __align__(1024) unsigned char raw[];
    __shared__ float f[kFactors * kPiece], dots[2][kPiece], sums[8];
    ptx::grid_dep_wait();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, c = 2 * (lane & 3);
    const int piece = blockIdx.x % a.pieces, bh = blockIdx.x / a.pieces, h = bh % a.H, b = bh / a.H, hk = h / a.share;
    const int live = min(sequence_length(a.lengths, b, a.L) - piece * kPiece, kPiece), there = min(a.L - piece * kPiece, kPiece);
    const long long row0 = (long long)b * a.L + (long long)piece * kPiece;
    const bool shared_key = a.dq_parts != nullptr;
    T *dq = static_cast<T*>(a.dq) + row0 * a.lddq + (long long)hk * a.K, *dk = static_cast<T*>(a.dk) + row0 * a.lddk + (long long)hk * a.K;
    const long long part0 = (row0 * a.H + h) * a.K;
    auto put = [&](int row, int col, float q, float k) {
        if (shared_key) {
            const long long at = part0 + (long long)row * a.H * a.K + col;
            a.dq_parts[at] = q, a.dk_parts[at] = k;
        } else {
            dq[row * a.lddq + col] = from_float<T>(q), dk[row * a.lddk + col] = from_float<T>(k);
        }
    };
    // padding
    for (int i = tid; i < (there - max(live, 0)) * a.K; i += 256) put(max(live, 0) + i / a.K, i % a.K, 0.f, 0.f);
    for (int i = max(live, 0) + tid; i < there; i += 256) a.dg[(row0 + i) * a.lddg + h] = 0.f, a.dbeta[(row0 + i) * a.lddbeta + h] = 0.f;
    if (live <= 0) return;

    const size_t unit = (size_t)bh * a.pieces + piece;
    for (int i = tid; i < kFactors * kPiece; i += 256) f[i] = a.factors[unit * (kFactors * kPiece) + i];
    const uint32_t base = ptx::smem_u32(raw);
    const uint32_t s_do = base, s_dv = s_do + (uint32_t)S::dout, s_e = s_dv + (uint32_t)S::update, s_s = s_e + (uint32_t)S::update, s_ds = s_s + (uint32_t)S::state;
    const int m0 = (warp & 3) * 16, side = warp >> 2;
    float Q[NT][4] = {}, A[NT][4] = {}, C[NT][4] = {}, P[4][4] = {}, Y[4][4] = {};
    float inner = 0.f;                                         // <S, dS>
    const T* dout = static_cast<const T*>(a.dout) + row0 * a.lddo + (long long)h * a.V;
    for (int v0 = 0; v0 < a.V; v0 += BLOCK) {
        const int rows = min(a.VP - v0, BLOCK);
        if (v0) __syncthreads();
        for (int p = 0; p < SUM; ++p) {
            const size_t at = (unit * SUM + p) * a.VP + v0;
            copy_rows<kPiece>(a.dupdates + at * kPiece, s_dv + p * (BLOCK * kPiece * 2), BLOCK, rows, tid, 256);
            copy_rows<kPiece>(a.updates + at * kPiece, s_e + p * (BLOCK * kPiece * 2), BLOCK, rows, tid, 256);
            copy_rows<KD>(a.states + at * KD, s_s + p * (BLOCK * KD * 2), BLOCK, rows, tid, 256);
            copy_rows<KD>(a.dstates + at * KD, s_ds + p * (BLOCK * KD * 2), BLOCK, rows, tid, 256);
        }
        copies_commit();
        for (int i = tid; i < kPiece * (BLOCK / 2); i += 256) {
            const int row = i / (BLOCK / 2), col = i % (BLOCK / 2) * 2;
            float x[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) x[j] = row < live && v0 + col + j < a.V ? to_float(dout[row * a.lddo + v0 + col + j]) : 0.f;
            uint32_t w[IN];
            split<IN>(x[0], x[1], w);
#pragma unroll
            for (int p = 0; p < IN; ++p)
                *reinterpret_cast<uint32_t*>(raw + (unit_at<BLOCK>(s_do + p * (kPiece * BLOCK * 2), row, col >> 3) - base) + (col & 7) * 2) = w[p];
        }
        copies_wait<0>();
        __syncthreads();
        for (int i = tid; i < BLOCK * KD / 8; i += 256) {      // (a unit of S times the same of dS)
            float x[8] = {}, y[8] = {};
#pragma unroll
            for (int p = SUM - 1; p >= 0; --p) {
                const uint32_t at = unit_at<KD>((uint32_t)(p * (BLOCK * KD * 2)), i / (KD / 8), i % (KD / 8));
                float w[8];
                unpack(*reinterpret_cast<const Pack<bf16, 8>*>(raw + (s_s - base) + at), w);
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] += w[e];
                unpack(*reinterpret_cast<const Pack<bf16, 8>*>(raw + (s_ds - base) + at), w);
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] += w[e];
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) inner = fmaf(x[e], y[e], inner);
        }
#pragma unroll
        for (int k0 = 0; k0 < BLOCK; k0 += 16) {
            if (k0 >= rows) break;
            uint32_t xo[IN][4], xv[SUM][4], xe[SUM][4];
#pragma unroll
            for (int p = 0; p < IN; ++p) left_mk<BLOCK>(xo[p], s_do + p * (kPiece * BLOCK * 2), m0, k0, lane);
#pragma unroll
            for (int p = 0; p < SUM; ++p) {
                left_km<kPiece>(xv[p], s_dv + p * (BLOCK * kPiece * 2), k0, m0, lane);
                left_km<kPiece>(xe[p], s_e + p * (BLOCK * kPiece * 2), k0, m0, lane);
            }
#pragma unroll
            for (int n = 0; n < 4; n += 2) {                   // dO E^T, dV E^T: this warp's 32 of the columns
                const int n0 = side * 32 + n * 8;
                if (n0 > m0) continue;
#pragma unroll
                for (int p = 0; p < SUM; ++p) {
                    uint32_t r[4];
                    right_kn<kPiece>(r, s_e + p * (BLOCK * kPiece * 2), k0, n0, lane);
#pragma unroll
                    for (int q = 0; q < IN; ++q)
                        if (p + q < SUM) mma(P[n], xo[q], r[0], r[1]), mma(P[n + 1], xo[q], r[2], r[3]);
                    mma_parts<SUM>(Y[n], Y[n + 1], xv, r, p);
                }
            }
#pragma unroll
            for (int n = 0; n < NT; n += 2) {
                const int n0 = side * HALF + n * 8;
#pragma unroll
                for (int p = 0; p < SUM; ++p) {
                    uint32_t r[4];
                    right_kn<KD>(r, s_s + p * (BLOCK * KD * 2), k0, n0, lane);
#pragma unroll
                    for (int q = 0; q < IN; ++q)
                        if (p + q < SUM) mma(Q[n], xo[q], r[0], r[1]), mma(Q[n + 1], xo[q], r[2], r[3]);
                    mma_parts<SUM>(A[n], A[n + 1], xv, r, p);
                    right_kn<KD>(r, s_ds + p * (BLOCK * KD * 2), k0, n0, lane);
                    mma_parts<SUM>(C[n], C[n + 1], xe, r, p);
                }
            }
        }
    }
    __syncthreads();                                           // (the factors too; what lies over V is not read any more)
    const uint32_t ks = base, qs = ks + (uint32_t)S::keys, s_p = qs + (uint32_t)S::keys, s_y = s_p + (uint32_t)S::square;
    copy_keys<KD, IN>(a, ks, 0, b, hk, piece, live, tid, 256);
    copy_keys<KD, IN>(a, qs, 1, b, hk, piece, live, tid, 256);
    copies_commit();
    const float *eg = f, *ed = f + kPiece, *be = f + 2 * kPiece, *high = f + 3 * kPiece, *low = f + 4 * kPiece;
#pragma unroll
    for (int n = 0; n < 4; ++n) {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int i = m0 + g + 8 * half, j = side * 32 + n * 8 + c;
            float pv[2], yv[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const float d = ex2(((high[i] - high[j + e]) + (low[i] - low[j + e])) * kLog2e) * be[j + e];
                pv[e] = j + e <= i ? a.scale * d * P[n][2 * half + e] : 0.f;
                yv[e] = j + e < i ? -d * Y[n][2 * half + e] : 0.f;
            }
            uint32_t wp[SUM], wy[SUM];
            split<SUM>(pv[0], pv[1], wp);
            split<SUM>(yv[0], yv[1], wy);
            const uint32_t at = unit_at<kPiece>(0, i, j >> 3) + (j & 7) * 2;
#pragma unroll
            for (int p = 0; p < SUM; ++p) {
                *reinterpret_cast<uint32_t*>(raw + (s_p - base) + p * (kPiece * kPiece * 2) + at) = wp[p];
                *reinterpret_cast<uint32_t*>(raw + (s_y - base) + p * (kPiece * kPiece * 2) + at) = wy[p];
            }
        }
    }
    const float g0 = eg[m0 + g], g1 = eg[m0 + g + 8], d0 = ed[m0 + g] * be[m0 + g], d1 = ed[m0 + g + 8] * be[m0 + g + 8];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float x = e < 2 ? g0 : g1;
            Q[n][e] *= a.scale * x, A[n][e] *= -x, C[n][e] *= e < 2 ? d0 : d1;
        }
    }
    copies_wait<0>();
    __syncthreads();
    // a number of K or Q, from its parts
    auto number = [&](uint32_t tile, int row, int col) {
        float2 x = make_float2(0.f, 0.f);
#pragma unroll
        for (int p = IN - 1; p >= 0; --p) {
            const float2 y = to_pair(*reinterpret_cast<const uint32_t*>(raw + (unit_at<KD>(tile + p * (kPiece * KD * 2), row, col >> 3) - base) + (col & 7) * 2), bf16());
            x.x += y.x, x.y += y.y;
        }
        return x;
    };
    // <S after, dS> = e^G_63 <S, dS> + sum over tokens of k . (e^(G_63 - G) beta E dS^T)
    float after = eg[kPiece - 1] * inner;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int col = side * HALF + n * 8 + c;
        const float2 k0 = number(ks, m0 + g, col), k1 = number(ks, m0 + g + 8, col);
        after = fmaf(k0.x, C[n][0], fmaf(k0.y, C[n][1], fmaf(k1.x, C[n][2], fmaf(k1.y, C[n][3], after))));
    }
#pragma unroll
    for (int d = 1; d < 32; d *= 2) after += __shfl_xor_sync(0xffffffffu, after, d);
    if (lane == 0) sums[warp] = after;
    // products over tokens
#pragma unroll
    for (int k0 = 0; k0 < kPiece; k0 += 16) {
        uint32_t r[4], x[SUM][4], y[SUM][4];
        if (k0 <= m0) {                                        // p K, y K: tokens up to these
#pragma unroll
            for (int p = 0; p < SUM; ++p) {
                left_mk<kPiece>(x[p], s_p + p * (kPiece * kPiece * 2), m0, k0, lane);
                left_mk<kPiece>(y[p], s_y + p * (kPiece * kPiece * 2), m0, k0, lane);
            }
#pragma unroll
            for (int n = 0; n < NT; n += 2) {
#pragma unroll
                for (int p = 0; p < IN; ++p) {
                    right_kn<KD>(r, ks + p * (kPiece * KD * 2), k0, side * HALF + n * 8, lane);
                    mma_parts<SUM>(Q[n], Q[n + 1], x, r, p);
                    mma_parts<SUM>(A[n], A[n + 1], y, r, p);
                }
            }
        }
        if (k0 >= m0) {                                        // p^T Q, y^T K: tokens from these on
#pragma unroll
            for (int p = 0; p < SUM; ++p) {
                left_km<kPiece>(x[p], s_p + p * (kPiece * kPiece * 2), k0, m0, lane);
                left_km<kPiece>(y[p], s_y + p * (kPiece * kPiece * 2), k0, m0, lane);
            }
#pragma unroll
            for (int n = 0; n < NT; n += 2) {
#pragma unroll
                for (int p = 0; p < IN; ++p) {
                    right_kn<KD>(r, qs + p * (kPiece * KD * 2), k0, side * HALF + n * 8, lane);
                    mma_parts<SUM>(C[n], C[n + 1], x, r, p);
                    right_kn<KD>(r, ks + p * (kPiece * KD * 2), k0, side * HALF + n * 8, lane);
                    mma_parts<SUM>(C[n], C[n + 1], y, r, p);
                }
            }
        }
    }
    float dot[2] = {0.f, 0.f};
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int col = side * HALF + n * 8 + c;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int row = m0 + g + 8 * half;
            const float2 k = number(ks, row, col), q = number(qs, row, col);
            dot[half] = fmaf(q.x, Q[n][2 * half], fmaf(q.y, Q[n][2 * half + 1], dot[half]));
            dot[half] = fmaf(k.x, A[n][2 * half] - C[n][2 * half], fmaf(k.y, A[n][2 * half + 1] - C[n][2 * half + 1], dot[half]));
#pragma unroll
            for (int e = 0; e < 2; ++e)
                if (row < live && col + e < a.K) put(row, col + e, Q[n][2 * half + e], A[n][2 * half + e] + C[n][2 * half + e]);
        }
    }
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        dot[half] += __shfl_xor_sync(0xffffffffu, dot[half], 1);
        dot[half] += __shfl_xor_sync(0xffffffffu, dot[half], 2);
        if (c == 0) dots[side][m0 + g + 8 * half] = dot[half];
    }
    __syncthreads();
    if (warp == 0) {                                           // sums from the last token back, two tokens a lane
        float last = 0.f;
#pragma unroll
        for (int w = 0; w < 8; ++w) last += sums[w];
        const float x1 = dots[0][63 - 2 * lane] + dots[1][63 - 2 * lane], x0 = dots[0][62 - 2 * lane] + dots[1][62 - 2 * lane];
        float s = x0 + x1;
        for (int d = 1; d < 32; d *= 2) {
            const float y = __shfl_up_sync(0xffffffffu, s, d);
            if (lane >= d) s += y;
        }
        const int row = 62 - 2 * lane;
        if (row < live) a.dg[(row0 + row) * a.lddg + h] = s + last;
        if (row + 1 < live) a.dg[(row0 + row + 1) * a.lddg + h] = (s - x0) + last;
    } else if (warp < 4 && warp >= 2) {
        const int row = (warp - 2) * 32 + lane, tiles = a.VP / 16;
        const float* from = a.dbeta_parts + unit * tiles * kPiece + row;
        float s = 0.f;
        for (int i = 0; i < tiles; ++i) s += from[i * kPiece];
        if (row < live) a.dbeta[(row0 + row) * a.lddbeta + h] = s;
    }
}

// Gradients of a key head from those of its value heads.
template <typename T>
__global__ void __launch_bounds__(256) delta_bwd_shared_kernel(const DeltaArgs a)
{
    ptx::grid_dep_wait();
    const long long n = (long long)a.B * a.L * a.Hk * a.K;
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n; i += (long long)gridDim.x * 256) {
        const int col = (int)(i % a.K), hk = (int)(i / a.K % a.Hk);
        const long long row = i / ((long long)a.K * a.Hk), at = (row * a.H + (long long)hk * a.share) * a.K + col;
        float q = 0.f, k = 0.f;
        for (int r = 0; r < a.share; ++r) q += a.dq_parts[at + (long long)r * a.K], k += a.dk_parts[at + (long long)r * a.K];
        static_cast<T*>(a.dq)[row * a.lddq + (long long)hk * a.K + col] = from_float<T>(q);
        static_cast<T*>(a.dk)[row * a.lddk + (long long)hk * a.K + col] = from_float<T>(k);
    }
}

template <typename T, int KD>
conv2d_status_t backward(const DeltaArgs& a, cudaStream_t stream)
{
    using W = Walk<T, KD>;
    static SmemLimit limit, limit_pieces;
    const int warps = delta_warps(a), across = (int)ceil_div_u(a.VP / 16, warps);
    const size_t smem = W::smem(warps);
    if (raise_smem_limit((const void*)delta_bwd_walk_kernel<T, KD>, smem, limit) != cudaSuccess) return CONV2D_ERR_CUDA;
    if (raise_smem_limit((const void*)delta_bwd_pieces_kernel<T, KD>, Piecewise<T, KD>::smem, limit_pieces) != cudaSuccess) return CONV2D_ERR_CUDA;
    const int per = 16 / (int)sizeof(T);
    const bool wide_do = a.V % per == 0 && rows_aligned(a.dout, a.lddo, sizeof(T), 16), wide_dv = a.V % per == 0 && rows_aligned(a.dv, a.lddv, sizeof(T), 16);
    if (launch_pdl(delta_bwd_walk_kernel<T, KD>, dim3((unsigned)(a.B * a.H) * across), dim3((warps + kLoaders) * 32), smem, stream, a, warps, across, wide_do,
                   wide_dv) != cudaSuccess)
        return CONV2D_ERR_CUDA;
    count_launch();
    if (launch_pdl(delta_bwd_pieces_kernel<T, KD>, dim3((unsigned)(a.B * a.H) * (unsigned)a.pieces), dim3(256), Piecewise<T, KD>::smem, stream, a) != cudaSuccess)
        return CONV2D_ERR_CUDA;
    count_launch();
    if (a.share > 1) {
        const long long blocks = ((long long)a.B * a.L * a.Hk * a.K + 255) / 256, most = 16LL * sm_count();
        if (launch_pdl(delta_bwd_shared_kernel<T>, dim3((unsigned)(blocks < most ? blocks : most)), dim3(256), 0, stream, a) != cudaSuccess) return CONV2D_ERR_CUDA;
        count_launch();
    }
    return CONV2D_OK;
}

template <typename T>
conv2d_status_t backward_typed(const DeltaArgs& a, cudaStream_t stream)
{
    if (a.K <= 32) return backward<T, 32>(a, stream);
    if (a.K <= 64) return backward<T, 64>(a, stream);
    return backward<T, 128>(a, stream);
}

size_t up16(size_t n) { return (n + 15) / 16 * 16; }
size_t dbeta_bytes(const DeltaLayout& l) { return l.units * (l.VP / 16) * kPiece * 4; }
size_t shared_bytes(const DeltaLayout& l) { return l.H > l.Hk ? up16((size_t)l.B * l.L * l.H * l.K * 4) : 0; }

}  // namespace

size_t delta_bwd_workspace_bytes(const DeltaLayout& l) { return l.saved_bytes() + l.keys_bytes() + dbeta_bytes(l) + 2 * shared_bytes(l); }

conv2d_status_t launch_delta_bwd(DeltaArgs a, conv2d_operand_t type, const void* states, void* workspace, cudaStream_t stream)
{
    const DeltaLayout l(a.B, a.L, a.Hk, a.H, a.K, a.V, type);
    a.share = a.H / a.Hk, a.pieces = l.pieces, a.VP = l.VP;
    unsigned char* kept = const_cast<unsigned char*>(static_cast<const unsigned char*>(states));      // (only read)
    a.t = reinterpret_cast<bf16*>(kept), a.p = reinterpret_cast<bf16*>(kept + l.units * l.square());
    a.factors = reinterpret_cast<float*>(kept + l.units * 2 * l.square());
    a.states = reinterpret_cast<bf16*>(kept + l.prepared_bytes());
    a.updates = reinterpret_cast<bf16*>(kept + l.prepared_bytes() + l.units * l.state_plane());
    unsigned char* at = static_cast<unsigned char*>(workspace);
    a.dstates = reinterpret_cast<bf16*>(at), at += l.units * l.state_plane();
    a.dupdates = reinterpret_cast<bf16*>(at), at += l.units * l.update_plane();
    const bool direct = delta_direct(a, type, l.KD);
    if (!direct) a.planes = reinterpret_cast<bf16*>(at);
    at += l.keys_bytes();
    a.dbeta_parts = reinterpret_cast<float*>(at), at += dbeta_bytes(l);
    if (a.share > 1) a.dq_parts = reinterpret_cast<float*>(at), a.dk_parts = reinterpret_cast<float*>(at + shared_bytes(l));
    if (!direct) {
        const conv2d_status_t st = launch_delta_prepare(a, type, false, stream);
        if (st != CONV2D_OK) return st;
    }
    if (type == CONV2D_OPERAND_BF16) return backward_typed<bf16>(a, stream);
    if (type == CONV2D_OPERAND_FP16) return backward_typed<fp16>(a, stream);
    return backward_typed<float>(a, stream);
}

}  // namespace conv2d_b200
