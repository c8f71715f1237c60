// Gated delta rule, forward: a block walks the pieces of one head of one sequence for up to 64 columns of V.
#include "delta_walk.cuh"

namespace conv2d_b200 {
namespace {

template <typename T, int KD>
__global__ void __launch_bounds__((kComputing + kLoaders) * 32, 1) delta_fwd_kernel(const DeltaArgs a, int warps, int across, bool wide_v, bool wide_o)
{
    using W = Walk<T, KD>;
    constexpr int IN = Parts<T>::in, SUM = Parts<T>::sum, OUT = Parts<T>::out, STAGES = W::stages;
    extern __shared__ __align__(1024) unsigned char raw[];
    ptx::grid_dep_wait();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, c = 2 * (lane & 3);
    const int v0 = (int)(blockIdx.x % across) * warps * 16, bh = blockIdx.x / across, h = bh % a.H, b = bh / a.H;
    const int len = sequence_length(a.lengths, b, a.L), pieces = (len + kPiece - 1) / kPiece;
    const bool computes = warp < warps;
    const int v = v0 + warp * 16;                              // this warp's first column
    const T* values = static_cast<const T*>(a.v);
    const int cols = min(warps * 16, a.V - v0);
    auto stage = [&](int i) { return Stage<T, KD>{raw + (STAGES == 2 ? (i & 1) * W::stage(warps) : 0), warps}; };
    auto load = [&](int i, int id, int threads) {
        load_piece<T, KD>(a, stage(i), values, a.ldv, wide_v, b, h, i, len - i * kPiece, v0, id, threads);
        copies_commit();
    };

    float S[KD / 8][4];                                        // S^T: rows g and g + 8 of the warp's columns, K in pairs
    const size_t state0 = ((size_t)b * a.H + h) * a.K * a.V;
#pragma unroll
    for (int n = 0; n < KD / 8; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int k = n * 8 + c + (e & 1), col = v + g + 8 * (e >> 1);
            S[n][e] = a.state_in && computes && k < a.K && col < a.V ? a.state_in[state0 + (size_t)k * a.V + col] : 0.f;
        }

    if (pieces > 0 && STAGES == 2) {
        load(0, tid, blockDim.x);
        copies_wait<0>();
    }
    __syncthreads();
    for (int i = 0; i < pieces; ++i) {
        if (STAGES == 1) {
            load(i, tid, blockDim.x);
            copies_wait<0>();
            __syncthreads();
        } else if (!computes) {
            if (i + 1 < pieces) load(i + 1, tid - warps * 32, blockDim.x - warps * 32);
            copies_wait<0>();
        }
        if (computes && v < a.V) {
            const Stage<T, KD> s = stage(i);
            const float* f = s.factors();
            const size_t unit = ((size_t)b * a.H + h) * a.pieces + i;
            float R[8][4] = {}, O[8][4] = {};
            // S^T K^T and S^T Q^T
#pragma unroll
            for (int n = 0; n < KD / 8; n += 2) {
                uint32_t x[SUM][4];
                left_of<SUM>(x, S[n], S[n + 1]);
                if (a.states) {
                    bf16* to = a.states + (unit * SUM * a.VP + v + g) * KD + n * 8 + c;
#pragma unroll
                    for (int p = 0; p < SUM; ++p, to += (size_t)a.VP * KD) {
                        *reinterpret_cast<uint32_t*>(to) = x[p][0], *reinterpret_cast<uint32_t*>(to + 8 * KD) = x[p][1];
                        *reinterpret_cast<uint32_t*>(to + 8) = x[p][2], *reinterpret_cast<uint32_t*>(to + 8 * KD + 8) = x[p][3];
                    }
                }
#pragma unroll
                for (int m = 0; m < 8; m += 2) {
#pragma unroll
                    for (int p = 0; p < IN; ++p) {
                        uint32_t r[4];
                        right_nk<KD>(r, s.k() + p * (kPiece * KD * 2), m * 8, n * 8, lane);
                        mma_parts<SUM>(R[m], R[m + 1], x, r, p);
                        right_nk<KD>(r, s.q() + p * (kPiece * KD * 2), m * 8, n * 8, lane);
#pragma unroll
                        for (int j = 0; j < OUT; ++j)
                            if (j + p < OUT) mma(O[m], x[j], r[0], r[1]), mma(O[m + 1], x[j], r[2], r[3]);
                    }
                }
            }
            // R = v - e^G S^T k, of this warp's columns; E = R - t (beta R)
            const T* vs = s.values() + warp * 16 + g;
            float E[8][4];
#pragma unroll
            for (int m = 0; m < 8; ++m) {
                const float2 eg = *reinterpret_cast<const float2*>(f + m * 8 + c);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float d = e & 1 ? eg.y : eg.x;
                    E[m][e] = fmaf(-d, R[m][e], to_float(vs[(m * 8 + c + (e & 1)) * s.pitch() + 8 * (e >> 1)]));
                    O[m][e] *= d;
                }
            }
#pragma unroll
            for (int m = 0; m < 8; ++m) {
                const float2 be = *reinterpret_cast<const float2*>(f + 2 * kPiece + m * 8 + c);
                R[m][0] = -be.x * E[m][0], R[m][1] = -be.y * E[m][1], R[m][2] = -be.x * E[m][2], R[m][3] = -be.y * E[m][3];
            }
#pragma unroll
            for (int j = 0; j < 8; j += 2) {                   // tokens j * 8 .. + 15 on tokens from there on
                uint32_t x[SUM][4];
                left_of<SUM>(x, R[j], R[j + 1]);
#pragma unroll
                for (int m = j; m < 8; m += 2) {
#pragma unroll
                    for (int p = 0; p < SUM; ++p) {
                        uint32_t r[4];
                        right_nk<kPiece>(r, s.t() + p * (kPiece * kPiece * 2), m * 8, j * 8, lane);
                        mma_parts<SUM>(E[m], E[m + 1], x, r, p);
                    }
                }
            }
            if (a.updates) {
#pragma unroll
                for (int m = 0; m < 8; ++m) {
                    uint32_t x[SUM], y[SUM];
                    split<SUM>(E[m][0], E[m][1], x);
                    split<SUM>(E[m][2], E[m][3], y);
                    bf16* to = a.updates + (unit * SUM * a.VP + v + g) * kPiece + m * 8 + c;
#pragma unroll
                    for (int p = 0; p < SUM; ++p, to += (size_t)a.VP * kPiece)
                        *reinterpret_cast<uint32_t*>(to) = x[p], *reinterpret_cast<uint32_t*>(to + 8 * kPiece) = y[p];
                }
            }
            // O += P (beta E)
#pragma unroll
            for (int m = 0; m < 8; ++m) {
                const float2 be = *reinterpret_cast<const float2*>(f + 2 * kPiece + m * 8 + c);
                E[m][0] *= be.x, E[m][1] *= be.y, E[m][2] *= be.x, E[m][3] *= be.y;
            }
#pragma unroll
            for (int j = 0; j < 8; j += 2) {
                uint32_t x[OUT][4];
                left_of<OUT>(x, E[j], E[j + 1]);
#pragma unroll
                for (int m = j; m < 8; m += 2) {
#pragma unroll
                    for (int p = 0; p < OUT; ++p) {
                        uint32_t r[4];
                        right_nk<kPiece>(r, s.p() + p * (kPiece * kPiece * 2), m * 8, j * 8, lane);
                        mma_parts<OUT>(O[m], O[m + 1], x, r, p);
                    }
                }
            }
            // S <- e^G_63 S + (e^(G_63 - G) beta E)^T K
            const float whole = f[kPiece - 1];
#pragma unroll
            for (int n = 0; n < KD / 8; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) S[n][e] *= whole;
#pragma unroll
            for (int j = 0; j < 8; j += 2) {
                const float2 d0 = *reinterpret_cast<const float2*>(f + kPiece + j * 8 + c), d1 = *reinterpret_cast<const float2*>(f + kPiece + j * 8 + 8 + c);
                const float u0[4] = {E[j][0] * d0.x, E[j][1] * d0.y, E[j][2] * d0.x, E[j][3] * d0.y};
                const float u1[4] = {E[j + 1][0] * d1.x, E[j + 1][1] * d1.y, E[j + 1][2] * d1.x, E[j + 1][3] * d1.y};
                uint32_t x[SUM][4];
                left_of<SUM>(x, u0, u1);
#pragma unroll
                for (int n = 0; n < KD / 8; n += 2) {
#pragma unroll
                    for (int p = 0; p < IN; ++p) {
                        uint32_t r[4];
                        right_kn<KD>(r, s.k() + p * (kPiece * KD * 2), j * 8, n * 8, lane);
                        mma_parts<SUM>(S[n], S[n + 1], x, r, p);
                    }
                }
            }
#pragma unroll
            for (int m = 0; m < 8; ++m)
#pragma unroll
                for (int e = 0; e < 4; ++e) O[m][e] *= a.scale;
            T* mine = reinterpret_cast<T*>(raw + STAGES * W::stage(warps)) + warp * kPiece * (16 + W::kPad);
            store_columns(O, mine, static_cast<T*>(a.o) + ((long long)b * a.L + (long long)i * kPiece) * a.ldo + (long long)h * a.V + v, a.ldo, len - i * kPiece,
                          a.V - v, wide_o, lane);
        }
        __syncthreads();
    }
    if (a.state_out && computes) {
#pragma unroll
        for (int n = 0; n < KD / 8; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int k = n * 8 + c + (e & 1), col = v + g + 8 * (e >> 1);
                if (k < a.K && col < a.V) a.state_out[state0 + (size_t)k * a.V + col] = S[n][e];
            }
    }
    zero_rows(static_cast<T*>(a.o) + (long long)b * a.L * a.ldo + (long long)h * a.V + v0, a.ldo, len, a.L, cols, tid, blockDim.x);
}

template <typename T, int KD>
conv2d_status_t walk(const DeltaArgs& a, cudaStream_t stream)
{
    using W = Walk<T, KD>;
    static SmemLimit limit;
    const int warps = delta_warps(a), across = (int)ceil_div_u(a.VP / 16, warps);
    const size_t smem = W::smem(warps);
    if (raise_smem_limit((const void*)delta_fwd_kernel<T, KD>, smem, limit) != cudaSuccess) return CONV2D_ERR_CUDA;
    const int per = 16 / (int)sizeof(T);
    const bool wide_v = a.V % per == 0 && rows_aligned(a.v, a.ldv, sizeof(T), 16), wide_o = a.V % per == 0 && rows_aligned(a.o, a.ldo, sizeof(T), 16);
    if (launch_pdl(delta_fwd_kernel<T, KD>, dim3((unsigned)(a.B * a.H) * across), dim3((warps + kLoaders) * 32), smem, stream, a, warps, across, wide_v, wide_o) !=
        cudaSuccess)
        return CONV2D_ERR_CUDA;
    count_launch();
    return CONV2D_OK;
}

template <typename T>
conv2d_status_t walk_typed(const DeltaArgs& a, cudaStream_t stream)
{
    if (a.K <= 32) return walk<T, 32>(a, stream);
    if (a.K <= 64) return walk<T, 64>(a, stream);
    return walk<T, 128>(a, stream);
}

}  // namespace

size_t delta_states_bytes(const DeltaLayout& l) { return l.prepared_bytes() + l.saved_bytes(); }
size_t delta_fwd_workspace_bytes(const DeltaLayout& l) { return l.prepared_bytes() + l.keys_bytes(); }

conv2d_status_t launch_delta_fwd(DeltaArgs a, conv2d_operand_t type, void* states, void* workspace, cudaStream_t stream)
{
    const DeltaLayout l(a.B, a.L, a.Hk, a.H, a.K, a.V, type);
    a.share = a.H / a.Hk, a.pieces = l.pieces, a.VP = l.VP;
    // (sections of whole multiples of 16 bytes)
    unsigned char* at = static_cast<unsigned char*>(states ? states : workspace);
    a.t = reinterpret_cast<bf16*>(at), a.p = reinterpret_cast<bf16*>(at + l.units * l.square());
    a.factors = reinterpret_cast<float*>(at + l.units * 2 * l.square());
    if (states) {
        a.states = reinterpret_cast<bf16*>(at + l.prepared_bytes());
        a.updates = reinterpret_cast<bf16*>(at + l.prepared_bytes() + l.units * l.state_plane());
    }
    if (!delta_direct(a, type, l.KD)) a.planes = reinterpret_cast<bf16*>(static_cast<unsigned char*>(workspace) + l.prepared_bytes());
    const conv2d_status_t st = launch_delta_prepare(a, type, true, stream);
    if (st != CONV2D_OK) return st;
    if (type == CONV2D_OPERAND_BF16) return walk_typed<bf16>(a, stream);
    if (type == CONV2D_OPERAND_FP16) return walk_typed<fp16>(a, stream);
    return walk_typed<float>(a, stream);
}

}  // namespace conv2d_b200
