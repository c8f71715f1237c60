// Gated delta rule: what a piece of 64 tokens needs of its keys, queries, decays and betas, before any state is known.
#include "delta_common.cuh"

namespace conv2d_b200 {
namespace {

// One block of four warps for one piece of one key head; K K^T and Q K^T are shared by its value heads.  Per value head: G by a scan over lanes in 64 bits
// (differences are taken of sums of decays that may be thousands: a float would leave them 2^-24 of those), A and P from the products, and t from
// (1 + A diag(beta)) t = A by blocks of 16: the four diagonal blocks are inverted column by column (64 threads, 16 steps), then warp j solves the 16
// columns j of t from the top down, t_ij = (1 + A_ii diag(beta))^-1 (A_ij - sum A_ik diag(beta) t_kj), transposed, so that every block is the left operand of the
// next products straight from the accumulators.  (One thread a column over all 64 rows, two warps of four idle: 17 us a head of latency, 322 us for
// 16384 tokens of 32 heads.)
template <typename T, int KD>
struct Prepare {
    static constexpr int IN = Parts<T>::in, THREADS = 128;
    static constexpr int tile = IN * 2 * kPiece * KD * 2, part = kPiece * kPiece * 2, inverse = kPiece * 32;      // bytes; of one part, one part
    static constexpr int at_square = tile, at_inverse = at_square + kSum * part, at_diagonal = at_inverse + kSum * inverse;
    static constexpr int smem = at_diagonal + kPiece * 17 * 4;
};
// Rows of 16 numbers: unit u of row r at u ^ (r / 4 & 1).
__device__ __forceinline__ uint32_t inverse_at(uint32_t base, int row, int unit) { return base + row * 32 + ((unit ^ ((row >> 2) & 1)) << 4); }

template <typename T, int KD>
__global__ void __launch_bounds__(128, 3) delta_prepare_kernel(const DeltaArgs a, bool squares)
{
    using S = Prepare<T, KD>;
    constexpr int IN = S::IN, HALF = 2 * kPiece * 128;         // bytes of 64 numbers of all rows
    extern __shared__ __align__(1024) unsigned char raw[];
    __shared__ float high[kPiece], low[kPiece], betas[kPiece];
    ptx::grid_dep_wait();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int piece = blockIdx.x % a.pieces, bk = blockIdx.x / a.pieces, hk = bk % a.Hk, b = bk / a.Hk;
    const int live = sequence_length(a.lengths, b, a.L) - piece * kPiece;
    if (live <= 0) return;
    const uint32_t base = ptx::smem_u32(raw), square = base + S::at_square, inverse = base + S::at_inverse;
    float* diagonal = reinterpret_cast<float*>(raw + S::at_diagonal);        // [64][17]
    const long long row0 = (long long)b * a.L + (long long)piece * kPiece;
    auto place = [&](int p, int row, int unit) { return unit_at<64>((p * (KD / 64) + (unit >> 3)) * HALF, row, unit & 7); };

    // keys and queries, as parts
    unsigned char* tile = a.keys + (size_t)blockIdx.x * S::tile;
    for (int which = 0; which < 2; ++which) {
        const T* from = static_cast<const T*>(which ? a.q : a.k) + row0 * (which ? a.ldq : a.ldk) + (long long)hk * a.K;
        const long long ld = which ? a.ldq : a.ldk;
        const bool wide = a.K % 8 == 0 && (reinterpret_cast<uintptr_t>(from) | (uintptr_t)(ld * sizeof(T))) % 16 == 0;
#pragma unroll 4
        for (int i = tid; i < kPiece * (KD / 8); i += S::THREADS) {
            const int row = i / (KD / 8), unit = i % (KD / 8);
            float f[8];
            if (row < live && wide && unit * 8 < a.K) {
                unpack(load_pack<T, 8>(from + row * ld + unit * 8), f);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) f[j] = row < live && unit * 8 + j < a.K ? to_float(from[row * ld + unit * 8 + j]) : 0.f;
            }
            uint32_t w[4][IN];
#pragma unroll
            for (int j = 0; j < 4; ++j) split<IN>(f[2 * j], f[2 * j + 1], w[j]);
#pragma unroll
            for (int p = 0; p < IN; ++p) {
                const uint4 v = make_uint4(w[0][p], w[1][p], w[2][p], w[3][p]);
                const uint32_t at = place(p, which * kPiece + row, unit);
                *reinterpret_cast<uint4*>(tile + at) = v;
                if (squares) *reinterpret_cast<uint4*>(raw + at) = v;
            }
        }
    }
    if (!squares) return;
    __syncthreads();

    // rows 16 warp .. + 15 of K K^T and Q K^T
    const int m0 = warp * 16, g = lane >> 2, c = 2 * (lane & 3);
    float kk[8][4] = {}, qk[8][4] = {};
#pragma unroll
    for (int k0 = 0; k0 < KD; k0 += 16) {
        uint32_t ak[IN][4], aq[IN][4];
        auto part = [&](int p) { return base + (p * (KD / 64) + k0 / 64) * HALF; };
#pragma unroll
        for (int p = 0; p < IN; ++p) {
            left_mk<64>(ak[p], part(p), m0, k0 % 64, lane);
            left_mk<64>(aq[p], part(p), kPiece + m0, k0 % 64, lane);
        }
#pragma unroll
        for (int n = 0; n < 8; n += 2) {
            if (n * 8 > m0) continue;                          // columns behind the rows are not looked at
#pragma unroll
            for (int p = 0; p < IN; ++p) {
                uint32_t r[4];
                right_nk<64>(r, part(p), n * 8, k0 % 64, lane);
                mma_parts<IN>(kk[n], kk[n + 1], ak, r, p);
                mma_parts<IN>(qk[n], qk[n + 1], aq, r, p);
            }
        }
    }

    for (int r = 0; r < a.share; ++r) {
        const int h = hk * a.share + r;
        const size_t unit = ((size_t)b * a.H + h) * a.pieces + piece;
        float* factors = a.factors + unit * (kFactors * kPiece);
        unsigned char* out = a.squares + unit * kSquares;      // [part][-t, P'][64 rows]
        if (warp == 0) {
            double x[2], sum;
            float be[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int token = 2 * lane + j;
                float v = token < live ? a.g[(row0 + token) * a.ldg + h] : 0.f;
                v = v < -10000.f ? -10000.f : v;               // (a sum of infinities would have no differences; NaN stays)
                x[j] = v, be[j] = token < live ? a.beta[(row0 + token) * a.ldbeta + h] : 0.f;
            }
            sum = x[0] + x[1];
            double before = sum;
#pragma unroll
            for (int d = 1; d < 32; d *= 2) {
                const double y = __shfl_up_sync(0xffffffffu, before, d);
                if (lane >= d) before += y;
            }
            const double whole = __shfl_sync(0xffffffffu, before, 31);
            double G = before - sum;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                G += x[j];
                const int i = 2 * lane + j;
                const float hi = (float)G, lo = (float)(G - (double)hi);
                high[i] = hi, low[i] = lo, betas[i] = be[j];
                factors[i] = ex2((float)(G * 1.4426950408889634));
                factors[kPiece + i] = ex2((float)((whole - G) * 1.4426950408889634));
                factors[2 * kPiece + i] = be[j];
                factors[3 * kPiece + i] = hi, factors[4 * kPiece + i] = lo;
            }
        }
        __syncthreads();
        // A, in parts and its diagonal blocks as numbers, and P
        float P[8][4];
#pragma unroll
        for (int n = 0; n < 8; ++n) {
            if (n * 8 > m0 + 8) {
#pragma unroll
                for (int e = 0; e < 4; ++e) P[n][e] = 0.f;
                continue;
            }
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int i = m0 + g + 8 * half, j = n * 8 + c;
                float av[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float d = ex2(((high[i] - high[j + e]) + (low[i] - low[j + e])) * kLog2e);
                    av[e] = j + e < i ? d * kk[n][2 * half + e] : 0.f;
                    P[n][2 * half + e] = j + e <= i ? d * qk[n][2 * half + e] : 0.f;
                    if (n * 8 >= m0) diagonal[i * 17 + (j & 15) + e] = av[e];
                }
                uint32_t w[kSum];
                split<kSum>(av[0], av[1], w);
#pragma unroll
                for (int p = 0; p < kSum; ++p) *reinterpret_cast<uint32_t*>(raw + (unit_at<64>(square + p * S::part, i, j >> 3) - base) + (j & 7) * 2) = w[p];
            }
        }
        __syncthreads();
        // columns of the inverses of 1 + A_ii diag(beta)
        if (tid < kPiece) {
            const int block = tid & ~15, col = tid & 15;
            float x[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                float s = 0.f;
#pragma unroll
                for (int l = 0; l < i; ++l) s = fmaf(diagonal[(block + i) * 17 + l], x[l], s);
                const float v = (i == col ? 1.f : 0.f) - s;
                x[i] = v * betas[block + i];                   // (as the rows below use it)
                uint32_t w[kSum];
                split<kSum>(v, 0.f, w);
#pragma unroll
                for (int p = 0; p < kSum; ++p)
                    *reinterpret_cast<uint16_t*>(raw + (inverse_at(inverse + p * S::inverse, block + i, col >> 3) - base) + (col & 7) * 2) = (uint16_t)w[p];
            }
        }
        __syncthreads();
        // columns 16 warp .. + 15 of t, transposed: X[i] has rows of them and columns of tokens 16 i .. + 15
        float X[4][2][4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float sum[2][4];
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) X[i][n][e] = 0.f;
            if (i < warp) continue;
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int row = 16 * i + 8 * n + c + (e & 1), col = m0 + g + 8 * (e >> 1);
                    float v = 0.f;
#pragma unroll
                    for (int p = kSum - 1; p >= 0; --p)
                        v += __uint_as_float((uint32_t)*reinterpret_cast<const uint16_t*>(raw + (unit_at<64>(square + p * S::part, row, col >> 3) - base) + (col & 7) * 2) << 16);
                    sum[n][e] = v;
                }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if (k >= i) break;
                if (k < warp) continue;
                float y[2][4];
#pragma unroll
                for (int n = 0; n < 2; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) y[n][e] = -betas[16 * k + 8 * n + c + (e & 1)] * X[k][n][e];
                uint32_t x[kSum][4];
                left_of<kSum>(x, y[0], y[1]);
#pragma unroll
                for (int p = kSum - 1; p >= 0; --p) {
                    uint32_t q[4];
                    right_nk<64>(q, square + p * S::part, 16 * i, 16 * k, lane);
                    mma_parts<kSum>(sum[0], sum[1], x, q, p);
                }
            }
            uint32_t x[kSum][4];
            left_of<kSum>(x, sum[0], sum[1]);
#pragma unroll
            for (int p = kSum - 1; p >= 0; --p) {
                uint32_t q[4];
                ldsm(q, inverse_at(inverse + p * S::inverse, 16 * i + ((lane >> 4) << 3) + (lane & 7), (lane >> 3) & 1));
                mma_parts<kSum>(X[i][0], X[i][1], x, q, p);
            }
        }
        __syncthreads();
        // -t in the place of A
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int e = 0; e < 4; e += 2) {               // (tokens c and c + 1: two rows of one column)
                    const int row = 16 * i + 8 * n + c, col = m0 + g + 4 * e;
                    uint32_t w[kSum];
                    // the diagonal block's upper half is zero but for what rounding leaves there
                    split<kSum>(row > col ? -X[i][n][e] : 0.f, row + 1 > col ? -X[i][n][e + 1] : 0.f, w);
#pragma unroll
                    for (int p = 0; p < kSum; ++p) {
                        *reinterpret_cast<uint16_t*>(raw + (unit_at<64>(square + p * S::part, row, col >> 3) - base) + (col & 7) * 2) = (uint16_t)w[p];
                        *reinterpret_cast<uint16_t*>(raw + (unit_at<64>(square + p * S::part, row + 1, col >> 3) - base) + (col & 7) * 2) = (uint16_t)(w[p] >> 16);
                    }
                }
        __syncthreads();
        // P' = P + (P diag(beta)) (-t), rows 16 warp .. + 15
        float W[8][4];
#pragma unroll
        for (int n = 0; n < 8; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) W[n][e] = P[n][e];
#pragma unroll
        for (int k = 0; k < 8; k += 2) {
            if (k * 8 > m0) continue;
            float y[2][4];
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) y[n][e] = betas[(k + n) * 8 + c + (e & 1)] * P[k + n][e];
            uint32_t x[kSum][4];
            left_of<kSum>(x, y[0], y[1]);
#pragma unroll
            for (int n = 0; n <= k; n += 2) {
#pragma unroll
                for (int p = kSum - 1; p >= 0; --p) {
                    uint32_t q[4];
                    right_kn<64>(q, square + p * S::part, k * 8, n * 8, lane);
                    mma_parts<kSum>(W[n], W[n + 1], x, q, p);
                }
            }
        }
#pragma unroll
        for (int n = 0; n < 8; ++n)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int i = m0 + g + 8 * half;
                uint32_t w[kSum];
                split<kSum>(W[n][2 * half], W[n][2 * half + 1], w);
#pragma unroll
                for (int p = 0; p < kSum; ++p) *reinterpret_cast<uint32_t*>(out + unit_at<64>((2 * p + 1) * S::part, i, n) + c * 2) = w[p];
            }
        for (int i = tid; i < kSum * S::part / 16; i += S::THREADS) {
            const int p = i / (S::part / 16), rest = i % (S::part / 16);
            *reinterpret_cast<uint4*>(out + 2 * p * S::part + rest * 16) = *reinterpret_cast<const uint4*>(raw + S::at_square + p * S::part + rest * 16);
        }
        __syncthreads();
    }
}

template <typename T, int KD>
conv2d_status_t prepare(const DeltaArgs& a, bool squares, cudaStream_t stream)
{
    using S = Prepare<T, KD>;
    static SmemLimit limit;
    if (raise_smem_limit((const void*)delta_prepare_kernel<T, KD>, S::smem, limit) != cudaSuccess) return CONV2D_ERR_CUDA;
    const long long blocks = (long long)a.B * a.Hk * a.pieces;
    if (launch_pdl(delta_prepare_kernel<T, KD>, dim3((unsigned)blocks), dim3(S::THREADS), S::smem, stream, a, squares) != cudaSuccess) return CONV2D_ERR_CUDA;
    count_launch();
    return CONV2D_OK;
}

template <typename T>
conv2d_status_t prepare_typed(const DeltaArgs& a, bool squares, cudaStream_t stream)
{
    return a.K <= 64 ? prepare<T, 64>(a, squares, stream) : prepare<T, 128>(a, squares, stream);
}

}  // namespace

conv2d_status_t launch_delta_prepare(const DeltaArgs& a, conv2d_operand_t type, bool squares, cudaStream_t stream)
{
    if (type == CONV2D_OPERAND_BF16) return prepare_typed<bf16>(a, squares, stream);
    if (type == CONV2D_OPERAND_FP16) return prepare_typed<fp16>(a, squares, stream);
    return prepare_typed<float>(a, squares, stream);
}

}  // namespace conv2d_b200
