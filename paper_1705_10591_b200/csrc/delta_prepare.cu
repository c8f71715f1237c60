// Gated delta rule: what a piece of 64 tokens needs of its keys, queries, decays and betas, before any state is known.
#include "delta_common.cuh"

namespace conv2d_b200 {
namespace {

// One block for one piece of one key head; K K^T and Q K^T are shared by its value heads.  Per value head: G by a scan over lanes in 64 bits
// (differences of sums of decays are taken of sums that may be thousands: a float would leave them 2^-24 of those), A and P from the products, and
// t column by column: row i of (1 + A diag(beta)) t = A gives t_ij from the t_lj above it, one thread a column.
template <typename T, int KD>
struct Prepare {
    static constexpr int IN = Parts<T>::in, SUM = Parts<T>::sum;
    static constexpr int THREADS = 128, PITCH = kPiece + 4;
    static constexpr size_t tile = (size_t)IN * kPiece * KD * 2;
    static constexpr size_t smem = 2 * tile + 2 * kPiece * PITCH * 4;
};

template <typename T, int KD>
__global__ void __launch_bounds__(128) delta_prepare_kernel(const DeltaArgs a, bool squares)
{
    using S = Prepare<T, KD>;
    constexpr int IN = S::IN, SUM = S::SUM, PITCH = S::PITCH;
    extern __shared__ __align__(1024) unsigned char raw[];
    __shared__ float high[kPiece], low[kPiece], betas[kPiece];
    ptx::grid_dep_wait();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int piece = blockIdx.x % a.pieces, bk = blockIdx.x / a.pieces, hk = bk % a.Hk, b = bk / a.Hk;
    const int live = sequence_length(a.lengths, b, a.L) - piece * kPiece;
    if (live <= 0) return;
    const uint32_t ks = ptx::smem_u32(raw), qs = ks + (uint32_t)S::tile;
    float* As = reinterpret_cast<float*>(raw + 2 * S::tile);
    float* ts = As + kPiece * PITCH;
    const long long row0 = (long long)b * a.L + (long long)piece * kPiece;

    // keys and queries, as parts
    for (int which = 0; which < 2; ++which) {
        const T* from = static_cast<const T*>(which ? a.q : a.k) + row0 * (which ? a.ldq : a.ldk) + (long long)hk * a.K;
        const long long ld = which ? a.ldq : a.ldk;
        const bool wide = a.K % 8 == 0 && (reinterpret_cast<uintptr_t>(from) | (uintptr_t)(ld * sizeof(T))) % 16 == 0;
        bf16* plane = a.planes ? a.planes + ((size_t)blockIdx.x * 2 + which) * (IN * kPiece * KD) : nullptr;
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
                *reinterpret_cast<uint4*>(raw + (unit_at<KD>((which ? qs : ks) + p * (kPiece * KD * 2), row, unit) - ks)) = v;
                if (plane) *reinterpret_cast<uint4*>(plane + (size_t)(p * kPiece + row) * KD + unit * 8) = v;
            }
        }
    }
    if (!squares) return;
    __syncthreads();

    // rows 16 warp .. + 15 of K K^T and Q K^T
    const int m0 = warp * 16, g = lane >> 2, c = lane & 3;
    float kk[8][4] = {}, qk[8][4] = {};
#pragma unroll
    for (int k0 = 0; k0 < KD; k0 += 16) {
        uint32_t ak[IN][4], aq[IN][4];
#pragma unroll
        for (int p = 0; p < IN; ++p) {
            left_mk<KD>(ak[p], ks + p * (kPiece * KD * 2), m0, k0, lane);
            left_mk<KD>(aq[p], qs + p * (kPiece * KD * 2), m0, k0, lane);
        }
#pragma unroll
        for (int n = 0; n < 8; n += 2) {
            if (n * 8 > m0) continue;                          // columns behind the rows are not looked at
#pragma unroll
            for (int p = 0; p < IN; ++p) {
                uint32_t r[4];
                right_nk<KD>(r, ks + p * (kPiece * KD * 2), n * 8, k0, lane);
                mma_parts<IN>(kk[n], kk[n + 1], ak, r, p);
                mma_parts<IN>(qk[n], qk[n + 1], aq, r, p);
            }
        }
    }

    for (int r = 0; r < a.share; ++r) {
        const int h = hk * a.share + r;
        const size_t unit = ((size_t)b * a.H + h) * a.pieces + piece;
        float* factors = a.factors + unit * (kFactors * kPiece);
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
        bf16* P = a.p + unit * (SUM * kPiece * kPiece);
#pragma unroll
        for (int n = 0; n < 8; ++n) {
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int i = m0 + g + 8 * half, j = n * 8 + 2 * c;
                float pv[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float d = ex2(((high[i] - high[j + e]) + (low[i] - low[j + e])) * kLog2e);
                    As[i * PITCH + j + e] = j + e < i ? d * kk[n][2 * half + e] : 0.f;
                    pv[e] = j + e <= i ? d * qk[n][2 * half + e] : 0.f;
                }
                uint32_t w[SUM];
                split<SUM>(pv[0], pv[1], w);
#pragma unroll
                for (int p = 0; p < SUM; ++p) *reinterpret_cast<uint32_t*>(P + (p * kPiece + i) * kPiece + j) = w[p];
            }
        }
        __syncthreads();
        if (tid < kPiece) {
            float x[kPiece];                                   // beta_l t_lj of this thread's column j = tid
#pragma unroll
            for (int i = 0; i < kPiece; ++i) {
                float s[4] = {As[i * PITCH + tid], 0.f, 0.f, 0.f};
#pragma unroll
                for (int l = 0; l < i; l += 4) {
                    const float4 q = *reinterpret_cast<const float4*>(As + i * PITCH + l);
                    s[0] = fmaf(-q.x, x[l], s[0]);
                    if (l + 1 < i) s[1] = fmaf(-q.y, x[l + 1], s[1]);
                    if (l + 2 < i) s[2] = fmaf(-q.z, x[l + 2], s[2]);
                    if (l + 3 < i) s[3] = fmaf(-q.w, x[l + 3], s[3]);
                }
                const float v = tid < i ? (s[0] + s[1]) + (s[2] + s[3]) : 0.f;
                ts[i * PITCH + tid] = v;
                x[i] = betas[i] * v;
            }
        }
        __syncthreads();
        bf16* t = a.t + unit * (SUM * kPiece * kPiece);
        for (int i = tid; i < kPiece * kPiece / 2; i += S::THREADS) {
            const int row = i / 32, col = i % 32 * 2;
            uint32_t w[SUM];
            split<SUM>(ts[row * PITCH + col], ts[row * PITCH + col + 1], w);
#pragma unroll
            for (int p = 0; p < SUM; ++p) *reinterpret_cast<uint32_t*>(t + (p * kPiece + row) * kPiece + col) = w[p];
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
    if (a.K <= 32) return prepare<T, 32>(a, squares, stream);
    if (a.K <= 64) return prepare<T, 64>(a, squares, stream);
    return prepare<T, 128>(a, squares, stream);
}

}  // namespace

conv2d_status_t launch_delta_prepare(const DeltaArgs& a, conv2d_operand_t type, bool squares, cudaStream_t stream)
{
    if (type == CONV2D_OPERAND_BF16) return prepare_typed<bf16>(a, squares, stream);
    if (type == CONV2D_OPERAND_FP16) return prepare_typed<fp16>(a, squares, stream);
    return prepare_typed<float>(a, squares, stream);
}

}  // namespace conv2d_b200
