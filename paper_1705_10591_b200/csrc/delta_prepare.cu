// Gated delta rule: what a piece of 64 tokens needs of its keys, queries, decays and betas, before any state is known.
#include "delta_common.cuh"

namespace conv2d_b200 {
namespace {

// One block of four warps for one piece of one key head; products of keys and queries are shared by its value heads.  Everything is computed transposed: warp w
// owns rows j = 16 w .. + 15 of
//   A^T_ji = e^(G_i - G_j) k_j.k_i (i > j),   P^T_ji = e^(G_i - G_j) k_j.q_i (i >= j),   t^T,   P'^T = P^T - t^T diag(beta) P^T,
// so that every block of 16 x 16 that it has computed is the left operand of its next products straight from the accumulators.  t^T comes from
// t^T (1 + diag(beta) A^T) = A^T from the left to the right: t^T_i = (A^T_ji - sum over k < i of t^T_k diag(beta) A^T_ki) (1 + diag(beta) A^T_ii)^-1, where the inverses
// of the four diagonal blocks are found column by column, 16 steps of 16 lanes.  (Powers of A would do without those steps, but for keys that are alike they
// grow to binomials, whose digits cancel.)  G is a scan over lanes in 64 bits: differences are taken of sums of decays that may be thousands, and a float would
// leave them 2^-24 of those.  What bounds it is latency, 12 warps an SM: barriers and dependent steps.
template <typename T, int KD>
struct Prepare {
    static constexpr int IN = Parts<T>::in, THREADS = 128, PITCH = 20;
    static constexpr int tile = IN * 2 * kPiece * KD * 2, part = kPiece * kPiece * 2, inverse = kPiece * 32;      // bytes; of one part, one part
    static constexpr int two = 2 * kSum * part;                                   // A^T and P^T, then what goes out: in the place of the keys and queries
    static constexpr int at_inverse = tile > two ? tile : two, at_diagonal = at_inverse + kSum * inverse;
    static constexpr int smem = at_diagonal + kPiece * PITCH * 4;
};
// Rows of 16 numbers: unit u of row r at u ^ (r / 4 & 1).
__device__ __forceinline__ uint32_t inverse_at(uint32_t base, int row, int unit) { return base + row * 32 + ((unit ^ ((row >> 2) & 1)) << 4); }

template <typename T, int KD, bool WIDE>
__global__ void __launch_bounds__(128, 3) delta_prepare_kernel(const DeltaArgs a, bool squares, int heads)
{
    using S = Prepare<T, KD>;
    constexpr int IN = S::IN, HALF = 2 * kPiece * 128;         // bytes of 64 numbers of all rows
    extern __shared__ __align__(1024) unsigned char raw[];
    __shared__ alignas(16) float high[kPiece], low[kPiece], betas[kPiece];
    ptx::grid_dep_wait();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    // this block's heads: `heads` of those that share the key, from `first_head` on
    const int groups = a.share / heads, key_unit = blockIdx.x / groups, first_head = blockIdx.x % groups * heads;
    const int piece = key_unit % a.pieces, bk = key_unit / a.pieces, hk = bk % a.Hk, b = bk / a.Hk;
    const int live = sequence_length(a.lengths, b, a.L) - piece * kPiece;
    if (live <= 0) return;
    const uint32_t base = ptx::smem_u32(raw), inverse = base + S::at_inverse;
    float* diagonal = reinterpret_cast<float*>(raw + S::at_diagonal);        // [64][PITCH]: row i of its block's A
    const long long row0 = (long long)b * a.L + (long long)piece * kPiece;
    auto place = [&](int p, int row, int unit) { return unit_at<64>((p * (KD / 64) + (unit >> 3)) * HALF, row, unit & 7); };

    // keys and queries, as parts; all that a thread takes of one (of both, where elements are short) is under way together
    unsigned char* tile = a.keys + (size_t)key_unit * S::tile;
    constexpr int UNITS = KD / 8, EACH = kPiece * UNITS / S::THREADS, AT_ONCE = sizeof(T) == 2 ? 2 : 1;
#pragma unroll
    for (int first = 0; first < 2; first += AT_ONCE) {
        Row<T, 8> x[AT_ONCE][EACH];
#pragma unroll
        for (int n = 0; n < AT_ONCE; ++n) {
            const bool query = first + n;
            const long long ld = query ? a.ldq : a.ldk;
            const T* from = static_cast<const T*>(query ? a.q : a.k) + row0 * ld + (long long)hk * a.K;
#pragma unroll
            for (int i = 0; i < EACH; ++i) {
                const int row = (tid + i * S::THREADS) / UNITS, unit = (tid + i * S::THREADS) % UNITS;
                x[n][i].template load<WIDE>(from + row * ld + unit * 8, row < live ? a.K - unit * 8 : 0);
            }
        }
#pragma unroll
        for (int n = 0; n < AT_ONCE; ++n) {
#pragma unroll
            for (int i = 0; i < EACH; ++i) {
                const int row = (tid + i * S::THREADS) / UNITS, unit = (tid + i * S::THREADS) % UNITS;
                uint4 v[IN];
                if constexpr (IN == 1) {
                    v[0] = *reinterpret_cast<const uint4*>(&x[n][i].p[0]);
                } else {
                    float f[8];
                    uint32_t w[4][IN];
                    x[n][i].get(f);
#pragma unroll
                    for (int j = 0; j < 4; ++j) split<IN>(f[2 * j], f[2 * j + 1], w[j]);
#pragma unroll
                    for (int p = 0; p < IN; ++p) v[p] = make_uint4(w[0][p], w[1][p], w[2][p], w[3][p]);
                }
#pragma unroll
                for (int p = 0; p < IN; ++p) {
                    const uint32_t at = place(p, (first + n) * kPiece + row, unit);
                    if (first_head == 0) *reinterpret_cast<uint4*>(tile + at) = v[p];
                    if (squares) *reinterpret_cast<uint4*>(raw + at) = v[p];
                }
            }
        }
    }
    if (!squares) return;
    float2 gate = make_float2(0.f, 0.f), beta = gate;          // of the first warp's two tokens a lane, a head ahead
    auto fetch = [&](int h) {
        const int token = 2 * lane;
        if (warp == 0) {
            gate.x = token < live ? a.g[(row0 + token) * a.ldg + h] : 0.f, gate.y = token + 1 < live ? a.g[(row0 + token + 1) * a.ldg + h] : 0.f;
            beta.x = token < live ? a.beta[(row0 + token) * a.ldbeta + h] : 0.f, beta.y = token + 1 < live ? a.beta[(row0 + token + 1) * a.ldbeta + h] : 0.f;
        }
    };
    fetch(hk * a.share + first_head);
    __syncthreads();

    // rows 16 warp .. + 15 of K K^T and K Q^T, columns from there on
    const int m0 = warp * 16, g = lane >> 2, c = 2 * (lane & 3);
    float kk[8][4] = {}, kq[8][4] = {};
#pragma unroll
    for (int k0 = 0; k0 < KD; k0 += 16) {
        uint32_t ak[IN][4];
        auto part = [&](int p) { return base + (p * (KD / 64) + k0 / 64) * HALF; };
#pragma unroll
        for (int p = 0; p < IN; ++p) left_mk<64>(ak[p], part(p), m0, k0 % 64, lane);
#pragma unroll
        for (int n = 0; n < 8; n += 2) {
            if (n * 8 < m0) continue;
            auto products = [&](float (&k1)[4], float (&k2)[4], float (&q1)[4], float (&q2)[4]) {
#pragma unroll
                for (int p = IN - 1; p >= 0; --p) {
                    uint32_t r[4];
                    right_nk<64>(r, part(p), n * 8, k0 % 64, lane);
                    mma_parts<IN>(k1, k2, ak, r, p);
                    right_nk<64>(r, part(p), kPiece + n * 8, k0 % 64, lane);
                    mma_parts<IN>(q1, q2, ak, r, p);
                }
            };
            if constexpr (IN == kSum) {                        // (an MMA cuts off what it adds, towards zero: o of keys of 128 fp32 numbers 1.0e-6 off with one sum, 3e-7 so)
                float s[4][4] = {};
                products(s[0], s[1], s[2], s[3]);
#pragma unroll
                for (int e = 0; e < 4; ++e) kk[n][e] += s[0][e], kk[n + 1][e] += s[1][e], kq[n][e] += s[2][e], kq[n + 1][e] += s[3][e];
            } else {
                products(kk[n], kk[n + 1], kq[n], kq[n + 1]);
            }
        }
    }
    __syncthreads();                                           // (their place is taken from here on)

    for (int r = first_head; r < first_head + heads; ++r) {
        const int h = hk * a.share + r;
        const size_t unit = ((size_t)b * a.H + h) * a.pieces + piece;
        if (warp == 0) {
            float* factors = reinterpret_cast<float*>(a.prepared + unit * kPrepared + kSquares);
            // (below -10000 taken as that: sums of infinities would have no differences; NaN stays)
            const double x[2] = {gate.x < -10000.f ? -10000.f : gate.x, gate.y < -10000.f ? -10000.f : gate.y};
            const float be[2] = {beta.x, beta.y};
            if (r + 1 < first_head + heads) fetch(h + 1);
            const double sum = x[0] + x[1];
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
            if (lane == 0) ptx::bulk_wait_group_read<0>();     // (what went out of the head before)
        }
        __syncthreads();
        // A^T and P^T: numbers (the left operands of these rows), parts (the right operands of all), the diagonal block of A
        float X[8][4], P[8][4];
#pragma unroll
        for (int n = 0; n < 8; ++n) {
            if (n * 8 < m0) {
#pragma unroll
                for (int e = 0; e < 4; ++e) X[n][e] = P[n][e] = 0.f;
                continue;
            }
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int j = m0 + g + 8 * half, i = n * 8 + c;
                const float hj = high[j], lj = low[j];
                const float2 hi = *reinterpret_cast<const float2*>(high + i), li = *reinterpret_cast<const float2*>(low + i);
                const float d0 = ex2(((hi.x - hj) + (li.x - lj)) * kLog2e), d1 = ex2(((hi.y - hj) + (li.y - lj)) * kLog2e);
                X[n][2 * half] = i > j ? d0 * kk[n][2 * half] : 0.f, X[n][2 * half + 1] = i + 1 > j ? d1 * kk[n][2 * half + 1] : 0.f;
                P[n][2 * half] = i >= j ? d0 * kq[n][2 * half] : 0.f, P[n][2 * half + 1] = i + 1 >= j ? d1 * kq[n][2 * half + 1] : 0.f;
                if (n * 8 < m0 + 16) {
                    diagonal[i * S::PITCH + (j & 15)] = X[n][2 * half], diagonal[(i + 1) * S::PITCH + (j & 15)] = X[n][2 * half + 1];
                }
                uint32_t wx[kSum], wp[kSum];
                split<kSum>(X[n][2 * half], X[n][2 * half + 1], wx);
                split<kSum>(P[n][2 * half], P[n][2 * half + 1], wp);
                const uint32_t at = unit_at<64>(0, j, n) + c * 2;
#pragma unroll
                for (int p = 0; p < kSum; ++p) {
                    *reinterpret_cast<uint32_t*>(raw + p * S::part + at) = wx[p];
                    *reinterpret_cast<uint32_t*>(raw + (kSum + p) * S::part + at) = wp[p];
                }
            }
        }
        __syncwarp();
        // column `lane` of (1 + A_ii diag(beta))^-1 of this warp's diagonal block; it is used transposed, [column][row]
        if (lane < 16) {
            float x[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                float s = i == lane ? 1.f : 0.f;
#pragma unroll
                for (int l = 0; l < i; l += 4) {
                    const float4 q = *reinterpret_cast<const float4*>(diagonal + (m0 + i) * S::PITCH + l);
                    s = fmaf(-q.x, x[l], s);
                    if (l + 1 < i) s = fmaf(-q.y, x[l + 1], s);
                    if (l + 2 < i) s = fmaf(-q.z, x[l + 2], s);
                    if (l + 3 < i) s = fmaf(-q.w, x[l + 3], s);
                }
                x[i] = s * betas[m0 + i];                      // (as the rows below use it; the product with beta is taken back below)
                uint32_t w[kSum];
                split<kSum>(s, 0.f, w);
#pragma unroll
                for (int p = 0; p < kSum; ++p)
                    *reinterpret_cast<uint16_t*>(raw + (inverse_at(inverse + p * S::inverse, m0 + i, lane >> 3) - base) + (lane & 7) * 2) = (uint16_t)w[p];
            }
        }
        __syncthreads();
        // t^T and P'^T: a block of 16 columns of t^T is done when those before it have been taken off, and is taken off all behind it, of P^T too
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (k < warp) continue;
            uint32_t x[kSum][4];
            float out[2][4] = {};
            left_of<kSum>(x, X[2 * k], X[2 * k + 1]);
#pragma unroll
            for (int p = kSum - 1; p >= 0; --p) {
                uint32_t q[4];
                ldsm(q, inverse_at(inverse + p * S::inverse, 16 * k + ((lane >> 4) << 3) + (lane & 7), (lane >> 3) & 1));
                mma_parts<kSum>(out[0], out[1], x, q, p);
            }
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) {                  // (below the diagonal is nothing but what rounding leaves there)
                    X[2 * k + n][e] = k > warp || 8 * n + c + (e & 1) > g + 8 * (e >> 1) ? out[n][e] : 0.f;
                    out[n][e] = -betas[16 * k + 8 * n + c + (e & 1)] * X[2 * k + n][e];
                }
            left_of<kSum>(x, out[0], out[1]);
#pragma unroll
            for (int i = k; i < 4; ++i) {
#pragma unroll
                for (int p = kSum - 1; p >= 0; --p) {
                    uint32_t q[4];
                    if (i > k) {
                        right_kn<64>(q, base + p * S::part, 16 * k, 16 * i, lane);
                        mma_parts<kSum>(X[2 * i], X[2 * i + 1], x, q, p);
                    }
                    right_kn<64>(q, base + (kSum + p) * S::part, 16 * k, 16 * i, lane);
                    mma_parts<kSum>(P[2 * i], P[2 * i + 1], x, q, p);
                }
            }
        }
        __syncthreads();
        // [part][-t^T, P'^T][64][64], out by one copy
#pragma unroll
        for (int n = 0; n < 8; ++n)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                uint32_t wx[kSum], wp[kSum];
                split<kSum>(-X[n][2 * half], -X[n][2 * half + 1], wx);
                split<kSum>(P[n][2 * half], P[n][2 * half + 1], wp);
                const uint32_t at = unit_at<64>(0, m0 + g + 8 * half, n) + c * 2;
#pragma unroll
                for (int p = 0; p < kSum; ++p) {
                    *reinterpret_cast<uint32_t*>(raw + 2 * p * S::part + at) = wx[p];
                    *reinterpret_cast<uint32_t*>(raw + (2 * p + 1) * S::part + at) = wp[p];
                }
            }
        ptx::fence_proxy_async_smem();
        __syncthreads();
        if (tid == 0) {
            asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(a.prepared + unit * kPrepared), "r"(base), "n"((int)kSquares) : "memory");
            ptx::bulk_commit_group();
        }
    }
    if (tid == 0) ptx::bulk_wait_group<0>();
}

template <typename T, int KD, bool WIDE>
conv2d_status_t prepare(const DeltaArgs& a, bool squares, cudaStream_t stream)
{
    using S = Prepare<T, KD>;
    static SmemLimit limit;
    if (raise_smem_limit((const void*)delta_prepare_kernel<T, KD, WIDE>, S::smem, limit) != cudaSuccess) return CONV2D_ERR_CUDA;
    // one head a block while an SM has room for all at once: keys and queries are read and multiplied for each then, but heads do not wait for one another
    const long long units = (long long)a.B * a.Hk * a.pieces;
    const int heads = !squares || units * a.share > 3LL * sm_count() ? a.share : 1;
    const long long blocks = units * (a.share / heads);
    if (launch_pdl(delta_prepare_kernel<T, KD, WIDE>, dim3((unsigned)blocks), dim3(S::THREADS), S::smem, stream, a, squares, heads) != cudaSuccess) return CONV2D_ERR_CUDA;
    count_launch();
    return CONV2D_OK;
}

template <typename T>
conv2d_status_t prepare_typed(const DeltaArgs& a, bool squares, cudaStream_t stream)
{
    const bool wide = a.K % 8 == 0 && rows_aligned(a.q, a.ldq, sizeof(T), 16) && rows_aligned(a.k, a.ldk, sizeof(T), 16);
    if (a.K <= 64) return wide ? prepare<T, 64, true>(a, squares, stream) : prepare<T, 64, false>(a, squares, stream);
    return wide ? prepare<T, 128, true>(a, squares, stream) : prepare<T, 128, false>(a, squares, stream);
}

}  // namespace

conv2d_status_t launch_delta_prepare(const DeltaArgs& a, conv2d_operand_t type, bool squares, cudaStream_t stream)
{
    if (type == CONV2D_OPERAND_BF16) return prepare_typed<bf16>(a, squares, stream);
    if (type == CONV2D_OPERAND_FP16) return prepare_typed<fp16>(a, squares, stream);
    return prepare_typed<float>(a, squares, stream);
}

}  // namespace conv2d_b200
