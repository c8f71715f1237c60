// Gated delta rule, one token of every sequence.
#include "delta_common.cuh"

namespace conv2d_b200 {
namespace {

// Every state is read and written once, which is all the time there is.  A block of 128 threads has one head's rows of K for up to 16 * VW columns of V: all of
// a thread's numbers (row `group`, `group` + groups, ..., of VW adjacent columns) are under way together and stay in registers, and since
//   o = scale (e^g S^T q + (k.q) u),
// S^T k and S^T q are summed over rows at once: one barrier between reading and writing.
template <typename T, int VW, int ROWS>
__global__ void __launch_bounds__(128) delta_step_kernel(const DeltaArgs a, int lanes, int across)
{
    __shared__ float ks[kMost], qs[kMost];
    __shared__ float2 sums[128 * VW];
    ptx::grid_dep_wait();
    const int tid = threadIdx.x, lane = tid % lanes, group = tid / lanes, groups = 128 / lanes;
    const int bh = blockIdx.x / across, h = bh % a.H, b = bh / a.H, hk = h / a.share;
    const int v = ((int)(blockIdx.x % across) * lanes + lane) * VW;
    const bool mine = v < a.V;
    const size_t at = (size_t)bh * a.K * a.V + v;
    float S[ROWS][VW];
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const int k = group + i * groups;
        const Pack<float, VW> p = load_masked<float, VW>(a.state_in + at + (size_t)k * a.V, mine && k < a.K);
#pragma unroll
        for (int e = 0; e < VW; ++e) S[i][e] = p.e[e];
    }
    if (tid < a.K) {
        ks[tid] = to_float(static_cast<const T*>(a.k)[b * a.ldk + (long long)hk * a.K + tid]);
        qs[tid] = to_float(static_cast<const T*>(a.q)[b * a.ldq + (long long)hk * a.K + tid]);
    }
    const float gate = a.g[b * a.ldg + h], decay = ex2(gate * kLog2e), beta = a.beta[b * a.ldbeta + h];
    float x[VW];
#pragma unroll
    for (int e = 0; e < VW; ++e) x[e] = mine ? to_float(static_cast<const T*>(a.v)[b * a.ldv + (long long)h * a.V + v + e]) : 0.f;
    __syncthreads();
    float2 s[VW];
#pragma unroll
    for (int e = 0; e < VW; ++e) s[e] = make_float2(0.f, 0.f);
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const int k = group + i * groups;
        if (k < a.K) {
            const float kk = ks[k], qq = qs[k];
#pragma unroll
            for (int e = 0; e < VW; ++e) {
                S[i][e] *= decay;
                s[e].x = fmaf(S[i][e], kk, s[e].x), s[e].y = fmaf(S[i][e], qq, s[e].y);
            }
        }
    }
#pragma unroll
    for (int e = 0; e < VW; ++e) sums[e * 128 + tid] = s[e];
    float kq = 0.f;
    for (int k = tid & 31; k < a.K; k += 32) kq = fmaf(ks[k], qs[k], kq);
#pragma unroll
    for (int d = 1; d < 32; d *= 2) kq += __shfl_xor_sync(0xffffffffu, kq, d);
    __syncthreads();
    float u[VW];
#pragma unroll
    for (int e = 0; e < VW; ++e) {
        float2 r = make_float2(0.f, 0.f);
        for (int i = 0; i < groups; ++i) {
            const float2 y = sums[e * 128 + i * lanes + lane];
            r.x += y.x, r.y += y.y;
        }
        u[e] = beta * (x[e] - r.x);
        if (group == 0 && mine) static_cast<T*>(a.o)[b * a.ldo + (long long)h * a.V + v + e] = from_float<T>(a.scale * fmaf(kq, u[e], r.y));
    }
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        const int k = group + i * groups;
        if (!mine || k >= a.K) continue;
        Pack<float, VW> p;
#pragma unroll
        for (int e = 0; e < VW; ++e) p.e[e] = fmaf(ks[k], u[e], S[i][e]);
        store_pack<float, VW>(a.state_out + at + (size_t)k * a.V, p);
    }
}

template <typename T, int VW, int ROWS>
conv2d_status_t step(const DeltaArgs& a, int lanes, cudaStream_t stream)
{
    const unsigned across = ceil_div_u(a.V, lanes * VW);
    if (launch_pdl(delta_step_kernel<T, VW, ROWS>, dim3((unsigned)(a.B * a.H) * across), dim3(128), 0, stream, a, lanes, (int)across) != cudaSuccess)
        return CONV2D_ERR_CUDA;
    count_launch();
    return CONV2D_OK;
}

template <typename T, int VW>
conv2d_status_t step_wide(const DeltaArgs& a, cudaStream_t stream)
{
    // as many as a row of the state has, from 4 up to 16: blocks of 64 columns hold 32 KB of a state of 128 x 128 in half the registers, and an SM has four of them where
    // it had two (256 tokens of 32 such heads, 1.08 GB, 60 calls in a row: 165 us, 6.5 TB/s, with 32 lanes 210, with 8 201; from some 900 calls in a row on 180)
    int lanes = 4;
    while (lanes < 16 && lanes * VW < a.V) lanes *= 2;
    const int rows = (a.K * lanes + 127) / 128;
    return rows <= 8 ? step<T, VW, 8>(a, lanes, stream) : step<T, VW, 16>(a, lanes, stream);
}

template <typename T>
conv2d_status_t step_typed(const DeltaArgs& a, cudaStream_t stream)
{
    if (a.V % 4 == 0 && rows_aligned(a.state_in, 4, 4, 16) && rows_aligned(a.state_out, 4, 4, 16)) return step_wide<T, 4>(a, stream);
    return step_wide<T, 1>(a, stream);
}

}  // namespace

conv2d_status_t launch_delta_step(const DeltaArgs& a, conv2d_operand_t type, cudaStream_t stream)
{
    if (type == CONV2D_OPERAND_BF16) return step_typed<bf16>(a, stream);
    if (type == CONV2D_OPERAND_FP16) return step_typed<fp16>(a, stream);
    return step_typed<float>(a, stream);
}

}  // namespace conv2d_b200
