// Selective state space scan, one token of every sequence.
#include "scan_common.cuh"

namespace conv2d_b200 {
namespace {

constexpr int kSpt = 4;                 // states of a thread

// One token: every state is read and written once, which is all the time there is.  A thread takes four adjacent states of one
// channel, for ROWS sequences at once (their loads are under way together, and A is loaded once for all).
template <typename T>
struct StepArgs {
    const T *u, *delta, *Bm, *Cm, *z;
    const float *A, *Dskip, *delta_bias, *state_in;
    T* y;
    float* state_out;
    int B, D, N, G, E, NL;
    unsigned across;                    // blocks for the channels of ROWS sequences
    long long ldu, lddelta, ldB, ldC, ldz, ldy;
    bool softplus;
};

template <typename T, int ROWS, bool QUADS>
__global__ void __launch_bounds__(128) scan_step_kernel(const StepArgs<T> a)
{
    ptx::grid_dep_wait();
    const unsigned id = blockIdx.x % a.across * 128 + threadIdx.x;
    const int n0 = (int)(id % a.NL) * kSpt;
    const bool mine = id / a.NL < (unsigned)a.D;
    const int d = mine ? (int)(id / a.NL) : 0, g = d / a.E;
    const long long b0 = (long long)(blockIdx.x / a.across) * ROWS;
    float A2[kSpt] = {}, h[ROWS][kSpt] = {}, Bv[ROWS][kSpt] = {}, Cv[ROWS][kSpt] = {}, u[ROWS], s[ROWS], z[ROWS];
    auto quad = [&](const float* p, float (&v)[kSpt]) {
        if (!mine) return;
        if (QUADS) {
            if (n0 < a.N) {
                const float4 q = *reinterpret_cast<const float4*>(p + n0);
                v[0] = q.x, v[1] = q.y, v[2] = q.z, v[3] = q.w;
            }
        } else {
#pragma unroll
            for (int i = 0; i < kSpt; ++i)
                if (n0 + i < a.N) v[i] = p[n0 + i];
        }
    };
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        const long long b = b0 + r;
        u[r] = s[r] = z[r] = 0.f;
        if (b >= a.B || !mine) continue;
        quad(a.state_in + ((size_t)b * a.D + d) * a.N, h[r]);
        u[r] = to_float(a.u[b * a.ldu + d]);
        s[r] = to_float(a.delta[b * a.lddelta + d]);
        if (a.z) z[r] = to_float(a.z[b * a.ldz + d]);
#pragma unroll
        for (int i = 0; i < kSpt; ++i) {
            if (n0 + i >= a.N) continue;
            Bv[r][i] = to_float(a.Bm[b * a.ldB + g * a.N + n0 + i]);
            Cv[r][i] = to_float(a.Cm[b * a.ldC + g * a.N + n0 + i]);
        }
    }
    quad(a.A + (size_t)d * a.N, A2);
#pragma unroll
    for (int i = 0; i < kSpt; ++i) A2[i] *= kLog2e;
    const float bias = a.delta_bias && mine ? a.delta_bias[d] : 0.f, skip = a.Dskip && mine ? a.Dskip[d] : 0.f;
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        const long long b = b0 + r;
        s[r] += bias;
        if (a.softplus) s[r] = softplus(s[r]);
        float v = 0.f;
#pragma unroll
        for (int i = 0; i < kSpt; ++i) {
            h[r][i] = fmaf(ex2(s[r] * A2[i]), h[r][i], s[r] * u[r] * Bv[r][i]);
            v = fmaf(Cv[r][i], h[r][i], v);
        }
        for (int m = 1; m < a.NL; m *= 2) v += __shfl_xor_sync(0xffffffffu, v, m);
        if (b >= a.B || !mine) continue;
        float* out = a.state_out + ((size_t)b * a.D + d) * a.N;
        if (QUADS) {
            if (n0 < a.N) *reinterpret_cast<float4*>(out + n0) = make_float4(h[r][0], h[r][1], h[r][2], h[r][3]);
        } else {
#pragma unroll
            for (int i = 0; i < kSpt; ++i)
                if (n0 + i < a.N) out[n0 + i] = h[r][i];
        }
        if (n0 == 0) {
            v = fmaf(skip, u[r], v);
            if (a.z) v *= z[r] * sigmoid(z[r]);
            a.y[b * a.ldy + d] = from_float<T>(v);
        }
    }
}

template <typename T, int ROWS, bool QUADS>
conv2d_status_t step(StepArgs<T> a, cudaStream_t stream)
{
    a.across = ceil_div_u((long long)a.D * a.NL, 128);
    const long long blocks = (long long)a.across * ceil_div_u(a.B, ROWS);
    if (blocks > 0x7fffffffLL) return CONV2D_ERR_SHAPE;
    if (launch_pdl(scan_step_kernel<T, ROWS, QUADS>, dim3((unsigned)blocks), dim3(128), 0, stream, a) != cudaSuccess) return CONV2D_ERR_CUDA;
    count_launch();
    return CONV2D_OK;
}

template <typename T>
conv2d_status_t step_typed(const ScanSeq& s, cudaStream_t stream)
{
    StepArgs<T> a;
    a.u = static_cast<const T*>(s.u), a.delta = static_cast<const T*>(s.delta), a.z = static_cast<const T*>(s.z);
    a.Bm = static_cast<const T*>(s.Bm), a.Cm = static_cast<const T*>(s.Cm);
    a.A = s.A, a.Dskip = s.Dskip, a.delta_bias = s.delta_bias, a.state_in = s.state_in, a.y = static_cast<T*>(s.y), a.state_out = s.state_out;
    a.B = s.B, a.D = s.D, a.N = s.N, a.G = s.G, a.E = s.D / s.G, a.NL = lanes_for(s.N, kSpt);
    a.ldu = s.ldu, a.lddelta = s.lddelta, a.ldB = s.ldB, a.ldC = s.ldC, a.ldz = s.ldz, a.ldy = s.ldy, a.softplus = s.softplus;
    const bool quads = s.N % 4 == 0 && rows_aligned(s.A, 4, 4, 16) && rows_aligned(s.state_in, 4, 4, 16) && rows_aligned(s.state_out, 4, 4, 16);
    // four sequences a thread once one each would be more threads than the machine holds
    const bool many = (long long)s.B * s.D * a.NL > (long long)sm_count() * 2048;
    if (quads) return many ? step<T, 4, true>(a, stream) : step<T, 1, true>(a, stream);
    return many ? step<T, 4, false>(a, stream) : step<T, 1, false>(a, stream);
}

}  // namespace

conv2d_status_t launch_scan_step(const ScanSeq& s, conv2d_operand_t type, cudaStream_t stream)
{
    if (type == CONV2D_OPERAND_BF16) return step_typed<bf16>(s, stream);
    if (type == CONV2D_OPERAND_FP16) return step_typed<fp16>(s, stream);
    return step_typed<float>(s, stream);
}

}  // namespace conv2d_b200
