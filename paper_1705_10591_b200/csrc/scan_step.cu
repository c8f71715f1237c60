// Selective state space scan, one token of every sequence.
#include "scan_common.cuh"

namespace conv2d_b200 {
namespace {

constexpr int kSpt = 4;                 // states of a thread

// One token: every state is read and written once, which is all the time there is.  A thread takes four adjacent states of one
// channel, of one sequence, or of four at once where there are many (their loads are under way together, A is loaded once for all, and each
// of the lanes of a channel does for one of the sequences what is done once for a channel: step size, gate, output).  256 x 4096 of 16 states in place:
// 37.5 us, 3.8 TB/s (without the look-ahead 47; memory is not full: step sizes, inputs, B and C are not fetched ahead, so every four sequences a warp waits for them
// once, eight of some 13 cycles between two instructions of a warp); 8 sequences are bound by the host's part of a call.
template <typename T>
struct StepArgs {
    const T *u, *delta, *Bm, *Cm, *z;
    const float *A, *Dskip, *delta_bias, *state_in;
    T* y;
    float* state_out;
    int B, D, N, G, E, NL, loops;       // loops: ROWS sequences after each other of a block
    unsigned across;                    // blocks for the channels of ROWS sequences
    long long ldu, lddelta, ldB, ldC, ldz, ldy;
    bool softplus, B_wide, C_wide;
};

// Four adjacent floats of which `real` exist.
template <bool QUADS>
__device__ __forceinline__ void load_states(const float* p, int real, float (&v)[kSpt])
{
    if (QUADS) {
        const float4 q = real > 0 ? *reinterpret_cast<const float4*>(p) : make_float4(0.f, 0.f, 0.f, 0.f);
        v[0] = q.x, v[1] = q.y, v[2] = q.z, v[3] = q.w;
    } else {
#pragma unroll
        for (int i = 0; i < kSpt; ++i) v[i] = i < real ? p[i] : 0.f;
    }
}
template <typename T>
__device__ __forceinline__ void load_inputs(const T* p, int real, bool wide, float (&v)[kSpt])
{
    if (wide) {
        unpack(real > 0 ? load_pack<T, kSpt>(p) : zero_pack<T, kSpt>(), v);
    } else {
#pragma unroll
        for (int i = 0; i < kSpt; ++i) v[i] = i < real ? to_float(p[i]) : 0.f;
    }
}

// Many sequences (QUADS, ROWS = 4): the states of the next four come in by asynchronous copies while these are stepped, `loops` fours in a row.
template <typename T, int ROWS, bool QUADS>
__global__ void __launch_bounds__(128) scan_step_kernel(const StepArgs<T> a)
{
    constexpr bool AHEAD = ROWS > 1 && QUADS;
    ptx::grid_dep_wait();
    __shared__ float4 ring[AHEAD ? 2 * ROWS * 128 : 1];
    const unsigned id = blockIdx.x % a.across * 128 + threadIdx.x;
    const int sl = (int)(id % a.NL), n0 = sl * kSpt;
    const bool mine = id / a.NL < (unsigned)a.D;
    const int d = mine ? (int)(id / a.NL) : 0, g = d / a.E, real = mine ? a.N - n0 : 0;
    // ROWS = 4 (a channel has four lanes or more): this lane's own sequence is b0 + sl % 4
    const int lane = threadIdx.x & 31, own = ROWS > 1 ? sl % ROWS : 0;
    const size_t next = (size_t)a.D * a.N;
    float A2[kSpt];
    load_states<QUADS>(a.A + (size_t)d * a.N + n0, real, A2);
#pragma unroll
    for (int i = 0; i < kSpt; ++i) A2[i] = decay_rate(A2[i]);
    const float bias = a.delta_bias && mine ? a.delta_bias[d] : 0.f, skip = a.Dskip && mine ? a.Dskip[d] : 0.f;
    const long long first = (long long)(blockIdx.x / a.across) * ROWS * a.loops;
    auto fetch = [&](int k) {
        const long long b0 = first + (long long)k * ROWS;
        const float* p = a.state_in + ((size_t)b0 * a.D + d) * a.N + n0;
#pragma unroll
        for (int r = 0; r < ROWS; ++r, p += next) {
            const bool there = k < a.loops && b0 + r < a.B && real > 0;
            copy_async<16>(ring + ((k & 1) * ROWS + r) * 128 + threadIdx.x, there ? p : a.state_in, there);
        }
        copies_commit();
    };
    if (AHEAD) fetch(0);
    for (int k = 0; k < a.loops; ++k) {
        const long long b0 = first + (long long)k * ROWS;
        if (b0 >= a.B) break;
        if (AHEAD) fetch(k + 1);
        const long long bo = b0 + own < a.B ? b0 + own : b0;
        float h[ROWS][kSpt], Bv[ROWS][kSpt], Cv[ROWS][kSpt];
        const size_t at = ((size_t)b0 * a.D + d) * a.N + n0;
        {
            const float* ph = a.state_in + at;
            const T *pb = a.Bm + b0 * a.ldB + (long long)g * a.N + n0, *pc = a.Cm + b0 * a.ldC + (long long)g * a.N + n0;
#pragma unroll
            for (int r = 0; r < ROWS; ++r, ph += next, pb += a.ldB, pc += a.ldC) {
                const int there = b0 + r < a.B ? real : 0;
                if (!AHEAD) load_states<QUADS>(ph, there, h[r]);
                load_inputs(pb, there, a.B_wide, Bv[r]);
                load_inputs(pc, there, a.C_wide, Cv[r]);
            }
        }
        const float u = mine ? to_float(a.u[bo * a.ldu + d]) : 0.f, z = mine && a.z ? to_float(a.z[bo * a.ldz + d]) : 0.f;
        float s = mine ? to_float(a.delta[bo * a.lddelta + d]) + bias : 0.f;
        if (a.softplus) s = softplus(s);
        const float su = s * u;
        if (AHEAD) {
            copies_wait<1>();
#pragma unroll
            for (int r = 0; r < ROWS; ++r) {
                const float4 q = ring[((k & 1) * ROWS + r) * 128 + threadIdx.x];
                h[r][0] = q.x, h[r][1] = q.y, h[r][2] = q.z, h[r][3] = q.w;
            }
        }
        float v[ROWS];
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            const int from = (lane & ~(ROWS - 1)) | r;
            const float sr = ROWS > 1 ? __shfl_sync(0xffffffffu, s, from) : s, sur = ROWS > 1 ? __shfl_sync(0xffffffffu, su, from) : su;
            v[r] = 0.f;
#pragma unroll
            for (int i = 0; i < kSpt; i += 2) {
                const float2 e = decay(both(sr), make_float2(A2[i], A2[i + 1]));
                const float2 x = __ffma2_rn(e, make_float2(h[r][i], h[r][i + 1]), __fmul2_rn(both(sur), make_float2(Bv[r][i], Bv[r][i + 1])));
                h[r][i] = x.x, h[r][i + 1] = x.y;
                v[r] = fmaf(Cv[r][i], x.x, v[r]);
                v[r] = fmaf(Cv[r][i + 1], x.y, v[r]);
            }
            if (b0 + r >= a.B || real <= 0) continue;
            float* out = a.state_out + at + r * next;
            if (QUADS) {
                *reinterpret_cast<float4*>(out) = make_float4(h[r][0], h[r][1], h[r][2], h[r][3]);
            } else {
#pragma unroll
                for (int i = 0; i < kSpt; ++i)
                    if (i < real) out[i] = h[r][i];
            }
        }
        if (ROWS > 1) sum_over_lanes<ROWS, ROWS, 1>(v, lane); // leaves the sum of this lane's own sequence
        for (int m = ROWS; m < a.NL; m *= 2) v[0] += __shfl_xor_sync(0xffffffffu, v[0], m);
        if (sl >= ROWS || !mine || b0 + own >= a.B) continue;
        float y = fmaf(skip, u, v[0]);
        if (a.z) y *= z * sigmoid(z);
        a.y[(b0 + own) * a.ldy + d] = from_float<T>(y);
    }
}

template <typename T, int ROWS, bool QUADS>
conv2d_status_t step(StepArgs<T> a, cudaStream_t stream)
{
    a.across = ceil_div_u((long long)a.D * a.NL, 128);
    // (fours in a row while the blocks are two for every place an SM has)
    a.loops = 1;
    while (ROWS > 1 && a.loops < 8 && (long long)a.across * ceil_div_u(a.B, 2 * ROWS * a.loops) >= 2LL * 5 * sm_count()) a.loops *= 2;
    const long long blocks = (long long)a.across * ceil_div_u(a.B, ROWS * a.loops);
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
    a.B_wide = s.N % kSpt == 0 && rows_aligned(s.Bm, s.ldB, sizeof(T), kSpt * sizeof(T)), a.C_wide = s.N % kSpt == 0 && rows_aligned(s.Cm, s.ldC, sizeof(T), kSpt * sizeof(T));
    // four sequences a thread once one each would be more threads than the machine holds (and a channel has four lanes to share them)
    const bool many = a.NL >= 4 && (long long)s.B * s.D * a.NL > (long long)sm_count() * 2048;
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
