// What the forward and the backward scan share: how a warp holds states, sums over lanes, step sizes, segments of time.
//
// A thread holds four adjacent states of one channel; NL lanes next to each other hold a channel's states (up to 4 NL, the
// power of two that covers N) and the 32 / NL groups of lanes of a warp adjacent channels.  So a sum over the states is a sum over NL lanes, a
// sum over channels one over 32 / NL lanes and the warps, and the states never leave the registers.
#pragma once

#include "seq_common.cuh"

namespace conv2d_b200 {

constexpr int kSpt = 4;                 // states of a thread
constexpr int kCheckpointRows = 16;     // the forward pass keeps the state before every 16th row for the backward pass
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.69314718055994531f;

__device__ __forceinline__ float ex2(float v)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}

// log(1 + e^v)
__device__ __forceinline__ float softplus(float v) { return (v > 0.f ? v : 0.f) + log1pf(__expf(-fabsf(v))); }

// Sums of NV values over the LANES lanes that differ in the bits LANES/2 * UNIT .. UNIT of the lane index.  While more than one value is left a lane hands half of
// them over and goes on with the sums of the other half, so that NV - 1 exchanges do for log2(LANES) * NV; at the end v[0 .. left) hold the
// values first .. first + left, left = max(1, NV / LANES), in every lane whose further bits are anything.
template <int NV, int LANES, int UNIT>
__device__ __forceinline__ int sum_over_lanes(float (&v)[NV], int lane)
{
    int cnt = NV, first = 0;
#pragma unroll
    for (int m = LANES / 2; m >= 1; m /= 2) {
        const int mask = m * UNIT;
        const bool upper = (lane & mask) != 0;
        if (cnt > 1) {
            cnt /= 2;
#pragma unroll
            for (int i = 0; i < NV / 2; ++i) {
                if (i < cnt) {
                    const float send = upper ? v[i] : v[i + cnt], keep = upper ? v[i + cnt] : v[i];
                    v[i] = keep + __shfl_xor_sync(0xffffffffu, send, mask);
                }
            }
            if (upper) first += cnt;
        } else {
            v[0] += __shfl_xor_sync(0xffffffffu, v[0], mask);
        }
    }
    return first;
}
// Whether this lane is the one of its equals that stores them: the bits that sum_over_lanes went through with a single value left are zero.
template <int NV, int LANES, int UNIT>
__device__ __forceinline__ bool first_of_equals(int lane)
{
    return NV >= LANES || (lane & ((LANES / NV - 1) * UNIT)) == 0;
}

__host__ __device__ constexpr int round4(int n) { return (n + 3) / 4 * 4; }

// Floats of one block of sums by channel: [D][NQ] for dA, [2][D] for dDskip and ddelta_bias, rounded so that the next begins on 16 bytes.
__host__ __device__ inline long long channel_floats(int D, int NQ) { return (long long)D * NQ + (2LL * D + 3) / 4 * 4; }

// Lanes that hold a channel's N states.
inline int lanes_for(int N)
{
    int nl = 1;
    while (nl * kSpt < N) nl *= 2;
    return nl;
}

// Joins the segments of sequences that were walked from zero: forward, h_in of a segment from the one before it,
//   H <- exp(A sum s) H + local,
// and the same from the last segment to the first for the gradients.  `local` [B][segs][D][NQ] is replaced by what each segment begins from.
template <bool REVERSE>
__global__ void __launch_bounds__(256) scan_join_kernel(float* local, const float* __restrict__ steps, const float* __restrict__ A,
                                                        const float* __restrict__ first, float* last, int B, int segs, int D, int N)
{
    ptx::grid_dep_wait();
    const int NQ = round4(N);
    const long long id = (long long)blockIdx.x * 256 + threadIdx.x;
    const int n = (int)(id % NQ);
    const long long bd = id / NQ;
    const int d = (int)(bd % D);
    const long long b = bd / D;
    if (b >= B) return;
    const bool real = n < N;
    const float a2 = real ? A[(size_t)d * N + n] * kLog2e : 0.f;
    float H = first && real ? first[((size_t)b * D + d) * N + n] : 0.f;
    for (int i = 0; i < segs; ++i) {
        const int seg = REVERSE ? segs - 1 - i : i;
        float* p = local + (((size_t)b * segs + seg) * D + d) * NQ + n;
        const float l = *p;
        *p = H;
        H = fmaf(ex2(a2 * steps[((size_t)b * segs + seg) * D + d]), H, l);
    }
    if (last && real) last[((size_t)b * D + d) * N + n] = H;
}

}  // namespace conv2d_b200
