// What the forward and the backward scan share: how a warp holds states, sums over lanes, step sizes, segments of time.
//
// A thread holds SPT adjacent states of one channel (eight or four).  A warp takes CL = 32 / NL adjacent channels: lane l the
// channel l % CL and the states from SPT * (l / CL) on, so that NL lanes hold a channel's states (SPT * NL, the power of two that covers N), B and C are the same
// for CL adjacent lanes (one access of 16 bytes costs 2.4 cycles of shared memory then, 4 where neighbours differ), and the states
// never leave the registers.
#pragma once

#include <type_traits>

#include "seq_common.cuh"

namespace conv2d_b200 {

constexpr int kCheckpointRows = 16;     // the forward pass keeps the state before every 16th row for the backward pass

// A2 = A log2(e).  What lies below fp32 (A of -infinity: a state that forgets everything) is taken as its lowest value, so that a step of zero, as rows of
// padding have it, is a decay of one there too.
__device__ __forceinline__ float decay_rate(float A)
{
    const float v = A * kLog2e;
    return v < -3.4e38f ? -3.4e38f : v;
}

// Decays exp(s A) = 2^(s A2) of two states.  The hardware's 2^x is low by 1.2e-8 of itself on average for x in -[0.001, 0.01], 0.6e-8 and 2.2e-8 a factor
// of ten to either side (measured over 2^20 values of each range), which states that remember a thousand rows would add up; the argument takes
// that much more.  2^kExpBias is 1: a step of zero leaves the state as it is.
constexpr float kExpBias = 1.2e-8f * kLog2e;
__device__ __forceinline__ float2 decay(float2 s, float2 A2)
{
    const float2 e = __ffma2_rn(s, A2, both(kExpBias));
    return make_float2(ex2(e.x), ex2(e.y));
}
// The same where it has been taken before: not to be kept in a register from there.
__device__ __forceinline__ float2 decay_again(float2 s, float2 A2)
{
    float2 e = __ffma2_rn(s, A2, both(kExpBias));
    asm volatile("ex2.approx.ftz.f32 %0, %0;" : "+f"(e.x));
    asm volatile("ex2.approx.ftz.f32 %0, %0;" : "+f"(e.y));
    return e;
}

// log(1 + e^v) = max(v, 0) + log(1 + w), w = e^-|v| in (0, 1], and log(1 + w) / w as a polynomial (interpolated at Chebyshev nodes; 3e-8, 2e-7
// with its roundings), so that small steps keep their digits and one special-function operation does.
__device__ __forceinline__ float2 softplus(float2 v)
{
    const float2 w = make_float2(ex2(-kLog2e * fabsf(v.x)), ex2(-kLog2e * fabsf(v.y)));
    constexpr float c[9] = {1.0f, -0.49999502301216125f, 0.33319270610809326f, -0.24844369292259216f, 0.19111430644989014f,
                            -0.13674770295619965f, 0.07836166769266129f, -0.02958850748836994f, 0.005253457929939032f};
    float2 p = both(c[8]);
#pragma unroll
    for (int i = 7; i >= 0; --i) p = __ffma2_rn(p, w, both(c[i]));
    return __ffma2_rn(p, w, make_float2(v.x > 0.f ? v.x : 0.f, v.y > 0.f ? v.y : 0.f));
}
__device__ __forceinline__ float softplus(float v) { return softplus(both(v)).x; }

// Sums of NV values over the LANES lanes that differ in the bits LANES/2 * UNIT .. UNIT of the lane index.  While more than one value is left a lane hands half of
// them over and goes on with the sums of the other half, so that NV - 1 exchanges do for log2(LANES) * NV; at the end v[0 .. left) hold the
// values first .. first + left, left = max(1, NV / LANES), in every lane whose further bits are anything.
// A stage of it: of log2(LANES), further ones do nothing.  (`stage` is known when compiled)
template <int NV, int LANES, int UNIT>
__device__ __forceinline__ void sum_stage(float (&v)[NV], int lane, int stage)
{
    const int m = LANES >> (stage + 1), cnt = NV >> stage;
    if (m == 0) return;
    const int mask = m * UNIT;
    const bool upper = (lane & mask) != 0;
    if (cnt > 1) {
#pragma unroll
        for (int i = 0; i < NV / 2; ++i) {
            if (i < cnt / 2) {
                const float send = upper ? v[i] : v[i + cnt / 2], keep = upper ? v[i + cnt / 2] : v[i];
                v[i] = keep + __shfl_xor_sync(0xffffffffu, send, mask);
            }
        }
    } else {
        v[0] += __shfl_xor_sync(0xffffffffu, v[0], mask);
    }
}
template <int NV, int LANES, int UNIT>
__device__ __forceinline__ void sum_over_lanes(float (&v)[NV], int lane)
{
#pragma unroll
    for (int stage = 0; LANES >> (stage + 1); ++stage) sum_stage<NV, LANES, UNIT>(v, lane, stage);
}
template <int NV, int LANES, int UNIT>
__device__ __forceinline__ int first_value(int lane)
{
    int first = 0;
#pragma unroll
    for (int stage = 0; LANES >> (stage + 1); ++stage)
        if (NV >> stage > 1 && (lane & (LANES >> (stage + 1)) * UNIT)) first += NV >> (stage + 1);
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

// Lanes that hold a channel's N states, `spt` each.
inline int lanes_for(int N, int spt)
{
    int nl = 1;
    while (nl * spt < N) nl *= 2;
    return nl;
}

// The largest unit, up to 16 bytes, in which rows of `width` elements that begin at p, ld elements apart, can be copied.
inline int copy_unit(const void* p, long long ld, long long width, int esize)
{
    int unit = 16;
    while (unit > esize && !(rows_aligned(p, ld, esize, unit) && width * esize % unit == 0)) unit /= 2;
    return unit;
}

// Copies a tile of ROWS rows of COLS elements, `ld` elements apart, into shared memory, where they lie one behind the other: rows from `live_rows` on
// and columns from `live_cols` on as zeros.  Units of 4 bytes and more go by asynchronous copies, which the caller commits and waits for.
template <int ROWS, int COLS, int UNIT, int THREADS, typename T>
__device__ __forceinline__ void copy_tile_by(T* dst, const T* src, int ld, int live_rows, int live_cols, int tid)
{
    constexpr int E = UNIT / (int)sizeof(T), PER_ROW = COLS / E, COUNT = ROWS * PER_ROW;
#pragma unroll
    for (int k = 0; k < (COUNT + THREADS - 1) / THREADS; ++k) {
        const int i = tid + k * THREADS;
        if (COUNT % THREADS != 0 && i >= COUNT) break;
        const int r = i / PER_ROW, c = i % PER_ROW * E;
        const bool real = r < live_rows && c < live_cols;
        const T* from = src + (real ? (long long)r * ld + c : 0);
        if constexpr (UNIT >= 4) copy_async<UNIT>(dst + i * E, from, real);
        else dst[i] = real ? *from : from_float<T>(0.f);
    }
}
template <int ROWS, int COLS, int THREADS, typename T>
__device__ __forceinline__ void copy_tile(T* dst, const T* src, int ld, int live_rows, int live_cols, int unit, int tid)
{
    constexpr int BYTES = COLS * (int)sizeof(T), NARROW = (int)sizeof(T);
    if (BYTES >= 16 && unit == 16) copy_tile_by<ROWS, COLS, BYTES >= 16 ? 16 : NARROW, THREADS>(dst, src, ld, live_rows, live_cols, tid);
    else if (BYTES >= 8 && unit >= 8) copy_tile_by<ROWS, COLS, BYTES >= 8 ? 8 : NARROW, THREADS>(dst, src, ld, live_rows, live_cols, tid);
    else if (unit >= 4) copy_tile_by<ROWS, COLS, 4, THREADS>(dst, src, ld, live_rows, live_cols, tid);
    else copy_tile_by<ROWS, COLS, NARROW, THREADS>(dst, src, ld, live_rows, live_cols, tid);
}
// Barrier among the THREADS helping threads of a block (the block's own barrier is number 0).
template <int THREADS> __device__ __forceinline__ void helpers_sync() { asm volatile("bar.sync 1, %0;" ::"n"(THREADS) : "memory"); }

// Four adjacent elements in shared memory.
template <typename T> __device__ __forceinline__ void load4(const T* p, float (&v)[4]) { unpack(load_pack<T, 4>(p), v); }

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
    const float a2 = real ? decay_rate(A[(size_t)d * N + n]) : 0.f;
    float H = first && real ? first[((size_t)b * D + d) * N + n] : 0.f;
    constexpr int AHEAD = 8;                                  // segments whose loads are under way together
    for (int i0 = 0; i0 < segs; i0 += AHEAD) {
        float l[AHEAD], s[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            const int i = min(i0 + j, segs - 1);
            const size_t at = ((size_t)b * segs + (REVERSE ? segs - 1 - i : i)) * D + d;
            l[j] = local[at * NQ + n], s[j] = steps[at];
        }
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            const int i = i0 + j;
            if (i >= segs) break;
            local[(((size_t)b * segs + (REVERSE ? segs - 1 - i : i)) * D + d) * NQ + n] = H;
            H = fmaf(ex2(a2 * s[j]), H, l[j]);
        }
    }
    if (last && real) last[((size_t)b * D + d) * N + n] = H;
}

}  // namespace conv2d_b200
