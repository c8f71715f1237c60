// What the operators along a sequence share: element types, vector loads and stores, activations.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "common.cuh"
#include "ptx.cuh"
#include "sequence_b200.h"

namespace conv2d_b200 {

using bf16 = __nv_bfloat16;
using fp16 = __half;

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(bf16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_float(fp16 v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ bf16 from_float<bf16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ fp16 from_float<fp16>(float v) { return __float2half_rn(v); }

// V adjacent elements as they lie in memory, moved by one access (two for eight fp32).
template <typename T, int V>
struct alignas(sizeof(T) * V > 16 ? 16 : sizeof(T) * V) Pack { T e[V]; };

template <typename T, int V> __device__ __forceinline__ Pack<T, V> load_pack(const T* p) { return *reinterpret_cast<const Pack<T, V>*>(p); }
template <typename T, int V> __device__ __forceinline__ void store_pack(T* p, const Pack<T, V>& v) { *reinterpret_cast<Pack<T, V>*>(p) = v; }
template <typename T, int V> __device__ __forceinline__ Pack<T, V> zero_pack()
{
    Pack<T, V> z;
#pragma unroll
    for (int i = 0; i < V; ++i) z.e[i] = from_float<T>(0.f);
    return z;
}
__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }
__device__ __forceinline__ float ex2(float v)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
__device__ __forceinline__ float rcp(float v)
{
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.69314718055994531f;

// 1 / (1 + e^-v) from the hardware's exponential and reciprocal: a few 2^-23 relative for |v| < 10, |v| 2^-23 beyond.  Two at a time, as everything
// here: the packed operations of the FMA pipe take one issue slot for two.
__device__ __forceinline__ float2 sigmoid(float2 v)
{
    const float2 t = __fmul2_rn(v, both(-kLog2e));
    const float2 d = __fadd2_rn(make_float2(ex2(t.x), ex2(t.y)), both(1.f));
    return make_float2(rcp(d.x), rcp(d.y));
}
__device__ __forceinline__ float sigmoid(float v) { return rcp(1.f + ex2(-kLog2e * v)); }

// The normal distribution function, (1 + erf(v / sqrt 2)) / 2, and e = e^(-v^2/2).  From the tail, so that its digits are kept where it is small (1 + erf
// would cancel): for a = |v| it is e t P(t), t = 1 / (1 + 0.27 a), and P, the scaled tail over t, is smooth in t as far as t = 0, where it is
// 0.27 / sqrt(2 pi): a polynomial of degree 8 that interpolates it at Chebyshev nodes of 0 <= a <= 14 (2.9e-8 of its value; 6 units of 2^-24 with its
// roundings).  Two special-function operations, as many as SiLU takes; CUDA's complementary error function instead takes twice as long
// (8 x 4096 x 512 in fp16, group norm with GELU: 65 us, 35 so) and costs the kernels, which hold every activation, registers that the others miss.
__device__ __forceinline__ float2 normal_cdf(float2 v, float2& e)
{
    const float2 q = __fmul2_rn(__fmul2_rn(v, v), both(-0.5f * kLog2e));
    e = make_float2(ex2(q.x), ex2(q.y));
    const float2 d = __ffma2_rn(make_float2(fabsf(v.x), fabsf(v.y)), both(0.27f), both(1.f)), t = make_float2(rcp(d.x), rcp(d.y));
    constexpr float c[9] = {0.10772209614515305f, 0.10751860588788986f, 0.10198036581277847f, 0.0714060589671135f, 0.10927720367908478f, -0.07121391594409943f,
                            0.17144468426704407f, -0.12724211812019348f, 0.029107028618454933f};
    float2 p = both(c[8]);
#pragma unroll
    for (int i = 7; i >= 0; --i) p = __ffma2_rn(p, t, both(c[i]));
    p = __fmul2_rn(__fmul2_rn(p, t), e);
    const float2 r = __ffma2_rn(p, both(-1.f), both(1.f));
    return make_float2(v.x < 0.f ? p.x : r.x, v.y < 0.f ? p.y : r.y);
}

// v <- act(v) for N values.  The activation is the same for a whole launch, a uniform branch; it is taken once for many values, since a branch for
// each would keep their operations apart (group norm of 8 x 4096 x 512 in fp16: 49 us so).
template <int N>
__device__ __forceinline__ void activate(float (&v)[N], int act)
{
    if (act == CONV2D_ACT_SILU) {
#pragma unroll
        for (int i = 0; i + 1 < N; i += 2) {
            const float2 x = make_float2(v[i], v[i + 1]), y = __fmul2_rn(x, sigmoid(x));
            v[i] = y.x, v[i + 1] = y.y;
        }
        if (N % 2) v[N - 1] *= sigmoid(v[N - 1]);
    } else if (act == CONV2D_ACT_RELU) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = v[i] < 0.f ? 0.f : v[i];      // (NaN stays NaN)
    } else if (act == CONV2D_ACT_GELU) {
#pragma unroll
        for (int i = 0; i + 1 < N; i += 2) {
            float2 e;
            const float2 x = make_float2(v[i], v[i + 1]), y = __fmul2_rn(x, normal_cdf(x, e));
            v[i] = y.x, v[i + 1] = y.y;
        }
        if (N % 2) {
            float2 e;
            v[N - 1] *= normal_cdf(both(v[N - 1]), e).x;
        }
    }
}
// g <- g act'(v)
template <int N>
__device__ __forceinline__ void times_slope(float (&g)[N], const float (&v)[N], int act)
{
    if (act == CONV2D_ACT_SILU) {
#pragma unroll
        for (int i = 0; i + 1 < N; i += 2) {
            // s (1 + v (1 - s)) = s + v s (1 - s)
            const float2 x = make_float2(v[i], v[i + 1]), s = sigmoid(x), r = __ffma2_rn(s, both(-1.f), both(1.f));
            const float2 y = __fmul2_rn(make_float2(g[i], g[i + 1]), __fmul2_rn(s, __ffma2_rn(x, r, both(1.f))));
            g[i] = y.x, g[i + 1] = y.y;
        }
        if (N % 2) {
            const float s = sigmoid(v[N - 1]);
            g[N - 1] *= s * fmaf(v[N - 1], 1.f - s, 1.f);
        }
    } else if (act == CONV2D_ACT_RELU) {
#pragma unroll
        for (int i = 0; i < N; ++i) g[i] = v[i] > 0.f ? g[i] : (v[i] <= 0.f ? 0.f : g[i] * v[i]);
    } else if (act == CONV2D_ACT_GELU) {
        constexpr float k = 0.39894228040143268f;            // 1 / sqrt(2 pi)
#pragma unroll
        for (int i = 0; i + 1 < N; i += 2) {
            float2 e;
            const float2 x = make_float2(v[i], v[i + 1]), f = normal_cdf(x, e);
            const float2 y = __fmul2_rn(make_float2(g[i], g[i + 1]), __ffma2_rn(__fmul2_rn(x, both(k)), e, f));
            g[i] = y.x, g[i + 1] = y.y;
        }
        if (N % 2) {
            float2 e;
            const float f = normal_cdf(both(v[N - 1]), e).x;
            g[N - 1] *= fmaf(v[N - 1] * k, e.x, f);
        }
    }
}

// Asynchronous copy of BYTES (4, 8 or 16) into shared memory; zeros where `real` is false (the address is not read then).
template <int BYTES>
__device__ __forceinline__ void copy_async(void* to, const void* from, bool real = true)
{
    const uint32_t dst = (uint32_t)__cvta_generic_to_shared(to);
    if (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(from), "r"(real ? 16 : 0) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(dst), "l"(from), "n"(BYTES), "r"(real ? BYTES : 0) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// Waits until all but the last PENDING groups of this thread's copies have arrived.
template <int PENDING> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(PENDING) : "memory"); }


// A thread's ring of RING groups of GROUP rows of one tensor in shared memory, by asynchronous copies: its packs of V elements,
// V * sizeof(T) >= 4 bytes.  Narrower ones are loaded when they are needed.
template <typename T, int V, int THREADS, int GROUP, int RING>
struct RowRing {
    static constexpr int bytes = V * (int)sizeof(T);
    static constexpr bool async = bytes >= 4;
    static constexpr size_t smem = async ? (size_t)RING * GROUP * THREADS * bytes : 0;
    unsigned char* mine;
    const T* p;                         // row 0, this thread's channels
    long long ld;
    // copies of rows t .. t + GROUP - 1, those from `live` on as zeros
    __device__ void issue(int q, int t, int live) const
    {
        if (!async) return;
        const T* from = p + (long long)t * ld;
        unsigned char* to = mine + (q & (RING - 1)) * (GROUP * THREADS * bytes);
        if (t + GROUP <= live) {
#pragma unroll
            for (int j = 0; j < GROUP; ++j, from += ld) copy_async<async ? bytes : 4>(to + j * (THREADS * bytes), from, true);
        } else {
#pragma unroll
            for (int j = 0; j < GROUP; ++j, from += ld) copy_async<async ? bytes : 4>(to + j * (THREADS * bytes), t + j < live ? from : p, t + j < live);
        }
    }
    __device__ Pack<T, V> get(int q, int t, int j, int live) const
    {
        if (async) return *reinterpret_cast<const Pack<T, V>*>(mine + (q & (RING - 1)) * (GROUP * THREADS * bytes) + j * (THREADS * bytes));
        return t + j < live ? load_pack<T, V>(p + (t + j) * ld) : zero_pack<T, V>();
    }
};

// Pairs of channels (one channel and zero for V = 1).
template <int V> constexpr int kPairs = (V + 1) / 2;
__device__ __forceinline__ float2 to_pair(uint32_t bits, bf16) { return make_float2(__uint_as_float(bits << 16), __uint_as_float(bits & 0xffff0000u)); }
__device__ __forceinline__ float2 to_pair(uint32_t bits, fp16) { return __half22float2(*reinterpret_cast<const __half2*>(&bits)); }
__device__ __forceinline__ uint32_t from_pair(float2 f, bf16)
{
    const __nv_bfloat162 h = __floats2bfloat162_rn(f.x, f.y);
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t from_pair(float2 f, fp16)
{
    const __half2 h = __floats2half2_rn(f.x, f.y);
    return *reinterpret_cast<const uint32_t*>(&h);
}
template <typename T, int V>
__device__ __forceinline__ void pairs(const Pack<T, V>& p, float2 (&f)[kPairs<V>])
{
    if constexpr (sizeof(T) == 2 && V % 2 == 0) {
#pragma unroll
        for (int i = 0; i < V / 2; ++i) f[i] = to_pair(reinterpret_cast<const uint32_t*>(&p)[i], T());
    } else {
#pragma unroll
        for (int i = 0; i < kPairs<V>; ++i) f[i] = make_float2(to_float(p.e[2 * i]), V > 1 ? to_float(p.e[V > 1 ? 2 * i + 1 : 0]) : 0.f);
    }
}
template <typename T, int V>
__device__ __forceinline__ Pack<T, V> pack_of(const float2 (&f)[kPairs<V>])
{
    Pack<T, V> p;
    if constexpr (sizeof(T) == 2 && V % 2 == 0) {
#pragma unroll
        for (int i = 0; i < V / 2; ++i) reinterpret_cast<uint32_t*>(&p)[i] = from_pair(f[i], T());
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) p.e[i] = from_float<T>(i % 2 ? f[i / 2].y : f[i / 2].x);
    }
    return p;
}

// The same as arrays.
template <typename T, int V> __device__ __forceinline__ void unpack(const Pack<T, V>& p, float (&f)[V])
{
    float2 q[kPairs<V>];
    pairs<T, V>(p, q);
#pragma unroll
    for (int i = 0; i < V; ++i) f[i] = i % 2 ? q[i / 2].y : q[i / 2].x;
}
template <typename T, int V> __device__ __forceinline__ Pack<T, V> pack(const float (&f)[V])
{
    float2 q[kPairs<V>];
#pragma unroll
    for (int i = 0; i < kPairs<V>; ++i) q[i] = make_float2(f[2 * i], V > 1 ? f[V > 1 ? 2 * i + 1 : 0] : 0.f);
    return pack_of<T, V>(q);
}

// Groups of rows all of which are there, and others: two versions of a loop's body, the first without checks.
struct Whole { static constexpr bool value = true; };
struct Cut { static constexpr bool value = false; };

// Rows of sequence b that hold tokens.
__device__ __forceinline__ int sequence_length(const int* lengths, int b, int L)
{
    if (!lengths) return L;
    const int n = lengths[b];
    return n < 0 ? 0 : (n > L ? L : n);
}

inline int element_size(conv2d_operand_t type) { return type == CONV2D_OPERAND_FP32 ? 4 : 2; }

// Whether rows that begin at p and lie ld elements apart can be moved in units of `bytes`.
inline bool rows_aligned(const void* p, long long ld, int esize, int bytes)
{
    return !p || (reinterpret_cast<uintptr_t>(p) % bytes == 0 && (ld * esize) % bytes == 0);
}

inline unsigned ceil_div_u(long long a, long long b) { return (unsigned)((a + b - 1) / b); }

// Sequences of one launch whose grid has `blocks` blocks for each: a grid holds at most `most` blocks.
inline int sequences_of_launch(long long blocks, long long most, int B)
{
    const long long forced = env_int("CONV2D_B200_SEQ_GRID", 0), n = (forced > 0 ? forced : most) / blocks;
    return n < 1 ? 1 : n < B ? (int)n : B;
}

// Column sums of partial sums [parts][cols], `ld` floats apart, added in a fixed order: 32 columns by 8 shares of the parts a block;
// `store` takes them.
template <typename Store>
__global__ void __launch_bounds__(256) column_sums_kernel(const float* __restrict__ in, long long parts, long long cols, long long ld, Store store)
{
    ptx::grid_dep_wait();
    __shared__ float sums[8][32];
    const long long col = (long long)blockIdx.x * 32 + threadIdx.x;
    float s = 0.f;
    if (col < cols) {
#pragma unroll 4
        for (long long p = threadIdx.y; p < parts; p += 8) s += in[p * ld + col];
    }
    sums[threadIdx.y][threadIdx.x] = s;
    __syncthreads();
    if (threadIdx.y || col >= cols) return;
    s = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) s += sums[j][threadIdx.x];
    store(col, s);
}
template <typename Store>
conv2d_status_t launch_column_sums(const float* in, long long parts, long long cols, long long ld, Store store, cudaStream_t stream)
{
    if (launch_pdl(column_sums_kernel<Store>, dim3(ceil_div_u(cols, 32)), dim3(32, 8), 0, stream, in, parts, cols, ld, store) != cudaSuccess)
        return CONV2D_ERR_CUDA;
    count_launch();
    return CONV2D_OK;
}

// Arguments of the launchers, as the entry points check them.
struct ConvSeq {
    const void *x, *w, *bias, *state_in, *dy, *dstate_out;
    void *y, *state_out, *dx, *dstate_in;
    float *dw, *dbias;
    const int* lengths;
    int B, L, D, K;
    long long ldx, ldy, lddy, lddx;
    conv2d_activation_t act;
    float* partials;
};
conv2d_status_t launch_conv1d_fwd(const ConvSeq& a, conv2d_operand_t type, cudaStream_t stream);
conv2d_status_t launch_conv1d_bwd(const ConvSeq& a, conv2d_operand_t type, cudaStream_t stream);
size_t conv1d_bwd_workspace_bytes(int B, int L, int D, int K);

struct ScanSeq {
    const void *u, *delta, *Bm, *Cm, *z, *dy;
    const float *A, *Dskip, *delta_bias, *state_in, *states_in, *dstate_out;
    const int* lengths;
    void *y, *du, *ddelta, *dB, *dC, *dz;
    float *state_out, *states, *dA, *dD, *ddelta_bias, *dstate_in;
    int B, L, D, N, G;
    long long ldu, lddelta, ldB, ldC, ldz, ldy, lddy, lddu, ldddelta, lddB, lddC, lddz;
    bool softplus;
    float* ws;
};
conv2d_status_t launch_scan_fwd(const ScanSeq& a, conv2d_operand_t type, cudaStream_t stream);
conv2d_status_t launch_scan_bwd(const ScanSeq& a, conv2d_operand_t type, cudaStream_t stream);
conv2d_status_t launch_scan_step(const ScanSeq& a, conv2d_operand_t type, cudaStream_t stream);
size_t scan_states_bytes(int B, int L, int D, int N);
size_t scan_fwd_workspace_bytes(int B, int L, int D, int N, int G);
size_t scan_bwd_workspace_bytes(int B, int L, int D, int N, int G);

struct NormSeq {
    const void *x, *dy;
    const float *gamma, *beta;
    void *y, *dx;
    float *mean, *rstd, *dgamma, *dbeta;
    int N, S, C, G;
    long long ldx, ldy, lddy, lddx;
    float eps;
    conv2d_activation_t act;
    float* ws;
};
conv2d_status_t launch_norm_fwd(const NormSeq& a, conv2d_operand_t type, cudaStream_t stream);
conv2d_status_t launch_norm_bwd(const NormSeq& a, conv2d_operand_t type, cudaStream_t stream);
size_t norm_fwd_workspace_bytes(int N, int S, int C, int G);
size_t norm_bwd_workspace_bytes(int N, int S, int C, int G);

}  // namespace conv2d_b200
