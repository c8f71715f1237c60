// RMS norm of rows, or of the heads of a row: with the residual's addition, a gate, an output in 8 bits; backward.
#include <cuda_fp8.h>

#include "rms_common.cuh"

namespace conv2d_b200 {
namespace {

constexpr int kMostThreads = 512, kMostWarps = kMostThreads / 32;  // of a row, and of a block: 128 registers each

// A row lies in the registers of blockDim.x threads (whole warps), NP packs of V elements each, in places threadIdx.x + j * blockDim.x; blockDim.y rows a block.
// What is summed over (a group), or shares a scale (a block of columns), is a run of packs:
enum { kRow = 0, kLanes = 1, kShared = 2 };
struct Runs {
    int packs, count, how, lanes; // packs of a run, runs of a row; over the row's threads, over `lanes` = 2^n adjacent lanes, or through shared memory
};
// The pack in place u, `packs` if there is none: groups of up to 32 packs are spread to 2^n lanes each, so that none lies in two warps.
__device__ __forceinline__ int pack_of_place(int u, const Runs& groups, int packs)
{
    if (groups.lanes == groups.packs) return u < packs ? u : packs;
    const int run = u / groups.lanes, at = u % groups.lanes;
    return at < groups.packs && run < groups.count ? run * groups.packs + at : packs;
}

struct Sum { static __device__ float of(float a, float b) { return a + b; } };
struct Max { static __device__ float of(float a, float b) { return fmaxf(a, b); } };

// The sum or the largest of 32 lanes' numbers (none below zero there, so that their bits are in order).
__device__ __forceinline__ float over_lanes(float v, Sum)
{
#pragma unroll
    for (int d = 1; d < 32; d *= 2) v += __shfl_xor_sync(0xffffffffu, v, d);
    return v;
}
__device__ __forceinline__ float over_lanes(float v, Max) { return __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(v))); }

// p[j], a value of each of this thread's packs (at[j], zero where there is none), becomes that of the pack's run.  All threads of the block come here.
// `turn` alternates between the two halves of the memory that whole rows' warps meet in: a half is written again after the other's barrier, so one is enough.
// What other runs meet in lies behind it.
template <typename Op, int HOW, int NP>
__device__ __forceinline__ void reduce_runs(float (&p)[NP], const int (&at)[NP], const Runs& r, int packs, float* shared, int& turn)
{
    const int tx = threadIdx.x, lane = tx & 31, warp = tx >> 5, warps = blockDim.x >> 5;
    const int how = HOW < 0 ? r.how : HOW;
    if (how == kLanes) {
#pragma unroll
        for (int j = 0; j < NP; ++j)
            for (int d = 1; d < r.lanes; d *= 2) p[j] = Op::of(p[j], __shfl_xor_sync(0xffffffffu, p[j], d));
    } else if (how == kRow) {
        float s = p[0];
#pragma unroll
        for (int j = 1; j < NP; ++j) s = Op::of(s, p[j]);
        s = over_lanes(s, Op());
        if (warps > 1) {
            float* mine = shared + turn + threadIdx.y * kMostWarps;
            turn ^= blockDim.y * kMostWarps;
            if (lane == 0) mine[warp] = s;
            __syncthreads();
            s = mine[0];
#pragma unroll
            for (int w = 1; w < kMostWarps; ++w)
                if (w < warps) s = Op::of(s, mine[w]);
        }
#pragma unroll
        for (int j = 0; j < NP; ++j) p[j] = s;
    } else {
        float *mine = shared + blockDim.y * 2 * kMostWarps + threadIdx.y * (packs + r.count), *runs = mine + packs;
#pragma unroll
        for (int j = 0; j < NP; ++j)
            if (at[j] < packs) mine[at[j]] = p[j];
        __syncthreads();
        for (int i = warp; i < r.count; i += warps) {
            const int end = min((i + 1) * r.packs, packs);
            float s = 0.f;
            for (int k = i * r.packs + lane; k < end; k += 32) s = Op::of(s, mine[k]);
#pragma unroll
            for (int d = 1; d < 32; d *= 2) s = Op::of(s, __shfl_xor_sync(0xffffffffu, s, d));
            if (lane == 0) runs[i] = s;
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < NP; ++j)
            if (at[j] < packs) p[j] = runs[at[j] / r.packs];
        __syncthreads();
    }
}

template <int V>
__device__ __forceinline__ void load_gamma(const float* gamma, int col, float (&f)[V])
{
    if (!gamma) {
#pragma unroll
        for (int e = 0; e < V; ++e) f[e] = 1.f;
    } else if (V % 4 == 0 && reinterpret_cast<uintptr_t>(gamma) % 16 == 0) {
#pragma unroll
        for (int e = 0; e + 3 < V; e += 4) {
            const float4 q = *reinterpret_cast<const float4*>(gamma + col + e);
            f[e] = q.x, f[e + 1] = q.y, f[e + 2] = q.z, f[e + 3] = q.w;
        }
    } else {
#pragma unroll
        for (int e = 0; e < V; ++e) f[e] = gamma[col + e];
    }
}

// Eight-bit codes of V numbers, to nearest.
template <int V>
__device__ __forceinline__ void store_codes(unsigned char* to, const float (&f)[V])
{
    Pack<unsigned char, V> p;
    if constexpr (V % 2 == 0) {
#pragma unroll
        for (int e = 0; e < V; e += 2) {
            const __nv_fp8x2_storage_t c = __nv_cvt_float2_to_fp8x2(make_float2(f[e], f[e + 1]), __NV_SATFINITE, __NV_E4M3);
            p.e[e] = (unsigned char)(c & 0xff), p.e[e + 1] = (unsigned char)(c >> 8);
        }
    } else {
        p.e[0] = __nv_cvt_float_to_fp8(f[0], __NV_SATFINITE, __NV_E4M3);
    }
    store_pack<unsigned char, V>(to, p);
}

// Places of a thread at most, for packs of V elements: 16384 elements in 512 threads.
constexpr int most_places(int v) { return v > 2 ? 8 : v > 1 ? 16 : 32; }

// Arithmetic of a pack's numbers, two at a time: these kernels are bound by what they issue next to what they move.
template <int V> __device__ __forceinline__ void add(float (&a)[V], const float (&b)[V])
{
#pragma unroll
    for (int e = 0; e + 1 < V; e += 2) {
        const float2 r = __fadd2_rn(make_float2(a[e], a[e + 1]), make_float2(b[e], b[e + 1]));
        a[e] = r.x, a[e + 1] = r.y;
    }
    if (V % 2) a[V - 1] += b[V - 1];
}
template <int V> __device__ __forceinline__ void times(float (&a)[V], const float (&b)[V])
{
#pragma unroll
    for (int e = 0; e + 1 < V; e += 2) {
        const float2 r = __fmul2_rn(make_float2(a[e], a[e + 1]), make_float2(b[e], b[e + 1]));
        a[e] = r.x, a[e + 1] = r.y;
    }
    if (V % 2) a[V - 1] *= b[V - 1];
}
template <int V> __device__ __forceinline__ void times(float (&a)[V], float b)
{
#pragma unroll
    for (int e = 0; e + 1 < V; e += 2) {
        const float2 r = __fmul2_rn(make_float2(a[e], a[e + 1]), both(b));
        a[e] = r.x, a[e + 1] = r.y;
    }
    if (V % 2) a[V - 1] *= b;
}
// c <- c + a b
template <int V> __device__ __forceinline__ void add_times(float (&c)[V], const float (&a)[V], const float (&b)[V])
{
#pragma unroll
    for (int e = 0; e + 1 < V; e += 2) {
        const float2 r = __ffma2_rn(make_float2(a[e], a[e + 1]), make_float2(b[e], b[e + 1]), make_float2(c[e], c[e + 1]));
        c[e] = r.x, c[e + 1] = r.y;
    }
    if (V % 2) c[V - 1] = fmaf(a[V - 1], b[V - 1], c[V - 1]);
}
template <int V> __device__ __forceinline__ void add_times(float (&c)[V], const float (&a)[V], float b)
{
#pragma unroll
    for (int e = 0; e + 1 < V; e += 2) {
        const float2 r = __ffma2_rn(make_float2(a[e], a[e + 1]), both(b), make_float2(c[e], c[e + 1]));
        c[e] = r.x, c[e + 1] = r.y;
    }
    if (V % 2) c[V - 1] = fmaf(a[V - 1], b, c[V - 1]);
}
template <int V> __device__ __forceinline__ float dot(const float (&a)[V], const float (&b)[V])
{
    if constexpr (V == 1) return a[0] * b[0];
    float2 s = __fmul2_rn(make_float2(a[0], a[V > 1]), make_float2(b[0], b[V > 1]));
#pragma unroll
    for (int e = 2; e + 1 < V; e += 2) s = __ffma2_rn(make_float2(a[e], a[e + 1]), make_float2(b[e], b[e + 1]), s);
    return s.x + s.y;
}
// The element of a row-major tensor: two factors of 31 bits.
__device__ __forceinline__ long long element(int row, long long ld, int col) { return (long long)row * (int)ld + col; }

// A thread's places in a ring of `stages` rows of TENSORS tensors, each for itself: it copies its own packs ahead and reads them back, with no barrier.  Without stages, where
// not even one row of a pass fits, it loads them when they are needed.
template <typename T, int V, int NP>
struct Ahead {
    static constexpr int bytes = V * (int)sizeof(T);
    static constexpr bool async = bytes >= 4;
    unsigned char* mine;
    int pitch, tensors, stages;
    __device__ Ahead(void* ring, int tensors_, int stages_) : pitch(blockDim.x * blockDim.y * bytes), tensors(tensors_), stages(async ? stages_ : 0)
    {
        mine = static_cast<unsigned char*>(ring) + (threadIdx.y * blockDim.x + threadIdx.x) * bytes;
    }
    __device__ unsigned char* slot(int stage, int tensor, int j) const { return mine + ((stage * tensors + tensor) * NP + j) * pitch; }
    // Tensor number `tensor` of a row; zeros where `there` says so.
    __device__ void fetch(int stage, int tensor, const void* from, int row, long long ld, const int (&col)[NP], const bool (&there)[NP]) const
    {
        if constexpr (async) {
#pragma unroll
            for (int j = 0; j < NP; ++j) copy_async<bytes>(slot(stage, tensor, j), static_cast<const T*>(from) + element(row, ld, col[j]), there[j]);
        }
    }
    __device__ Pack<T, V> get(int stage, int tensor, const void* from, int row, long long ld, int j, int col, bool there) const
    {
        if (async && stages) return *reinterpret_cast<const Pack<T, V>*>(slot(stage, tensor, j));
        return load_masked<T, V>(static_cast<const T*>(from) + element(row, ld, col), there);
    }
    // until the oldest of `stages` rows under way is there
    __device__ void wait() const
    {
        if (stages == 4) copies_wait<3>();
        else if (stages == 3) copies_wait<2>();
        else if (stages == 2) copies_wait<1>();
        else if (stages == 1) copies_wait<0>();
    }
};

// What a call has, as constants of its kernel: whether there is a second tensor to add (residual, dh), a gate, y and y8, and which lanes share groups and scales.  The
// branches on them and what they keep apart would be a third of all that these kernels issue, and these are bound by that (8192 x 4096 with a residual to 8 bits: 50M
// instructions and 67 us so, 36M and 48 with constants; 16384 x 2048 to 16 bits: 56 us and 41).  kAny looks at the arguments: the other
// calls (to 8 bits with a gate, of heads 61 to 66 us, of rows 68, or without a residual, 52 to 56: 8192 x 4096 of bf16), and rows too large for two packs a thread.
enum { kSecond = 1, kGate = 2, kY = 4, kY8 = 8, kGroupLanes = 16, kBlockLanes = 32, kAny = -1 };
template <int KIND> __device__ __forceinline__ bool has(int what, const void* given) { return KIND < 0 ? given != nullptr : (KIND & what) != 0; }
template <int KIND>
struct Ways { static constexpr int group = KIND < 0 ? -1 : KIND & kGroupLanes ? kLanes : kRow, block = KIND < 0 ? -1 : KIND & kBlockLanes ? kLanes : kRow; };

// A block takes rows gridDim.x * blockDim.y apart, the next ones' numbers under way while it computes.
template <typename T, int V, int NP, int KIND>
__global__ void __launch_bounds__(kMostThreads, V > 2 && NP <= 2 ? 2 : 1) rms_fwd_kernel(const RmsArgs a, Runs groups, Runs blocks, int packs, int channels, int stages, int ring)
{
    extern __shared__ float4 shared4[];
    float* shared = reinterpret_cast<float*>(shared4);
    ptx::grid_dep_wait();
    const float inverse = 1.f / channels;
    const bool second = has<KIND>(kSecond, a.residual), gated = has<KIND>(kGate, a.z), whole = has<KIND>(kY, a.y), coded = has<KIND>(kY8, a.y8);
    const int gate = second ? 2 : 1, step = gridDim.x * blockDim.y;
    const Ahead<T, V, NP> ahead(shared4 + ring, gate + (gated ? 1 : 0), stages);
    stages = ahead.stages;
    int at[NP], col[NP], group[NP], block[NP];
    float w[NP][V];
#pragma unroll
    for (int j = 0; j < NP; ++j) {
        const int p = at[j] = pack_of_place(threadIdx.x + j * blockDim.x, groups, packs);
        col[j] = p < packs ? p * V : 0;
        group[j] = a.G > 1 ? p / groups.packs : 0;
        block[j] = blocks.count > 1 ? p / blocks.packs : 0;
    }
    auto fetch = [&](int stage, int row) {
        bool there[NP];
#pragma unroll
        for (int j = 0; j < NP; ++j) there[j] = row < a.M && at[j] < packs;
        row = row < a.M ? row : 0;
        ahead.fetch(stage, 0, a.x, row, a.ldx, col, there);
        if (second) ahead.fetch(stage, 1, a.residual, row, a.ldr, col, there);
        if (gated) ahead.fetch(stage, gate, a.z, row, a.ldz, col, there);
        copies_commit();
    };
    int row = blockIdx.x * blockDim.y + threadIdx.y, stage = 0, turn = 0;
    for (int i = 0; i < stages; ++i) fetch(i, row + i * step);
#pragma unroll
    for (int j = 0; j < NP; ++j) load_gamma<V>(a.gamma, at[j] < packs ? (at[j] - group[j] * groups.packs) * V : 0, w[j]);
    for (int row0 = blockIdx.x * blockDim.y; row0 < a.M; row0 += step, row += step) {
        float f[NP][V], s[NP];
        Pack<T, V> px[NP], pr[NP], pz[NP];
        bool there[NP];
        ahead.wait();
#pragma unroll
        for (int j = 0; j < NP; ++j) {
            there[j] = row < a.M && at[j] < packs;
            px[j] = ahead.get(stage, 0, a.x, row, a.ldx, j, col[j], there[j]);
            if (second) pr[j] = ahead.get(stage, 1, a.residual, row, a.ldr, j, col[j], there[j]);
            if (gated) pz[j] = ahead.get(stage, gate, a.z, row, a.ldz, j, col[j], there[j]);
        }
#pragma unroll
        for (int j = 0; j < NP; ++j) {
            unpack<T, V>(px[j], f[j]);
            if (second) {                                  // the sum as it is stored is what is normalised, so that the backward pass sees the same
                float r[V];
                unpack<T, V>(pr[j], r);
                add<V>(f[j], r);
                const Pack<T, V> sum = pack<T, V>(f[j]);
                unpack<T, V>(sum, f[j]);
                if (there[j]) store_pack<T, V>(static_cast<T*>(a.h) + element(row, a.ldh, col[j]), sum);
            }
            float part[V];                                     // of the mean: each square by itself, since a mean does not overflow where its terms do not, but a sum of two may
#pragma unroll
            for (int e = 0; e < V; ++e) part[e] = f[j][e];
            times<V>(part, inverse);
            s[j] = dot<V>(f[j], part);
        }
        reduce_runs<Sum, Ways<KIND>::group>(s, at, groups, packs, shared, turn);
        if (stages) {
            fetch(stage, row + stages * step);
            stage = stage + 1 == stages ? 0 : stage + 1;
        }
        float most[NP];
#pragma unroll
        for (int j = 0; j < NP; ++j) {
            const float r = rsqrtf(s[j] + a.eps);
            if (a.rstd && there[j] && at[j] == group[j] * groups.packs) a.rstd[(long long)row * a.G + group[j]] = r;
            times<V>(f[j], r);
            times<V>(f[j], w[j]);
            if (gated) {
                float z[V];
                unpack<T, V>(pz[j], z);
                activate(z, CONV2D_ACT_SILU);
                times<V>(f[j], z);
            }
            if (whole && there[j]) store_pack<T, V>(static_cast<T*>(a.y) + element(row, a.ldy, col[j]), pack<T, V>(f[j]));
            most[j] = 0.f;
#pragma unroll
            for (int e = 0; e < V; ++e) most[j] = fmaxf(most[j], fabsf(f[j][e]));
            if (!there[j]) most[j] = 0.f;
        }
        if (!coded) continue;
        reduce_runs<Max, Ways<KIND>::block>(most, at, blocks, packs, shared, turn);
#pragma unroll
        for (int j = 0; j < NP; ++j) {
            if (!there[j]) continue;
            const float scale = fmaxf(most[j] / 448.f, 1.17549435e-38f);
            if (at[j] == block[j] * blocks.packs) a.scales[(long long)row * blocks.count + block[j]] = scale;
            // the quotient, put right by what it leaves: not one rounding more than a division's before the codes'.  Over an infinite scale it leaves nothing:
            // finite numbers are zero (times the scale they would be NaN), infinite ones NaN
            const float up = 1.f / scale, down = up > 0.f ? -scale : 0.f;
            float q[V];
#pragma unroll
            for (int e = 0; e < V; ++e) q[e] = f[j][e];
            times<V>(q, up);
            add_times<V>(f[j], q, down);
            add_times<V>(q, f[j], up);
            store_codes<V>(static_cast<unsigned char*>(a.y8) + element(row, a.ld8, col[j]), q);
        }
    }
}

// Backward: with n = dy gamma silu(z) and m = h r,   dx = r (n - m mean(n m)) + dh.  Rows as in the forward pass; a block keeps its sums for gamma in registers until the
// end, when they are added over its rows and groups.
template <typename T, int V, int NP, int KIND>
__global__ void __launch_bounds__(kMostThreads, 1) rms_bwd_kernel(const RmsArgs a, Runs groups, int packs, int channels, int stages, int ring)
{
    extern __shared__ float4 shared4[];
    float* shared = reinterpret_cast<float*>(shared4);
    ptx::grid_dep_wait();
    const float inverse = 1.f / channels;
    const bool second = has<KIND>(kSecond, a.dh), gated = has<KIND>(kGate, a.z);
    const int gate = second ? 3 : 2, step = gridDim.x * blockDim.y;
    const Ahead<T, V, NP> ahead(shared4 + ring, gate + (gated ? 1 : 0), stages);
    stages = ahead.stages;
    float w[NP][V], dw[NP][V], next[NP];
    int at[NP], col[NP], group[NP];
#pragma unroll
    for (int j = 0; j < NP; ++j) {
        const int p = at[j] = pack_of_place(threadIdx.x + j * blockDim.x, groups, packs);
        col[j] = p < packs ? p * V : 0;
        group[j] = a.G > 1 && p < packs ? p / groups.packs : 0;
#pragma unroll
        for (int e = 0; e < V; ++e) dw[j][e] = 0.f;
    }
    auto fetch = [&](int stage, int row) {
        bool there[NP];
#pragma unroll
        for (int j = 0; j < NP; ++j) there[j] = row < a.M && at[j] < packs;
        row = row < a.M ? row : 0;
        ahead.fetch(stage, 0, a.x, row, a.ldx, col, there);
        ahead.fetch(stage, 1, a.dy, row, a.lddy, col, there);
        if (second) ahead.fetch(stage, 2, a.dh, row, a.lddh, col, there);
        if (gated) ahead.fetch(stage, gate, a.z, row, a.ldz, col, there);
        copies_commit();
    };
    auto fetch_r = [&](int row) {
#pragma unroll
        for (int j = 0; j < NP; ++j) next[j] = load_masked<float, 1>(a.rstd_in + (long long)row * a.G + group[j], row < a.M && at[j] < packs).e[0];
    };
    int row = blockIdx.x * blockDim.y + threadIdx.y, stage = 0, turn = 0;
    for (int i = 0; i < stages; ++i) fetch(i, row + i * step);
    fetch_r(row);
#pragma unroll
    for (int j = 0; j < NP; ++j) load_gamma<V>(a.gamma, at[j] < packs ? (at[j] - group[j] * groups.packs) * V : 0, w[j]);
    for (int row0 = blockIdx.x * blockDim.y; row0 < a.M; row0 += step, row += step) {
        float m[NP][V], n[NP][V], s[NP], r[NP];
        Pack<T, V> ph[NP], py[NP], pd[NP], pz[NP];
        bool there[NP];
        ahead.wait();
#pragma unroll
        for (int j = 0; j < NP; ++j) {
            there[j] = row < a.M && at[j] < packs;
            ph[j] = ahead.get(stage, 0, a.x, row, a.ldx, j, col[j], there[j]);
            py[j] = ahead.get(stage, 1, a.dy, row, a.lddy, j, col[j], there[j]);
            if (second) pd[j] = ahead.get(stage, 2, a.dh, row, a.lddh, j, col[j], there[j]);
            if (gated) pz[j] = ahead.get(stage, gate, a.z, row, a.ldz, j, col[j], there[j]);
        }
#pragma unroll
        for (int j = 0; j < NP; ++j) {
            unpack<T, V>(ph[j], m[j]);
            unpack<T, V>(py[j], n[j]);
            r[j] = next[j];
            times<V>(m[j], r[j]);
            if (gated) {
                float z[V], dz[V];
                unpack<T, V>(pz[j], z);
#pragma unroll
                for (int e = 0; e < V; ++e) dz[e] = n[j][e];
                times<V>(dz, w[j]);
                times<V>(dz, m[j]);
                times_slope(dz, z, CONV2D_ACT_SILU);
                activate(z, CONV2D_ACT_SILU);
                times<V>(n[j], z);
                if (there[j]) store_pack<T, V>(static_cast<T*>(a.dz) + element(row, a.lddz, col[j]), pack<T, V>(dz));
            }
            add_times<V>(dw[j], n[j], m[j]);
            times<V>(n[j], w[j]);
            float part[V];                                     // (likewise)
#pragma unroll
            for (int e = 0; e < V; ++e) part[e] = m[j][e];
            times<V>(part, inverse);
            s[j] = dot<V>(n[j], part);
        }
        fetch_r(row + step);
        reduce_runs<Sum, Ways<KIND>::group>(s, at, groups, packs, shared, turn);
#pragma unroll
        for (int j = 0; j < NP; ++j) {
            add_times<V>(n[j], m[j], -s[j]);
            times<V>(n[j], r[j]);
            if (second) {
                float d[V];
                unpack<T, V>(pd[j], d);
                add<V>(n[j], d);
            }
            if (there[j]) store_pack<T, V>(static_cast<T*>(a.dx) + element(row, a.lddx, col[j]), pack<T, V>(n[j]));
        }
        if (stages) {
            fetch(stage, row + stages * step);
            stage = stage + 1 == stages ? 0 : stage + 1;
        }
    }
    if (!a.dgamma) return;
    __syncthreads();
    float* mine = shared + threadIdx.y * a.C;
#pragma unroll
    for (int j = 0; j < NP; ++j) {
        const int p = at[j];
        if (p >= packs) continue;
#pragma unroll
        for (int e = 0; e < V; ++e) mine[p * V + e] = dw[j][e];
    }
    __syncthreads();
    for (int c = threadIdx.y * blockDim.x + threadIdx.x; c < channels; c += blockDim.x * blockDim.y) {
        float s = 0.f;
        for (int i = c; i < a.C * (int)blockDim.y; i += channels) s += shared[i];
        a.ws[(size_t)blockIdx.x * channels + c] = s;
    }
}

// Sums over the blocks' parts, 32 columns by 32 shares of the parts a block.
__global__ void __launch_bounds__(1024) rms_gamma_kernel(const float* __restrict__ parts, float* __restrict__ out, int blocks, int channels)
{
    __shared__ float sums[32][33];
    ptx::grid_dep_wait();
    const int c = blockIdx.x * 32 + threadIdx.x;
    float s = 0.f;
    if (c < channels) {
#pragma unroll 8
        for (int p = threadIdx.y; p < blocks; p += 32) s += parts[(size_t)p * channels + c];
    }
    sums[threadIdx.y][threadIdx.x] = s;
    __syncthreads();
    s = sums[threadIdx.x][threadIdx.y];
#pragma unroll
    for (int d = 1; d < 32; d *= 2) s += __shfl_xor_sync(0xffffffffu, s, d);
    if (threadIdx.x == 0 && blockIdx.x * 32 + threadIdx.y < channels) out[blockIdx.x * 32 + threadIdx.y] = s;
}

// How a row's packs are spread: at least two a thread (four of one or two elements), up to 512 threads; small rows share a block of about 256.
struct RowPlan {
    int v, packs, threads, rows, np;
    Runs groups;
    RowPlan(int C, int G, int v_) : v(v_), packs(C / v_)
    {
        groups = Runs{packs / G, G, kShared, packs / G};
        if (G == 1) groups.how = kRow;
        else if (groups.packs <= 32) {
            groups.how = kLanes;
            for (groups.lanes = 1; groups.lanes < groups.packs;) groups.lanes *= 2;
        }
        spread();
        if (np > most_places(v)) {                             // (the largest rows have no room for places without a pack)
            groups.how = kShared, groups.lanes = groups.packs;
            spread();
        }
    }
    void spread()
    {
        const int places = groups.lanes * groups.count, each = v > 2 ? 2 : 4;
        threads = (places + each - 1) / each;
        threads = threads > kMostThreads ? kMostThreads : (threads + 31) / 32 * 32;
        np = (places + threads - 1) / threads;
        rows = threads >= 256 ? 1 : 256 / threads;
    }
    // runs that share a scale
    Runs blocks(int elements) const
    {
        const int n = elements / v;
        Runs r{n, (packs + n - 1) / n, kShared, n};
        if (r.count == 1) r.how = kRow;
        else if (n == groups.packs && groups.how == kLanes) return groups;
        else if (groups.lanes == groups.packs && n <= 32 && (n & (n - 1)) == 0) r.how = kLanes;
        return r;
    }
};
size_t shared_bytes(const RowPlan& p, const Runs& r) { return r.how == kLanes ? 0 : (size_t)p.rows * (2 * kMostWarps + (r.how == kShared ? p.packs + r.count : 0)) * 4; }

// Blocks of a pass with `regs` registers a thread: as many as run at once, and the rows that each has under way, up to four, in the shared memory that `used` bytes leave.
struct Spread {
    int blocks, stages;
    Spread(const RmsArgs& a, const RowPlan& p, int regs, int row_bytes, size_t used)
    {
        const int each = p.threads * p.rows * regs, resident = 65536 / each > 1 ? 65536 / each : 1;
        const long long all = ((long long)a.M + p.rows - 1) / p.rows, most = (long long)resident * sm_count();
        blocks = (int)(all < most ? all : most);
        const size_t room = 220 * 1024 / resident, left = room > used ? room - used : 0, fit = left / ((size_t)row_bytes * p.rows);
        const long long rows = (all + blocks - 1) / blocks;    // of a block
        stages = (int)(fit < 4 ? fit : 4);
        if (stages > rows) stages = (int)rows;
    }
};

template <typename T, int V, int NP, int KIND>
conv2d_status_t forward(const RmsArgs& a, const RowPlan& p, cudaStream_t stream)
{
    static SmemLimit limit;
    const Runs groups = p.groups, blocks = p.blocks(a.y8 ? a.block : a.C);
    const size_t one = shared_bytes(p, groups), two = shared_bytes(p, blocks), sums = ((one > two ? one : two) + 15) / 16 * 16;
    const int row_bytes = (1 + !!a.residual + !!a.z) * NP * p.threads * V * (int)sizeof(T);
    const Spread spread(a, p, V > 2 && NP <= 2 ? 64 : 128, row_bytes, sums);
    const size_t smem = sums + (size_t)spread.stages * row_bytes * p.rows;
    if (raise_smem_limit((const void*)rms_fwd_kernel<T, V, NP, KIND>, smem, limit) != cudaSuccess) return CONV2D_ERR_CUDA;
    if (launch_pdl(rms_fwd_kernel<T, V, NP, KIND>, dim3(spread.blocks), dim3(p.threads, p.rows), smem, stream, a, groups, blocks, p.packs, a.C / a.G, spread.stages,
                   (int)(sums / 16)) != cudaSuccess)
        return CONV2D_ERR_CUDA;
    count_launch();
    return CONV2D_OK;
}

// Most blocks of the backward pass, whose partial sums are added afterwards.
int most_bwd_blocks(int M) { return M < 4 * sm_count() ? M : 4 * sm_count(); }

template <typename T, int V, int NP, int KIND>
conv2d_status_t backward(const RmsArgs& a, const RowPlan& p, cudaStream_t stream)
{
    static SmemLimit limit;
    const Runs groups = p.groups;
    const size_t runs = shared_bytes(p, groups), dw = a.dgamma ? (size_t)p.rows * a.C * 4 : 0, sums = ((runs > dw ? runs : dw) + 15) / 16 * 16;
    const int row_bytes = (2 + !!a.dh + !!a.z) * NP * p.threads * V * (int)sizeof(T), channels = a.C / a.G;
    const Spread spread(a, p, 128, row_bytes, sums);
    const size_t smem = sums + (size_t)spread.stages * row_bytes * p.rows;
    if (raise_smem_limit((const void*)rms_bwd_kernel<T, V, NP, KIND>, smem, limit) != cudaSuccess) return CONV2D_ERR_CUDA;
    if (launch_pdl(rms_bwd_kernel<T, V, NP, KIND>, dim3(spread.blocks), dim3(p.threads, p.rows), smem, stream, a, groups, p.packs, channels, spread.stages,
                   (int)(sums / 16)) != cudaSuccess)
        return CONV2D_ERR_CUDA;
    count_launch();
    if (!a.dgamma) return CONV2D_OK;
    if (launch_pdl(rms_gamma_kernel, dim3(ceil_div_u(channels, 32)), dim3(32, 32), 0, stream, a.ws, a.dgamma, spread.blocks, channels) != cudaSuccess) return CONV2D_ERR_CUDA;
    count_launch();
    return CONV2D_OK;
}

// Whether rows can be moved in packs of V elements of which none lies in two groups or two blocks of a scale.
template <typename T>
bool packs_fit(const RmsArgs& a, int V)
{
    const int e = sizeof(T), n = V * e;
    return (a.C / a.G) % V == 0 && (!a.y8 || (a.block % V == 0 && rows_aligned(a.y8, a.ld8, 1, V))) && rows_aligned(a.x, a.ldx, e, n) && rows_aligned(a.residual, a.ldr, e, n) &&
           rows_aligned(a.z, a.ldz, e, n) && rows_aligned(a.y, a.ldy, e, n) && rows_aligned(a.h, a.ldh, e, n) && rows_aligned(a.dy, a.lddy, e, n) &&
           rows_aligned(a.dh, a.lddh, e, n) && rows_aligned(a.dx, a.lddx, e, n) && rows_aligned(a.dz, a.lddz, e, n);
}

// The kernel for what the call has, of the kinds named, or the one for any.
template <typename T, int V, int NP, int KIND, int... MORE>
conv2d_status_t forward_of(int kind, const RmsArgs& a, const RowPlan& p, cudaStream_t stream)
{
    if constexpr (KIND == kAny) return forward<T, V, NP, kAny>(a, p, stream);
    else return kind == KIND ? forward<T, V, NP, KIND>(a, p, stream) : forward_of<T, V, NP, MORE...>(kind, a, p, stream);
}
template <typename T, int V, int NP, int KIND, int... MORE>
conv2d_status_t backward_of(int kind, const RmsArgs& a, const RowPlan& p, cudaStream_t stream)
{
    if constexpr (KIND == kAny) return backward<T, V, NP, kAny>(a, p, stream);
    else return kind == KIND ? backward<T, V, NP, KIND>(a, p, stream) : backward_of<T, V, NP, MORE...>(kind, a, p, stream);
}
template <typename T, int V, int NP>
conv2d_status_t either(const RmsArgs& a, const RowPlan& p, bool bwd, cudaStream_t stream)
{
    if constexpr (V * sizeof(T) == 16 && NP <= 2) {            // kinds: the norm at a layer's entry, of its heads, at its exit but for one in 8 bits
        const Runs blocks = p.blocks(a.y8 ? a.block : a.C);
        int kind = (a.residual || a.dh ? kSecond : 0) | (a.z ? kGate : 0) | (a.y ? kY : 0) | (a.y8 ? kY8 : 0) | (p.groups.how == kLanes ? kGroupLanes : 0) |
                   (a.y8 && blocks.how == kLanes ? kBlockLanes : 0);
        if (p.groups.how == kShared || blocks.how == kShared) kind = kAny;
        if (bwd) return backward_of<T, V, NP, kSecond, 0, kGate, kGroupLanes, kGate | kGroupLanes, kAny>(kind, a, p, stream);
        return forward_of<T, V, NP, kSecond | kY, kSecond | kY8, kSecond | kY8 | kBlockLanes, kY, kGate | kY, kGroupLanes | kY, kGroupLanes | kGate | kY, kAny>(kind, a, p, stream);
    }
    return bwd ? backward<T, V, NP, kAny>(a, p, stream) : forward<T, V, NP, kAny>(a, p, stream);
}
// Packs of V elements, or the next smaller that fit.
template <typename T, int V>
conv2d_status_t rms_packed(const RmsArgs& a, bool bwd, cudaStream_t stream)
{
    if constexpr (V > 2) {
        if (packs_fit<T>(a, V)) {
            const RowPlan p(a.C, a.G, V);
            if (p.np == 1) return either<T, V, 1>(a, p, bwd, stream);
            if (p.np == 2) return either<T, V, 2>(a, p, bwd, stream);
            return p.np <= 4 ? either<T, V, 4>(a, p, bwd, stream) : either<T, V, 8>(a, p, bwd, stream);
        }
        return rms_packed<T, V / 2>(a, bwd, stream);
    } else {
        if (V == 2 && !packs_fit<T>(a, V)) return rms_packed<T, 1>(a, bwd, stream);
        const RowPlan p(a.C, a.G, V);
        if (p.np <= 4) return either<T, V, 4>(a, p, bwd, stream);
        if (p.np <= 8) return either<T, V, 8>(a, p, bwd, stream);
        if (V == 2 || p.np <= 16) return either<T, V, 16>(a, p, bwd, stream);
        return either<T, 1, 32>(a, p, bwd, stream);
    }
}

conv2d_status_t rms(const RmsArgs& a, conv2d_operand_t type, bool bwd, cudaStream_t stream)
{
    if (type == CONV2D_OPERAND_BF16) return rms_packed<bf16, 8>(a, bwd, stream);
    if (type == CONV2D_OPERAND_FP16) return rms_packed<fp16, 8>(a, bwd, stream);
    return rms_packed<float, 4>(a, bwd, stream);
}

}  // namespace

// (a row of partial sums for every block, whichever way the rows are spread)
size_t rms_bwd_workspace_bytes(int M, int C, int G) { return ((size_t)most_bwd_blocks(M) * (C / G) * 4 + 15) / 16 * 16; }
conv2d_status_t launch_rms_fwd(const RmsArgs& a, conv2d_operand_t type, cudaStream_t stream) { return rms(a, type, false, stream); }
conv2d_status_t launch_rms_bwd(const RmsArgs& a, conv2d_operand_t type, cudaStream_t stream) { return rms(a, type, true, stream); }

}  // namespace conv2d_b200
