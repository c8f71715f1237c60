// RMS norm of rows, or of the heads of a row: with the residual's addition, a gate, an output in 8 bits; backward.
#include <cuda_fp8.h>

#include "rms_common.cuh"

namespace conv2d_b200 {
namespace {

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

// p[j], a value of each of this thread's packs (at[j], zero where there is none), becomes that of the pack's run.  All threads of the block come here.
template <typename Op, int NP>
__device__ __forceinline__ void reduce_runs(float (&p)[NP], const int (&at)[NP], const Runs& r, int packs, float* shared)
{
    const int tx = threadIdx.x, lane = tx & 31, warp = tx >> 5, warps = blockDim.x >> 5;
    if (r.how == kLanes) {
#pragma unroll
        for (int j = 0; j < NP; ++j)
            for (int d = 1; d < r.lanes; d *= 2) p[j] = Op::of(p[j], __shfl_xor_sync(0xffffffffu, p[j], d));
    } else if (r.how == kRow) {
        float s = p[0];
#pragma unroll
        for (int j = 1; j < NP; ++j) s = Op::of(s, p[j]);
#pragma unroll
        for (int d = 1; d < 32; d *= 2) s = Op::of(s, __shfl_xor_sync(0xffffffffu, s, d));
        if (warps > 1) {
            float* mine = shared + threadIdx.y * 32;
            if (lane == 0) mine[warp] = s;
            __syncthreads();
            s = lane < warps ? mine[lane] : 0.f;               // (neutral for the maximum of absolute values too)
#pragma unroll
            for (int d = 1; d < 32; d *= 2) s = Op::of(s, __shfl_xor_sync(0xffffffffu, s, d));
            __syncthreads();
        }
#pragma unroll
        for (int j = 0; j < NP; ++j) p[j] = s;
    } else {
        float *mine = shared + threadIdx.y * (packs + r.count), *runs = mine + packs;
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

constexpr int kMostThreads = 512;                              // of a block: 128 registers each
// Places of a thread at most, for packs of V elements: 16384 elements in 512 threads.
constexpr int most_places(int v) { return v > 2 ? 8 : v > 1 ? 16 : 32; }

// Every row has its block, and an SM four of 256 threads at once: walks over rows with the next row's numbers under way, as the backward pass takes them, need the
// registers of half of those (8192 x 4096 to 8 bits 74 us so, 53 without).
template <typename T, int V, int NP>
__global__ void __launch_bounds__(kMostThreads, V > 2 && NP <= 2 ? 2 : 1) rms_fwd_kernel(const RmsArgs a, Runs groups, Runs blocks, int packs, int channels)
{
    extern __shared__ float shared[];
    ptx::grid_dep_wait();
    const long long row = (long long)blockIdx.x * blockDim.y + threadIdx.y;
    const bool real = row < a.M;
    const T *x = static_cast<const T*>(a.x) + row * a.ldx, *res = static_cast<const T*>(a.residual) + (a.residual ? row * a.ldr : 0);
    const float inverse = 1.f / channels;
    float f[NP][V], s[NP];
    Pack<T, V> px[NP], pr[NP], pz[NP];
    int at[NP];
#pragma unroll
    for (int j = 0; j < NP; ++j) {
        const int p = at[j] = pack_of_place(threadIdx.x + j * blockDim.x, groups, packs);
        const bool there = real && p < packs;
        px[j] = load_masked<T, V>(x + p * V, there);
        if (a.residual) pr[j] = load_masked<T, V>(res + p * V, there);
        if (a.z) pz[j] = load_masked<T, V>(static_cast<const T*>(a.z) + row * a.ldz + p * V, there);
    }
#pragma unroll
    for (int j = 0; j < NP; ++j) {
        const int p = at[j];
        unpack<T, V>(px[j], f[j]);
        if (a.residual) {                                      // the sum as it is stored is what is normalised, so that the backward pass sees the same
            float r[V];
            unpack<T, V>(pr[j], r);
#pragma unroll
            for (int e = 0; e < V; ++e) f[j][e] += r[e];
            const Pack<T, V> sum = pack<T, V>(f[j]);
            unpack<T, V>(sum, f[j]);
            if (real && p < packs) store_pack<T, V>(static_cast<T*>(a.h) + row * a.ldh + p * V, sum);
        }
        s[j] = 0.f;
#pragma unroll
        for (int e = 0; e < V; ++e) s[j] = fmaf(f[j][e], f[j][e], s[j]);
        s[j] *= inverse;                                       // (a mean does not overflow where its terms do not, a sum of thousands would)
    }
    reduce_runs<Sum>(s, at, groups, packs, shared);
    float most[NP];
#pragma unroll
    for (int j = 0; j < NP; ++j) {
        const int p = at[j];
        const float r = rsqrtf(s[j] + a.eps);
        const bool there = real && p < packs;
        const int group = a.G > 1 ? p / groups.packs : 0;
        if (a.rstd && there && p == group * groups.packs) a.rstd[row * a.G + group] = r;
        float w[V];
        if (there) load_gamma<V>(a.gamma, (p - group * groups.packs) * V, w);
#pragma unroll
        for (int e = 0; e < V; ++e) f[j][e] = there ? f[j][e] * r * w[e] : 0.f;
        if (a.z) {
            float z[V];
            unpack<T, V>(pz[j], z);
            activate(z, CONV2D_ACT_SILU);
#pragma unroll
            for (int e = 0; e < V; ++e) f[j][e] *= z[e];
        }
        if (a.y && there) store_pack<T, V>(static_cast<T*>(a.y) + row * a.ldy + p * V, pack<T, V>(f[j]));
        most[j] = 0.f;
#pragma unroll
        for (int e = 0; e < V; ++e) most[j] = fmaxf(most[j], fabsf(f[j][e]));
    }
    if (!a.y8) return;
    reduce_runs<Max>(most, at, blocks, packs, shared);
#pragma unroll
    for (int j = 0; j < NP; ++j) {
        const int p = at[j];
        if (!real || p >= packs) continue;
        const float scale = fmaxf(most[j] * (1.f / 448.f), 1.17549435e-38f), up = 1.f / scale;
        const int block = blocks.count > 1 ? p / blocks.packs : 0;
        if (p == block * blocks.packs) a.scales[row * blocks.count + block] = scale;
#pragma unroll
        for (int e = 0; e < V; ++e) f[j][e] *= up;
        store_codes<V>(static_cast<unsigned char*>(a.y8) + row * a.ld8 + p * V, f[j]);
    }
}

// Backward: with n = dy gamma silu(z) and m = h r,   dx = r (n - m mean(n m)) + dh.  A block takes rows gridDim.x * blockDim.y apart, the next one's numbers under way
// while it computes, and keeps its sums for gamma in registers until the end, when they are added over its rows and groups.
template <typename T, int V, int NP>
__global__ void __launch_bounds__(kMostThreads, 1) rms_bwd_kernel(const RmsArgs a, Runs groups, int packs, int channels)
{
    extern __shared__ float shared[];
    ptx::grid_dep_wait();
    const float inverse = 1.f / channels;
    float w[NP][V], dw[NP][V], r[NP];
    int group[NP], at[NP];
    Pack<T, V> ph[NP], py[NP], pd[NP], pz[NP];
    const long long step = (long long)gridDim.x * blockDim.y;
    auto fetch = [&](long long row) {
#pragma unroll
        for (int j = 0; j < NP; ++j) {
            const int p = at[j];
            const bool there = row < a.M && p < packs;
            ph[j] = load_masked<T, V>(static_cast<const T*>(a.x) + row * a.ldx + p * V, there);
            py[j] = load_masked<T, V>(static_cast<const T*>(a.dy) + row * a.lddy + p * V, there);
            if (a.dh) pd[j] = load_masked<T, V>(static_cast<const T*>(a.dh) + row * a.lddh + p * V, there);
            if (a.z) pz[j] = load_masked<T, V>(static_cast<const T*>(a.z) + row * a.ldz + p * V, there);
            r[j] = load_masked<float, 1>(a.rstd_in + row * a.G + group[j], there).e[0];
        }
    };
#pragma unroll
    for (int j = 0; j < NP; ++j) {
        const int p = at[j] = pack_of_place(threadIdx.x + j * blockDim.x, groups, packs);
        group[j] = a.G > 1 ? p / groups.packs : 0;
        if (p < packs) load_gamma<V>(a.gamma, (p - group[j] * groups.packs) * V, w[j]);
#pragma unroll
        for (int e = 0; e < V; ++e) dw[j][e] = 0.f, w[j][e] = p < packs ? w[j][e] : 0.f;
    }
    fetch((long long)blockIdx.x * blockDim.y + threadIdx.y);
    for (long long row0 = (long long)blockIdx.x * blockDim.y; row0 < a.M; row0 += step) {
        const long long row = row0 + threadIdx.y;
        const bool real = row < a.M;
        float m[NP][V], n[NP][V], d[NP][V], s[NP], rr[NP];
#pragma unroll
        for (int j = 0; j < NP; ++j) {
            const int p = at[j];
            unpack<T, V>(ph[j], m[j]);
            unpack<T, V>(py[j], n[j]);
            if (a.dh) unpack<T, V>(pd[j], d[j]);
            rr[j] = r[j];
#pragma unroll
            for (int e = 0; e < V; ++e) m[j][e] *= rr[j];
            if (a.z) {
                float z[V], dz[V];
                unpack<T, V>(pz[j], z);
#pragma unroll
                for (int e = 0; e < V; ++e) dz[e] = n[j][e] * w[j][e] * m[j][e];
                times_slope(dz, z, CONV2D_ACT_SILU);
                activate(z, CONV2D_ACT_SILU);
#pragma unroll
                for (int e = 0; e < V; ++e) n[j][e] *= z[e];
                if (real && p < packs) store_pack<T, V>(static_cast<T*>(a.dz) + row * a.lddz + p * V, pack<T, V>(dz));
            }
            s[j] = 0.f;
#pragma unroll
            for (int e = 0; e < V; ++e) {
                dw[j][e] = fmaf(n[j][e], m[j][e], dw[j][e]);
                n[j][e] *= w[j][e];
                s[j] = fmaf(n[j][e], m[j][e], s[j]);
            }
        }
        fetch(row + step);
        reduce_runs<Sum>(s, at, groups, packs, shared);
#pragma unroll
        for (int j = 0; j < NP; ++j) {
            const int p = at[j];
            const float mean = s[j] * inverse;
#pragma unroll
            for (int e = 0; e < V; ++e) n[j][e] = rr[j] * fmaf(-m[j][e], mean, n[j][e]);
            if (a.dh) {
#pragma unroll
                for (int e = 0; e < V; ++e) n[j][e] += d[j][e];
            }
            if (real && p < packs) store_pack<T, V>(static_cast<T*>(a.dx) + row * a.lddx + p * V, pack<T, V>(n[j]));
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
size_t shared_bytes(const RowPlan& p, const Runs& r) { return r.how == kShared ? (size_t)p.rows * (p.packs + r.count) * 4 : r.how == kRow ? p.rows * 32 * 4 : 0; }

template <typename T, int V, int NP>
conv2d_status_t forward(const RmsArgs& a, const RowPlan& p, cudaStream_t stream)
{
    static SmemLimit limit;
    const Runs groups = p.groups, blocks = p.blocks(a.y8 ? a.block : a.C);
    const size_t one = shared_bytes(p, groups), two = shared_bytes(p, blocks), smem = one > two ? one : two;
    if (raise_smem_limit((const void*)rms_fwd_kernel<T, V, NP>, smem, limit) != cudaSuccess) return CONV2D_ERR_CUDA;
    if (launch_pdl(rms_fwd_kernel<T, V, NP>, dim3(ceil_div_u(a.M, p.rows)), dim3(p.threads, p.rows), smem, stream, a, groups, blocks, p.packs, a.C / a.G) !=
        cudaSuccess)
        return CONV2D_ERR_CUDA;
    count_launch();
    return CONV2D_OK;
}

// Blocks of the backward pass: two for every SM, whose partial sums are added afterwards.
int bwd_blocks(int M, int rows)
{
    const long long all = ((long long)M + rows - 1) / rows, most = 2LL * sm_count();
    return (int)(all < most ? all : most);
}

template <typename T, int V, int NP>
conv2d_status_t backward(const RmsArgs& a, const RowPlan& p, cudaStream_t stream)
{
    static SmemLimit limit;
    const Runs groups = p.groups;
    const size_t runs = shared_bytes(p, groups), sums = a.dgamma ? (size_t)p.rows * a.C * 4 : 0, smem = runs > sums ? runs : sums;
    if (raise_smem_limit((const void*)rms_bwd_kernel<T, V, NP>, smem, limit) != cudaSuccess) return CONV2D_ERR_CUDA;
    const int blocks = bwd_blocks(a.M, p.rows), channels = a.C / a.G;
    if (launch_pdl(rms_bwd_kernel<T, V, NP>, dim3(blocks), dim3(p.threads, p.rows), smem, stream, a, groups, p.packs, channels) != cudaSuccess) return CONV2D_ERR_CUDA;
    count_launch();
    if (!a.dgamma) return CONV2D_OK;
    if (launch_pdl(rms_gamma_kernel, dim3(ceil_div_u(channels, 32)), dim3(32, 32), 0, stream, a.ws, a.dgamma, blocks, channels) != cudaSuccess) return CONV2D_ERR_CUDA;
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

template <typename T, int V, int NP>
conv2d_status_t either(const RmsArgs& a, const RowPlan& p, bool bwd, cudaStream_t stream)
{
    return bwd ? backward<T, V, NP>(a, p, stream) : forward<T, V, NP>(a, p, stream);
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
size_t rms_bwd_workspace_bytes(int M, int C, int G) { return ((size_t)bwd_blocks(M, 1) * (C / G) * 4 + 15) / 16 * 16; }
conv2d_status_t launch_rms_fwd(const RmsArgs& a, conv2d_operand_t type, cudaStream_t stream) { return rms(a, type, false, stream); }
conv2d_status_t launch_rms_bwd(const RmsArgs& a, conv2d_operand_t type, cudaStream_t stream) { return rms(a, type, true, stream); }

}  // namespace conv2d_b200
