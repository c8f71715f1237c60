// Short causal convolution of every channel along the sequence, channels last.
//
//   a[b,t,d] = bias[d] + sum_k w[d,k] xe[b,t-(K-1)+k,d],   y = act(a),   xe = (state_in rows | x rows)
//
// 2K flops an element: memory decides, if the loads are far enough ahead and little is done beside them.  A thread owns V adjacent channels (8 or
// 16 bytes where the rows allow it) and walks down a piece of the sequence with the last K rows in registers, so that every element is loaded once
// but for the K-1 rows before the piece.  The rows come in by asynchronous copies into a ring of shared memory that belongs to the thread, three
// groups of four rows ahead; loads into registers were too few at a time (4 x 4096 x 4096 in bf16: 88 us, backward 638).  Products and
// activations are packed, two channels an instruction.  52 us so (5.2 TB/s; the floor is 41), backward 112 (3.6 TB/s; the floor is 61): 150 registers
// leave three blocks of four warps an SM, which issue in 62 % of the cycles while memory and the FMA pipe are half busy, and every piece of 64 rows waits for its
// taps, its window and its first rows in turn.
#include "seq_common.cuh"

namespace conv2d_b200 {
namespace {

constexpr int kThreads = 128;
constexpr int kGroup = 4, kRing = 4;    // rows of a group, groups of the ring

// w[k][pair], bias[pair] of the channels from c on
template <typename T, int V, int K>
__device__ __forceinline__ void load_taps(const T* w, const T* bias, int c, float2 (&wt)[K][kPairs<V>], float2 (&bt)[kPairs<V>])
{
    float f[K + 1][V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        f[K][i] = bias ? to_float(bias[c + i]) : 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k) f[k][i] = to_float(w[(size_t)(c + i) * K + k]);
    }
#pragma unroll
    for (int i = 0; i < kPairs<V>; ++i) {
        bt[i] = make_float2(f[K][2 * i], V > 1 ? f[K][V > 1 ? 2 * i + 1 : 0] : 0.f);
#pragma unroll
        for (int k = 0; k < K; ++k) wt[k][i] = make_float2(f[k][2 * i], V > 1 ? f[k][V > 1 ? 2 * i + 1 : 0] : 0.f);
    }
}

template <typename T>
struct FwdArgs {
    const T *x, *w, *bias, *state_in;
    const int* lengths;
    T *y, *state_out;
    int B, L, D, rows, pieces, packs;   // rows of a piece, pieces of a sequence, channel packs of a row
    long long ldx, ldy;
    int act;
};

// Blocks an SM: with 112 registers, as the activations' branches take them where nothing holds them, four taps had four (3 x 1083 x 1928 in fp16 12.2 us, 11.6 with five).
constexpr int fwd_blocks(int K) { return K == 1 ? 7 : K == 2 ? 6 : K <= 4 ? 5 : 4; }

template <typename T, int V, int K>
__global__ void __launch_bounds__(kThreads, fwd_blocks(K)) conv1d_fwd_kernel(const FwdArgs<T> a)
{
    constexpr int P = kPairs<V>;
    ptx::grid_dep_wait();
    extern __shared__ float4 smem4[];
    const unsigned id = blockIdx.x * kThreads + threadIdx.x;      // (the launcher keeps the number of threads below 2^31)
    const int c = (int)(id % a.packs) * V;
    const unsigned rest = id / a.packs;
    const int piece = (int)(rest % a.pieces);
    const long long b = rest / a.pieces;
    if (b >= a.B) return;
    const int len = sequence_length(a.lengths, (int)b, a.L);
    T* y = a.y + b * a.L * a.ldy + c;
    const int t0 = piece * a.rows, t1 = min(t0 + a.rows, a.L), live = min(t1, len);
    using Ring = RowRing<T, V, kThreads, kGroup, kRing>;
    const Ring x{reinterpret_cast<unsigned char*>(smem4) + threadIdx.x * Ring::bytes, a.x + b * a.L * a.ldx + c, a.ldx};
#pragma unroll
    for (int q = 0; q < kRing - 1; ++q) {
        x.issue(q, t0 + q * kGroup, live);
        copies_commit();
    }

    float2 w[K][P], bias[P];
    load_taps<T, V, K>(a.w, a.bias, c, w, bias);
    // the row t of the extended sequence, as stored (t < len)
    auto row = [&](int t) -> Pack<T, V> {
        if (t >= 0) return load_pack<T, V>(x.p + t * a.ldx);
        return a.state_in ? load_pack<T, V>(a.state_in + ((size_t)b * (K - 1) + (t + K - 1)) * a.D + c) : zero_pack<T, V>();
    };
    float2 win[kGroup + K - 1][P];      // rows t-(K-1) .. t+3
    if (t0 < live) {
#pragma unroll
        for (int k = 0; k < K - 1; ++k) pairs<T, V>(row(t0 - (K - 1) + k), win[k]);
    }
    if (piece == 0 && a.state_out) {
        // the last K-1 rows of (state_in | x[0 .. len)); all are read before any is written, and no other piece reads state_in
        // (a piece has at least K-1 rows), so the two states may be one buffer
        Pack<T, V> last[K > 1 ? K - 1 : 1];
#pragma unroll
        for (int k = 0; k < K - 1; ++k) last[k] = row(len - (K - 1) + k);
#pragma unroll
        for (int k = 0; k < K - 1; ++k) store_pack(a.state_out + ((size_t)b * (K - 1) + k) * a.D + c, last[k]);
    }
    T* to = y + (long long)t0 * a.ldy;
    auto group = [&](int q, int t, auto whole) {
        copies_wait<kRing - 2>();
#pragma unroll
        for (int j = 0; j < kGroup; ++j) pairs<T, V>(x.get(q, t, j, live), win[K - 1 + j]);
        x.issue(q + kRing - 1, t + (kRing - 1) * kGroup, live);
        copies_commit();
        float out[kGroup * 2 * P];
#pragma unroll
        for (int j = 0; j < kGroup; ++j) {
#pragma unroll
            for (int i = 0; i < P; ++i) {
                float2 s = bias[i];
#pragma unroll
                for (int k = 0; k < K; ++k) s = __ffma2_rn(w[k][i], win[j + k][i], s);
                out[2 * (j * P + i)] = s.x, out[2 * (j * P + i) + 1] = s.y;
            }
        }
        activate(out, a.act);
#pragma unroll
        for (int j = 0; j < kGroup; ++j, to += a.ldy) {
            float2 o[P];
#pragma unroll
            for (int i = 0; i < P; ++i) o[i] = make_float2(out[2 * (j * P + i)], out[2 * (j * P + i) + 1]);
            if (decltype(whole)::value || t + j < live) store_pack(to, pack_of<T, V>(o));
        }
#pragma unroll
        for (int k = 0; k < K - 1; ++k)
#pragma unroll
            for (int i = 0; i < P; ++i) win[k][i] = win[kGroup + k][i];
    };
    int q = 0, t = t0;
#pragma unroll 1
    for (; t + kGroup <= live; t += kGroup, ++q) group(q, t, Whole());
    if (t < live) group(q, t, Cut());
    for (int t = max(t0, len); t < t1; ++t) store_pack(y + t * a.ldy, zero_pack<T, V>());
}

// Backward.  g = dy act'(a) needs the K rows of x that a is made of, dx[t] needs g of the K rows from t on: a thread walks from the first
// row of its piece to K-1 rows beyond its last, with K rows of x and of g in registers, and adds up the gradients of
// its channels' taps in fp32.  The blocks join the sums of the threads that own the same channels and write one partial sum each;
// a second kernel adds those in a fixed order, so that results do not depend on timing.
template <typename T>
struct BwdArgs {
    const T *x, *w, *bias, *state_in, *dy, *dstate_out;
    const int* lengths;
    T *dx, *dstate_in;
    float* partials;                    // [blockIdx.x][K+1][D]
    int B, L, D, pieces, packs;         // packs: of channels, from those that the pointers name on
    unsigned jobs;                      // pieces of all sequences
    long long ldx, lddy, lddx;
    int act;
};

constexpr int kBwdGroup = 2, kBwdRing = 4;     // (groups of four rows: 130 us on 4 x 4096 x 4096, 122 so)
constexpr int kBwdRows = 64;            // rows of a piece: K-1 rows of x before and K-1 of both inputs after it are read again

template <typename T, int V, int K>
__global__ void __launch_bounds__(kThreads) conv1d_bwd_kernel(const BwdArgs<T> a)
{
    constexpr int P = kPairs<V>;
    ptx::grid_dep_wait();
    extern __shared__ float4 smem4[];   // the rings, then the sums [blockDim.y][K+1][blockDim.x * V]
    using Ring = RowRing<T, V, kThreads, kBwdGroup, kBwdRing>;
    const int tid = threadIdx.y * blockDim.x + threadIdx.x;
    const int pk = blockIdx.y * blockDim.x + threadIdx.x, c = pk * V;
    float2 dw[K][P], db[P], w[K][P], bias[P];
#pragma unroll
    for (int i = 0; i < P; ++i) {
        db[i] = both(0.f);
#pragma unroll
        for (int k = 0; k < K; ++k) dw[k][i] = both(0.f);
    }
    if (pk < a.packs) load_taps<T, V, K>(a.w, a.bias, c, w, bias);
    for (unsigned job = blockIdx.x * blockDim.y + threadIdx.y; job < a.jobs && pk < a.packs; job += gridDim.x * blockDim.y) {
        const int piece = (int)(job % a.pieces);
        const long long b = job / a.pieces;
        const int len = sequence_length(a.lengths, (int)b, a.L);
        const int t0 = piece * kBwdRows, t1 = min(t0 + kBwdRows, a.L);
        const Ring x{reinterpret_cast<unsigned char*>(smem4) + tid * Ring::bytes, a.x + b * a.L * a.ldx + c, a.ldx};
        const Ring dy{reinterpret_cast<unsigned char*>(smem4) + Ring::smem + tid * Ring::bytes, a.dy + b * a.L * a.lddy + c, a.lddy};
        T* dx = a.dx + b * a.L * a.lddx + c;
        // the first piece also has the K-1 rows of the state
        const int first = piece == 0 && a.dstate_in ? -(K - 1) : t0;
        const int stop = min(t1, len), end = stop + K - 1;    // t walks the rows of g; the row of dx that it completes is t-(K-1)
#pragma unroll
        for (int q = 0; q < kBwdRing - 1; ++q) {
            x.issue(q, t0 + q * kBwdGroup, len);
            dy.issue(q, t0 + q * kBwdGroup, len);
            copies_commit();
        }
        float2 xw[kBwdGroup + K - 1][P], gw[kBwdGroup + K - 1][P];  // rows t-(K-1) .. t+3 of xe and of g
#pragma unroll
        for (int k = 0; k < K - 1; ++k) {
            const int t = t0 - (K - 1) + k;
            Pack<T, V> p = zero_pack<T, V>();
            if (t >= 0 && t < len) p = load_pack<T, V>(x.p + t * a.ldx);
            if (t < 0 && a.state_in) p = load_pack<T, V>(a.state_in + ((size_t)b * (K - 1) + (t + K - 1)) * a.D + c);
            pairs<T, V>(p, xw[k]);
#pragma unroll
            for (int i = 0; i < P; ++i) gw[k][i] = both(0.f);
        }
        auto group = [&](int q, int t, auto whole) {
            copies_wait<kBwdRing - 2>();
            float g[kBwdGroup * 2 * P], pre[kBwdGroup * 2 * P];
#pragma unroll
            for (int j = 0; j < kBwdGroup; ++j) {
                float2 gi[P];
                pairs<T, V>(x.get(q, t, j, len), xw[K - 1 + j]);
                pairs<T, V>(dy.get(q, t, j, len), gi);        // (zero behind the sequence)
#pragma unroll
                for (int i = 0; i < P; ++i) g[2 * (j * P + i)] = gi[i].x, g[2 * (j * P + i) + 1] = gi[i].y;
            }
            x.issue(q + kBwdRing - 1, t + (kBwdRing - 1) * kBwdGroup, len);
            dy.issue(q + kBwdRing - 1, t + (kBwdRing - 1) * kBwdGroup, len);
            copies_commit();
#pragma unroll
            for (int j = 0; j < kBwdGroup; ++j) {
#pragma unroll
                for (int i = 0; i < P; ++i) {
                    float2 s = bias[i];
#pragma unroll
                    for (int k = 0; k < K; ++k) s = __ffma2_rn(w[k][i], xw[j + k][i], s);
                    pre[2 * (j * P + i)] = s.x, pre[2 * (j * P + i) + 1] = s.y;
                }
            }
            times_slope(g, pre, a.act);
            if (!decltype(whole)::value) {      // behind the sequence an overflowing slope must not make zeros NaN
#pragma unroll
                for (int j = 0; j < kBwdGroup; ++j)
#pragma unroll
                    for (int i = 0; i < 2 * P; ++i)
                        if (t + j >= len) g[2 * j * P + i] = 0.f;
            }
#pragma unroll
            for (int j = 0; j < kBwdGroup; ++j) {
#pragma unroll
                for (int i = 0; i < P; ++i) gw[K - 1 + j][i] = make_float2(g[2 * (j * P + i)], g[2 * (j * P + i) + 1]);
                // each row of g counts once, in its own piece
                if (!decltype(whole)::value && t + j >= stop) continue;
#pragma unroll
                for (int i = 0; i < P; ++i) {
                    db[i] = __fadd2_rn(db[i], gw[K - 1 + j][i]);
#pragma unroll
                    for (int k = 0; k < K; ++k) dw[k][i] = __ffma2_rn(gw[K - 1 + j][i], xw[j + k][i], dw[k][i]);
                }
            }
            T* to = dx + (long long)(t - (K - 1)) * a.lddx;
#pragma unroll
            for (int j = 0; j < kBwdGroup; ++j, to += a.lddx) {
                const int td = t + j - (K - 1);
                if (!decltype(whole)::value && (td < first || td >= stop)) continue;
                float2 out[P];
#pragma unroll
                for (int i = 0; i < P; ++i) {
                    out[i] = __fmul2_rn(w[0][i], gw[j + K - 1][i]);
#pragma unroll
                    for (int k = 1; k < K; ++k) out[i] = __ffma2_rn(w[k][i], gw[j + K - 1 - k][i], out[i]);
                }
                if (decltype(whole)::value) {
                    store_pack(to, pack_of<T, V>(out));
                    continue;
                }
                if (a.dstate_out && td >= len - (K - 1)) {
                    float2 e[P];
                    pairs<T, V>(load_pack<T, V>(a.dstate_out + ((size_t)b * (K - 1) + (td - len + K - 1)) * a.D + c), e);
#pragma unroll
                    for (int i = 0; i < P; ++i) out[i] = __fadd2_rn(out[i], e[i]);
                }
                if (td >= 0) store_pack(to, pack_of<T, V>(out));
                else store_pack(a.dstate_in + ((size_t)b * (K - 1) + (td + K - 1)) * a.D + c, pack_of<T, V>(out));
            }
#pragma unroll
            for (int k = 0; k < K - 1; ++k)
#pragma unroll
                for (int i = 0; i < P; ++i) xw[k][i] = xw[kBwdGroup + k][i], gw[k][i] = gw[kBwdGroup + k][i];
        };
        // a group is whole where all its rows of g are the piece's own and all rows of dx that it completes are, too (and so none of
        // the last K-1, to which a gradient of the state behind the sequence comes)
        int q = 0, t = t0;
#pragma unroll 1
        for (; t < end && t < t0 + K - 1; t += kBwdGroup, ++q) group(q, t, Cut());
#pragma unroll 1
        for (; t + kBwdGroup <= stop; t += kBwdGroup, ++q) group(q, t, Whole());
#pragma unroll 1
        for (; t < end; t += kBwdGroup, ++q) group(q, t, Cut());
        copies_wait<0>();               // (the ring is free for the next piece)
        for (int t = max(t0, len); t < t1; ++t) store_pack(dx + t * a.lddx, zero_pack<T, V>());
    }
    if (!a.partials) return;
    const int width = blockDim.x * V;
    float* sums = reinterpret_cast<float*>(smem4);            // (over the rings)
    __syncthreads();
    float* own = sums + (size_t)threadIdx.y * (K + 1) * width + threadIdx.x * V;
#pragma unroll
    for (int i = 0; i < V; ++i) {
#pragma unroll
        for (int k = 0; k < K; ++k) own[k * width + i] = i % 2 ? dw[k][i / 2].y : dw[k][i / 2].x;
        own[K * width + i] = i % 2 ? db[i / 2].y : db[i / 2].x;
    }
    __syncthreads();
    for (int i = tid; i < (K + 1) * width; i += kThreads) {
        const int k = i / width, ch = blockIdx.y * width + i % width;
        if (ch >= a.packs * V) continue;
        float s = 0.f;
        for (int j = 0; j < (int)blockDim.y; ++j) s += sums[(size_t)j * (K + 1) * width + i];
        a.partials[((size_t)blockIdx.x * (K + 1) + k) * a.D + ch] = s;
    }
}

// Column (k, d) of the partial sums [parts][K+1][D]: dw[d][k], and dbias[d] for k = K.
struct TapStore {
    float *dw, *dbias;
    int D, K;
    __device__ void operator()(long long col, float s) const
    {
        const long long k = col / D, d = col % D;
        if (k < K) {
            if (dw) dw[d * K + k] = s;
        } else if (dbias) {
            dbias[d] = s;
        }
    }
};

// Blocks of the backward pass: tx channel packs by ty pieces at a time; as many shares of the pieces (each a partial sum of the taps'
// gradients) as fill the machine four times.
struct BwdPlan { int pieces, tx, ty; long long jobs, parts, across; };
BwdPlan bwd_plan(int B, int L, int D, int V)
{
    BwdPlan p;
    const int packs = D / V;
    p.tx = 1;
    while (p.tx < 32 && p.tx < packs) p.tx *= 2;
    p.ty = kThreads / p.tx;
    p.across = ceil_div_u(packs, p.tx);
    p.pieces = (int)ceil_div_u(L, kBwdRows);
    p.jobs = (long long)B * p.pieces;
    const long long full = (p.jobs + p.ty - 1) / p.ty, most = (16LL * 148 + p.across - 1) / p.across;
    p.parts = full < most ? full : most;
    return p;
}

template <typename T, int V, int K>
conv2d_status_t fwd(const ConvSeq& s, cudaStream_t stream)
{
    FwdArgs<T> a;
    a.x = static_cast<const T*>(s.x), a.w = static_cast<const T*>(s.w), a.bias = static_cast<const T*>(s.bias);
    a.state_in = static_cast<const T*>(s.state_in), a.lengths = s.lengths;
    a.y = static_cast<T*>(s.y), a.state_out = static_cast<T*>(s.state_out);
    a.B = s.B, a.L = s.L, a.D = s.D, a.ldx = s.ldx, a.ldy = s.ldy, a.act = s.act;
    a.packs = s.D / V;
    // Short pieces until the machine is full: 8 rows are the fewest (not below K-1), 64 the most
    a.rows = 64;
    while (a.rows > 8 && (long long)a.packs * s.B * ceil_div_u(s.L, a.rows) < (long long)sm_count() * 1024) a.rows /= 2;
    a.pieces = (int)ceil_div_u(s.L, a.rows);
    // (threads are counted in 32 bits)
    const long long threads = (long long)a.packs * a.pieces;
    const int most = sequences_of_launch(ceil_div_u(threads, kThreads), 0x7fffff00 / kThreads, s.B);
    for (int b0 = 0; b0 < s.B; b0 += most) {
        FwdArgs<T> r = a;
        const size_t rows = (size_t)b0 * s.L, state = (size_t)b0 * (K - 1) * s.D;
        r.x += rows * s.ldx, r.y += rows * s.ldy;
        if (r.state_in) r.state_in += state;
        if (r.state_out) r.state_out += state;
        if (r.lengths) r.lengths += b0;
        r.B = s.B - b0 < most ? s.B - b0 : most;
        if (launch_pdl(conv1d_fwd_kernel<T, V, K>, dim3(ceil_div_u(threads * r.B, kThreads)), dim3(kThreads), RowRing<T, V, kThreads, kGroup, kRing>::smem, stream, r) != cudaSuccess)
            return CONV2D_ERR_CUDA;
        count_launch();
    }
    return CONV2D_OK;
}

template <typename T, int V, int K>
conv2d_status_t bwd(const ConvSeq& s, cudaStream_t stream)
{
    BwdArgs<T> a;
    a.x = static_cast<const T*>(s.x), a.w = static_cast<const T*>(s.w), a.bias = static_cast<const T*>(s.bias);
    a.state_in = static_cast<const T*>(s.state_in), a.dy = static_cast<const T*>(s.dy), a.dstate_out = static_cast<const T*>(s.dstate_out);
    a.lengths = s.lengths, a.dx = static_cast<T*>(s.dx), a.dstate_in = static_cast<T*>(s.dstate_in);
    a.B = s.B, a.L = s.L, a.D = s.D, a.ldx = s.ldx, a.lddy = s.lddy, a.lddx = s.lddx, a.act = s.act;
    const BwdPlan p = bwd_plan(s.B, s.L, s.D, V);
    a.pieces = p.pieces, a.packs = s.D / V, a.jobs = (unsigned)p.jobs;
    a.partials = s.dw || s.dbias ? s.partials : nullptr;
    const size_t rings = 2 * RowRing<T, V, kThreads, kBwdGroup, kBwdRing>::smem, sums = (size_t)kThreads * V * (K + 1) * sizeof(float), smem = rings > sums ? rings : sums;
    static SmemLimit limit;
    if (raise_smem_limit(reinterpret_cast<const void*>(conv1d_bwd_kernel<T, V, K>), smem, limit) != cudaSuccess) return CONV2D_ERR_CUDA;
    // channels lie along the grid's y; more than 65535 blocks of them (2^21 channels, one a thread) take a launch for every so many
    for (long long at = 0; at < p.across; at += 65535) {
        BwdArgs<T> r = a;
        const long long c = at * p.tx * V, across = p.across - at < 65535 ? p.across - at : 65535;
        const auto shift = [c](auto& q) { if (q) q += c; };
        shift(r.x), shift(r.bias), shift(r.state_in), shift(r.dy), shift(r.dstate_out), shift(r.dx), shift(r.dstate_in), shift(r.partials);
        r.w += c * K;
        r.packs = (int)((s.D - c) / V);
        if (launch_pdl(conv1d_bwd_kernel<T, V, K>, dim3((unsigned)p.parts, (unsigned)across), dim3(p.tx, p.ty), smem, stream, r) != cudaSuccess)
            return CONV2D_ERR_CUDA;
        count_launch();
    }
    if (!a.partials) return CONV2D_OK;
    return launch_column_sums(a.partials, p.parts, (long long)(K + 1) * s.D, (long long)(K + 1) * s.D, TapStore{s.dw, s.dbias, s.D, K}, stream);
}

template <typename T, int V>
conv2d_status_t fwd_taps(const ConvSeq& s, cudaStream_t stream)
{
    switch (s.K) {
        case 1: return fwd<T, V, 1>(s, stream);
        case 2: return fwd<T, V, 2>(s, stream);
        case 3: return fwd<T, V, 3>(s, stream);
        case 4: return fwd<T, V, 4>(s, stream);
        case 5: return fwd<T, V, 5>(s, stream);
        case 6: return fwd<T, V, 6>(s, stream);
        case 7: return fwd<T, V, 7>(s, stream);
        case 8: return fwd<T, V, 8>(s, stream);
    }
    return CONV2D_ERR_UNSUPPORTED;
}
template <typename T, int V>
conv2d_status_t bwd_taps(const ConvSeq& s, cudaStream_t stream)
{
    switch (s.K) {
        case 1: return bwd<T, V, 1>(s, stream);
        case 2: return bwd<T, V, 2>(s, stream);
        case 3: return bwd<T, V, 3>(s, stream);
        case 4: return bwd<T, V, 4>(s, stream);
        case 5: return bwd<T, V, 5>(s, stream);
        case 6: return bwd<T, V, 6>(s, stream);
        case 7: return bwd<T, V, 7>(s, stream);
        case 8: return bwd<T, V, 8>(s, stream);
    }
    return CONV2D_ERR_UNSUPPORTED;
}

// V channels a thread where every row of every tensor begins on a boundary of V elements, else one.
template <typename T, int V>
bool wide(const ConvSeq& s)
{
    constexpr int e = sizeof(T), n = e * V > 16 ? 16 : e * V;
    return s.D % V == 0 && rows_aligned(s.x, s.ldx, e, n) && rows_aligned(s.y, s.ldy, e, n) && rows_aligned(s.dy, s.lddy, e, n)
        && rows_aligned(s.dx, s.lddx, e, n) && rows_aligned(s.state_in, s.D, e, n) && rows_aligned(s.state_out, s.D, e, n)
        && rows_aligned(s.dstate_in, s.D, e, n) && rows_aligned(s.dstate_out, s.D, e, n);
}

template <typename T>
conv2d_status_t fwd_typed(const ConvSeq& s, cudaStream_t stream)
{
    return wide<T, 4>(s) ? fwd_taps<T, 4>(s, stream) : fwd_taps<T, 1>(s, stream);
}
template <typename T>
conv2d_status_t bwd_typed(const ConvSeq& s, cudaStream_t stream)
{
    return wide<T, 4>(s) ? bwd_taps<T, 4>(s, stream) : bwd_taps<T, 1>(s, stream);
}

}  // namespace

size_t conv1d_bwd_workspace_bytes(int B, int L, int D, int K)
{
    long long parts = bwd_plan(B, L, D, 1).parts;
    if (D % 4 == 0) {
        const long long p = bwd_plan(B, L, D, 4).parts;
        parts = p > parts ? p : parts;
    }
    return (size_t)parts * (K + 1) * D * sizeof(float);
}

conv2d_status_t launch_conv1d_fwd(const ConvSeq& s, conv2d_operand_t type, cudaStream_t stream)
{
    if (type == CONV2D_OPERAND_BF16) return fwd_typed<bf16>(s, stream);
    if (type == CONV2D_OPERAND_FP16) return fwd_typed<fp16>(s, stream);
    return fwd_typed<float>(s, stream);
}
conv2d_status_t launch_conv1d_bwd(const ConvSeq& s, conv2d_operand_t type, cudaStream_t stream)
{
    if (type == CONV2D_OPERAND_BF16) return bwd_typed<bf16>(s, stream);
    if (type == CONV2D_OPERAND_FP16) return bwd_typed<fp16>(s, stream);
    return bwd_typed<float>(s, stream);
}

}  // namespace conv2d_b200
