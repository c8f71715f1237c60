// Short causal convolution of every channel along the sequence, channels last.
//
//   a[b,t,d] = bias[d] + sum_k w[d,k] xe[b,t-(K-1)+k,d],   y = act(a),   xe = (state_in rows | x rows)
//
// 2K flops an element: memory decides.  A thread owns V adjacent channels (16 bytes where the rows allow it) and walks
// down a piece of the sequence with the last K rows in registers, so that every element is loaded once but for the K-1
// rows before the piece; the loads of four rows are under way together.
#include "seq_common.cuh"

namespace conv2d_b200 {
namespace {

constexpr int kThreads = 128;
constexpr int kAhead = 4;               // rows whose loads are under way together

template <typename T>
struct FwdArgs {
    const T *x, *w, *bias, *state_in;
    const int* lengths;
    T *y, *state_out;
    int B, L, D, rows, pieces, packs;   // rows of a piece, pieces of a sequence, channel packs of a row
    long long ldx, ldy;
    int act;
};

template <typename T, int V, int K>
__global__ void __launch_bounds__(kThreads) conv1d_fwd_kernel(const FwdArgs<T> a)
{
    ptx::grid_dep_wait();
    const unsigned id = blockIdx.x * kThreads + threadIdx.x;      // (the launcher keeps the number of threads below 2^31)
    const int c = (int)(id % a.packs) * V;
    const unsigned rest = id / a.packs;
    const int piece = (int)(rest % a.pieces);
    const long long b = rest / a.pieces;
    if (b >= a.B) return;
    const int len = sequence_length(a.lengths, (int)b, a.L);
    const T* x = a.x + b * a.L * a.ldx + c;
    T* y = a.y + b * a.L * a.ldy + c;
    const int t0 = piece * a.rows, t1 = min(t0 + a.rows, a.L), live = min(t1, len);

    float w[K][V], bias[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        bias[i] = a.bias ? to_float(a.bias[c + i]) : 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k) w[k][i] = to_float(a.w[(size_t)(c + i) * K + k]);
    }
    // the row t of the extended sequence, as stored (t < len)
    auto row = [&](int t) -> Pack<T, V> {
        if (t >= 0) return load_pack<T, V>(x + t * a.ldx);
        return a.state_in ? load_pack<T, V>(a.state_in + ((size_t)b * (K - 1) + (t + K - 1)) * a.D + c) : zero_pack<T, V>();
    };

    float win[K][V];                    // win[k]: row t-(K-1)+k
    if (t0 < live) {
#pragma unroll
        for (int k = 0; k < K - 1; ++k) unpack(row(t0 - (K - 1) + k), win[k + 1]);
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
    for (int t = t0; t < live; t += kAhead) {
        Pack<T, V> in[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) in[j] = t + j < live ? load_pack<T, V>(x + (t + j) * a.ldx) : zero_pack<T, V>();
        float out[kAhead * V];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
#pragma unroll
            for (int k = 0; k < K - 1; ++k)
#pragma unroll
                for (int i = 0; i < V; ++i) win[k][i] = win[k + 1][i];
            unpack(in[j], win[K - 1]);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                float s = bias[i];
#pragma unroll
                for (int k = 0; k < K; ++k) s = fmaf(w[k][i], win[k][i], s);
                out[j * V + i] = s;
            }
        }
        activate(out, a.act);
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            if (t + j >= live) break;
            float o[V];
#pragma unroll
            for (int i = 0; i < V; ++i) o[i] = out[j * V + i];
            store_pack(y + (t + j) * a.ldy, pack<T, V>(o));
        }
    }
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
    int B, L, D, pieces, packs;
    unsigned jobs;                      // pieces of all sequences
    long long ldx, lddy, lddx;
    int act;
};

constexpr int kBwdThreads = 256;
constexpr int kBwdRows = 32;            // rows of a piece: K-1 rows of x before and K-1 of both inputs after it are read again

template <typename T, int V, int K>
__global__ void __launch_bounds__(kBwdThreads) conv1d_bwd_kernel(const BwdArgs<T> a)
{
    ptx::grid_dep_wait();
    extern __shared__ float sums[];     // [blockDim.y][K+1][blockDim.x * V]
    const int pk = blockIdx.y * blockDim.x + threadIdx.x;
    const int c = pk * V;
    float dw[K][V] = {}, db[V] = {}, w[K][V], bias[V];
    if (pk < a.packs) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            bias[i] = a.bias ? to_float(a.bias[c + i]) : 0.f;
#pragma unroll
            for (int k = 0; k < K; ++k) w[k][i] = to_float(a.w[(size_t)(c + i) * K + k]);
        }
    }
    for (unsigned job = blockIdx.x * blockDim.y + threadIdx.y; job < a.jobs && pk < a.packs; job += gridDim.x * blockDim.y) {
        const int piece = (int)(job % a.pieces);
        const long long b = job / a.pieces;
        const int len = sequence_length(a.lengths, (int)b, a.L);
        const T* x = a.x + b * a.L * a.ldx + c;
        const T* dy = a.dy + b * a.L * a.lddy + c;
        T* dx = a.dx + b * a.L * a.lddx + c;
        const int t0 = piece * kBwdRows, t1 = min(t0 + kBwdRows, a.L);
        auto row = [&](int t) -> Pack<T, V> {
            if (t >= len) return zero_pack<T, V>();
            if (t >= 0) return load_pack<T, V>(x + t * a.ldx);
            return a.state_in ? load_pack<T, V>(a.state_in + ((size_t)b * (K - 1) + (t + K - 1)) * a.D + c) : zero_pack<T, V>();
        };
        // the first piece also has the K-1 rows of the state
        const int first = piece == 0 && a.dstate_in ? -(K - 1) : t0;
        const int stop = min(t1, len);
        float xw[K > 1 ? K - 1 : 1][V], gw[K][V] = {};        // rows t-(K-1) .. t-1 of xe, t-(K-1) .. t of g
#pragma unroll
        for (int k = 0; k < K - 1; ++k) unpack(row(t0 - (K - 1) + k), xw[k]);
        // t walks the rows of g; the row of dx that it completes is t-(K-1)
        for (int t = t0; t < stop + K - 1; t += kAhead) {
            Pack<T, V> xin[kAhead], gin[kAhead];
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                xin[j] = row(t + j);
                gin[j] = t + j < len ? load_pack<T, V>(dy + (t + j) * a.lddy) : zero_pack<T, V>();
            }
            // a of the rows, then g
            float pre[kAhead * V], g[kAhead * V], xk[kAhead + K - 1][V];
#pragma unroll
            for (int k = 0; k < K - 1; ++k)
#pragma unroll
                for (int i = 0; i < V; ++i) xk[k][i] = xw[k][i];
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                float gi[V];
                unpack(xin[j], xk[K - 1 + j]);
                unpack(gin[j], gi);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    float s = bias[i];
#pragma unroll
                    for (int k = 0; k < K; ++k) s = fmaf(w[k][i], xk[j + k][i], s);
                    pre[j * V + i] = s;
                    g[j * V + i] = gi[i];
                }
            }
            times_slope(g, pre, a.act);
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                const int tt = t + j;
                const bool real = tt < len, own = tt < stop;      // each row of g counts once, in its own piece
#pragma unroll
                for (int k = 0; k < K - 1; ++k)
#pragma unroll
                    for (int i = 0; i < V; ++i) gw[k][i] = gw[k + 1][i];
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float gi = real ? g[j * V + i] : 0.f, go = own ? gi : 0.f;
                    gw[K - 1][i] = gi;
                    db[i] += go;
#pragma unroll
                    for (int k = 0; k < K; ++k) dw[k][i] = fmaf(go, xk[j + k][i], dw[k][i]);
                }
                const int td = tt - (K - 1);
                if (td < first || td >= stop) continue;
                float out[V];
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    float s = 0.f;
#pragma unroll
                    for (int k = 0; k < K; ++k) s = fmaf(w[k][i], gw[K - 1 - k][i], s);
                    out[i] = s;
                }
                if (a.dstate_out && td >= len - (K - 1)) {
                    float e[V];
                    unpack(load_pack<T, V>(a.dstate_out + ((size_t)b * (K - 1) + (td - len + K - 1)) * a.D + c), e);
#pragma unroll
                    for (int i = 0; i < V; ++i) out[i] += e[i];
                }
                if (td >= 0) store_pack(dx + td * a.lddx, pack<T, V>(out));
                else store_pack(a.dstate_in + ((size_t)b * (K - 1) + (td + K - 1)) * a.D + c, pack<T, V>(out));
            }
#pragma unroll
            for (int k = 0; k < K - 1; ++k)
#pragma unroll
                for (int i = 0; i < V; ++i) xw[k][i] = xk[kAhead + k][i];
        }
        for (int t = max(t0, len); t < t1; ++t) store_pack(dx + t * a.lddx, zero_pack<T, V>());
    }
    if (!a.partials) return;
    const int width = blockDim.x * V;
    float* own = sums + (size_t)threadIdx.y * (K + 1) * width + threadIdx.x * V;
#pragma unroll
    for (int i = 0; i < V; ++i) {
#pragma unroll
        for (int k = 0; k < K; ++k) own[k * width + i] = dw[k][i];
        own[K * width + i] = db[i];
    }
    __syncthreads();
    for (int i = threadIdx.y * blockDim.x + threadIdx.x; i < (K + 1) * width; i += kBwdThreads) {
        const int k = i / width, ch = blockIdx.y * width + i % width;
        if (ch >= a.D) continue;
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
// gradients) as fill the machine twice.
struct BwdPlan { int pieces, tx, ty; long long jobs, parts, across; };
BwdPlan bwd_plan(int B, int L, int D, int V)
{
    BwdPlan p;
    const int packs = D / V;
    p.tx = 1;
    while (p.tx < 32 && p.tx < packs) p.tx *= 2;
    p.ty = kBwdThreads / p.tx;
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
    // Short pieces until the machine is full: 8 rows are the fewest (not below K-1), 32 the most
    a.rows = 32;
    while (a.rows > 8 && (long long)a.packs * s.B * ceil_div_u(s.L, a.rows) < (long long)sm_count() * 1024) a.rows /= 2;
    a.pieces = (int)ceil_div_u(s.L, a.rows);
    const long long threads = (long long)a.packs * a.pieces * s.B;
    if (threads > 0x7fffff00LL) return CONV2D_ERR_SHAPE;
    if (launch_pdl(conv1d_fwd_kernel<T, V, K>, dim3(ceil_div_u(threads, kThreads)), dim3(kThreads), 0, stream, a) != cudaSuccess) return CONV2D_ERR_CUDA;
    count_launch();
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
    if (p.across > 65535 || p.jobs > 0x7fff0000LL) return CONV2D_ERR_SHAPE;
    const size_t smem = (size_t)kBwdThreads * V * (K + 1) * sizeof(float);
    static SmemLimit limit;
    if (raise_smem_limit(reinterpret_cast<const void*>(conv1d_bwd_kernel<T, V, K>), smem, limit) != cudaSuccess) return CONV2D_ERR_CUDA;
    if (launch_pdl(conv1d_bwd_kernel<T, V, K>, dim3((unsigned)p.parts, (unsigned)p.across), dim3(p.tx, p.ty), smem, stream, a) != cudaSuccess)
        return CONV2D_ERR_CUDA;
    count_launch();
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
    constexpr int V = 16 / sizeof(T);
    return wide<T, V>(s) ? fwd_taps<T, V>(s, stream) : fwd_taps<T, 1>(s, stream);
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
