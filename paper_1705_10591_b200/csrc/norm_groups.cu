// Group norm with an activation, channels last.
//
//   m, q = mean and variance of the S x E elements of sample n and group g (E = C / G),  x^ = (x - m) / sqrt(q + eps),
//   y = act(gamma x^ + beta);   backward, with d = dy act'(.):
//   s1[n,c] = sum_s d,  s2[n,c] = sum_s d x^,  dbeta = sum_n s1,  dgamma = sum_n s2,
//   dx = rstd (gamma d - mean(gamma s1) - x^ mean(gamma s2))
//
// Memory decides: the floor is one reading of the inputs and one writing of the output.  Statistics come before the output, so the
// elements have to stay on chip in between:
//   rows     S = 1 and at most four packs of 16 bytes a lane (groups of 1024 16-bit elements, 512 fp32, fewer where they are not aligned): the elements of a
//            group lie together and stay in the registers of 1 to 32 lanes.
//   slab     a thread-block cluster takes the rows of a few groups of one sample, every block a part of the rows, which stay in its shared
//            memory; the blocks exchange their statistics through distributed shared memory.
//   stream   slabs that do not fit, and tensors above a size (make_norm_plan): one kernel for the statistics of parts, one that reads
//            the elements again (from L2 where they are still there).
// Measured: rows 26.8 us for 8192 x 4096 in bf16 (5 TB/s; the floor is 20.5, what is left is the two sums over lanes in a row and the few samples
// that a thread has under way), with the backward pass 92.  Stream, forward, 8 x 4096 x 512 in fp16 28 us; training step of 32 x 3136 x 256 in bf16 91.3 us:
// 14 + 26 forward, 32 + 32 backward, 5.6 for the parameters' gradients (each alone, under a profiler).  The output kernel of the forward pass keeps the special-function
// units busy for 64 % of its time, with 78 registers and so three blocks an SM, whose warps wait for them in turn; the others wait for latencies, at 40 to 48 % of memory's rate.
// Where the plan falls short: it goes by bytes alone.  Wide groups of single rows are streams or slabs of one row (8192 x 4096 in one group, bf16: 133 us
// forward, 704 with the backward pass, whose partial sums are one a sample), and a block takes one sample however short (16384 x 4 x 512: 1.2 and 3.7 ms).
// Statistics of a part are taken around one of its own values and joined by counts and means, so that a mean far
// from zero costs no digits.
#include <cooperative_groups.h>

#include "seq_common.cuh"

namespace conv2d_b200 {
namespace {

namespace cg = cooperative_groups;

constexpr int kRowThreads = 256;        // rows
constexpr int kThreads = 256, kWarps = kThreads / 32;        // slab, stream
constexpr int kRing = 4;                // groups of a ring
// Rows of a group: two (four take the backward pass to 240 registers); eight of single elements, whose loads, where they are too narrow to be copied
// asynchronously, wait for memory once a group (1 x 5795 x 4064 in groups of 127 channels, bf16, forward: 151 us with two, 79 so).
template <int V> constexpr int kGroup = V == 1 ? 8 : 2;

template <typename T>
struct NormArgs {
    const T *x, *dy;
    const float *gamma, *beta;
    T *y, *dx;
    float *mean, *rstd;
    float4* part_stats;                 // [N][G][parts]: what the parts of a slab have found (stream)
    float* channels;                    // [N * parts or chunks][2][C]: partial sums of dbeta, dgamma
    int N, S, C, G, E;
    long long ldx, ldy, lddy, lddx;
    float eps;
    int act;
    int lanes, chunks, chunk;           // rows: lanes of a group; chunks of samples, samples of a chunk
    int tile_groups, tiles, parts, part_rows, ev;   // ev: packs of a group
};

// ------------------------------------------------------------------------------------------------------------- rows

__device__ __forceinline__ float lanes_sum(float v, int lanes)
{
    for (int m = 1; m < lanes; m *= 2) v += __shfl_xor_sync(0xffffffffu, v, m);
    return v;
}
// Several sums over the same lanes, under way together.
template <int N> __device__ __forceinline__ void lanes_sums(float (&v)[N], int lanes)
{
#pragma unroll
    for (int m = 1; m < 32; m *= 2) {
        if (m >= lanes) break;
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], m);
    }
}

template <int V>
__device__ __forceinline__ void load_params(const float* p, float dflt, int c, bool real, float (&out)[V])
{
#pragma unroll
    for (int i = 0; i < V; ++i) out[i] = p && real ? p[c + i] : dflt;
}

// gamma and beta of a pack, 1 and 0 where there are none
template <int V>
__device__ __forceinline__ void load_scale(const float* gamma, const float* beta, int c, bool real, float2 (&g)[kPairs<V>], float2 (&b)[kPairs<V>])
{
    float gf[V], bf[V];
    load_params<V>(gamma, 1.f, c, real, gf);
    load_params<V>(beta, 0.f, c, real, bf);
#pragma unroll
    for (int k = 0; k < kPairs<V>; ++k) {
        g[k] = make_float2(gf[2 * k], V > 1 ? gf[V > 1 ? 2 * k + 1 : 0] : 0.f);
        b[k] = make_float2(bf[2 * k], V > 1 ? bf[V > 1 ? 2 * k + 1 : 0] : 0.f);
    }
}

// A thread's packs of a chunk of samples: NV of one group, lane l the packs l, l + lanes, ..; they come in through a ring of four groups of ROWS samples.
template <typename T, int V, int NV, int ROWS>
struct SampleRing {
    static constexpr int RING = 4, bytes = V * (int)sizeof(T);
    static constexpr bool async = bytes >= 4;
    static constexpr size_t smem = async ? (size_t)RING * ROWS * NV * kRowThreads * bytes : 0;
    unsigned char* mine;
    const T* p;                         // of the chunk's first sample, pack 0
    long long ld;
    int apart;                          // elements from one of the thread's packs to the next
    __device__ void issue(int q, int n, int count, const bool (&real)[NV]) const
    {
        if (!async) return;
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            const bool in = n + r < count;
            const T* from = p + (in ? (n + r) * ld : 0);
#pragma unroll
            for (int k = 0; k < NV; ++k)
                copy_async<async ? bytes : 4>(mine + (size_t)(((q & (RING - 1)) * ROWS + r) * NV + k) * (kRowThreads * bytes), from + (real[k] ? k * apart : 0), in && real[k]);
        }
    }
    __device__ Pack<T, V> get(int q, int n, int r, int k, int count, const bool (&real)[NV]) const
    {
        if (async) return *reinterpret_cast<const Pack<T, V>*>(mine + (size_t)(((q & (RING - 1)) * ROWS + r) * NV + k) * (kRowThreads * bytes));
        return n + r < count && real[k] ? load_pack<T, V>(p + (n + r) * ld + k * apart) : zero_pack<T, V>();
    }
};

template <typename T, int V, int NV, int ROWS>
__global__ void __launch_bounds__(kRowThreads) norm_rows_fwd_kernel(const NormArgs<T> a)
{
    constexpr int P = kPairs<V>;
    ptx::grid_dep_wait();
    extern __shared__ float4 smem4[];
    const unsigned cols = (kRowThreads + (unsigned)a.G * a.lanes - 1) / kRowThreads;
    const unsigned col = blockIdx.x % cols * kRowThreads + threadIdx.x;
    const int g = (int)(col / a.lanes), l = (int)(col % a.lanes);
    const long long n0 = (long long)(blockIdx.x / cols) * a.chunk;
    const int count = (int)min((long long)a.chunk, a.N - n0), c = g * a.E + l * V, apart = a.lanes * V;
    bool real[NV];
    float2 gamma[NV][P], beta[NV][P];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        real[k] = g < a.G && (l + k * a.lanes) * V < a.E;
        load_scale<V>(a.gamma, a.beta, c + k * apart, real[k], gamma[k], beta[k]);
    }
    using Ring = SampleRing<T, V, NV, ROWS>;
    const Ring x{reinterpret_cast<unsigned char*>(smem4) + threadIdx.x * Ring::bytes, a.x + (real[0] ? n0 * a.ldx + c : 0), a.ldx, apart};
#pragma unroll
    for (int q = 0; q < Ring::RING - 1; ++q) {
        x.issue(q, q * ROWS, count, real);
        copies_commit();
    }
    const float inv = 1.f / a.E;
    const bool first = l == 0 && g < a.G;
    T* y = a.y + n0 * a.ldy + c;
    float *mean_out = a.mean && first ? a.mean + n0 * a.G + g : nullptr, *rstd_out = a.rstd && first ? a.rstd + n0 * a.G + g : nullptr;
    int q = 0;
#pragma unroll 1
    for (int n = 0; n < count; n += ROWS, ++q) {
        copies_wait<Ring::RING - 2>();
        float2 v[ROWS][NV][P];
        float mean[ROWS], rstd[ROWS];
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            float2 s = both(0.f);
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                pairs<T, V>(x.get(q, n, r, k, count, real), v[r][k]);
#pragma unroll
                for (int i = 0; i < P; ++i) s = __fadd2_rn(s, v[r][k][i]);
            }
            mean[r] = V > 1 ? s.x + s.y : s.x;
        }
        x.issue(q + Ring::RING - 1, n + (Ring::RING - 1) * ROWS, count, real);
        copies_commit();
        lanes_sums(mean, a.lanes);
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            mean[r] *= inv;
            float2 s = both(0.f);
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                float2 t = both(0.f);
#pragma unroll
                for (int i = 0; i < P; ++i) {
                    v[r][k][i] = __fadd2_rn(v[r][k][i], both(-mean[r]));
                    t = __ffma2_rn(v[r][k][i], v[r][k][i], t);
                }
                if (real[k]) s = __fadd2_rn(s, t);
            }
            rstd[r] = V > 1 ? s.x + s.y : s.x;
        }
        lanes_sums(rstd, a.lanes);
        float o[ROWS * NV * 2 * P];
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            rstd[r] = rsqrtf(fmaf(rstd[r], inv, a.eps));
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int i = 0; i < P; ++i) {
                    const float2 w = __ffma2_rn(__fmul2_rn(v[r][k][i], both(rstd[r])), gamma[k][i], beta[k][i]);
                    o[2 * ((r * NV + k) * P + i)] = w.x, o[2 * ((r * NV + k) * P + i) + 1] = w.y;
                }
        }
        activate(o, a.act);
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            if (n + r >= count) break;
            if (mean_out) *mean_out = mean[r], mean_out += a.G;
            if (rstd_out) *rstd_out = rstd[r], rstd_out += a.G;
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                float2 w[P];
#pragma unroll
                for (int i = 0; i < P; ++i) w[i] = make_float2(o[2 * ((r * NV + k) * P + i)], o[2 * ((r * NV + k) * P + i) + 1]);
                if (real[k]) store_pack(y + k * apart, pack_of<T, V>(w));
            }
            y += a.ldy;
        }
    }
}

template <typename T, int V, int NV, int ROWS>
__global__ void __launch_bounds__(kRowThreads) norm_rows_bwd_kernel(const NormArgs<T> a)
{
    constexpr int P = kPairs<V>;
    ptx::grid_dep_wait();
    extern __shared__ float4 smem4[];
    const unsigned cols = (kRowThreads + (unsigned)a.G * a.lanes - 1) / kRowThreads;
    const unsigned col = blockIdx.x % cols * kRowThreads + threadIdx.x;
    const int g = (int)(col / a.lanes), l = (int)(col % a.lanes);
    const long long chunk = blockIdx.x / cols, n0 = chunk * a.chunk;
    const int count = (int)min((long long)a.chunk, a.N - n0), c = g * a.E + l * V, apart = a.lanes * V;
    bool real[NV];
    float2 gamma[NV][P], beta[NV][P], sum1[NV][P], sum2[NV][P];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        real[k] = g < a.G && (l + k * a.lanes) * V < a.E;
        load_scale<V>(a.gamma, a.beta, c + k * apart, real[k], gamma[k], beta[k]);
#pragma unroll
        for (int i = 0; i < P; ++i) sum1[k][i] = sum2[k][i] = both(0.f);
    }
    using Ring = SampleRing<T, V, NV, ROWS>;
    const Ring x{reinterpret_cast<unsigned char*>(smem4) + threadIdx.x * Ring::bytes, a.x + (real[0] ? n0 * a.ldx + c : 0), a.ldx, apart};
    const Ring dy{x.mine + Ring::smem, a.dy + (real[0] ? n0 * a.lddy + c : 0), a.lddy, apart};
#pragma unroll
    for (int q = 0; q < Ring::RING - 1; ++q) {
        x.issue(q, q * ROWS, count, real);
        dy.issue(q, q * ROWS, count, real);
        copies_commit();
    }
    const float inv = 1.f / a.E;
    const float *mean_in = a.mean + n0 * a.G + (g < a.G ? g : 0), *rstd_in = a.rstd + n0 * a.G + (g < a.G ? g : 0);
    T* dx = a.dx + n0 * a.lddx + c;
    float mean[ROWS], rstd[ROWS];                            // of the next samples, read one group ahead
    auto read = [&](int n) {
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            const bool in = n + r < count;
            mean[r] = in ? mean_in[(long long)(n + r) * a.G] : 0.f;
            rstd[r] = in ? rstd_in[(long long)(n + r) * a.G] : 0.f;
        }
    };
    read(0);
    int q = 0;
#pragma unroll 1
    for (int n = 0; n < count; n += ROWS, ++q) {
        copies_wait<Ring::RING - 2>();
        float2 xn[ROWS][NV][P];
        float d[ROWS * NV * 2 * P], pre[ROWS * NV * 2 * P], m[2 * ROWS], scale[ROWS];
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            scale[r] = rstd[r];
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                float2 w[P];
                pairs<T, V>(x.get(q, n, r, k, count, real), xn[r][k]);
                pairs<T, V>(dy.get(q, n, r, k, count, real), w);     // (zero outside the group and behind the last sample)
#pragma unroll
                for (int i = 0; i < P; ++i) {
                    const int at = 2 * ((r * NV + k) * P + i);
                    xn[r][k][i] = __fmul2_rn(__fadd2_rn(xn[r][k][i], both(-mean[r])), both(rstd[r]));
                    const float2 z = __ffma2_rn(xn[r][k][i], gamma[k][i], beta[k][i]);
                    d[at] = w[i].x, d[at + 1] = w[i].y, pre[at] = z.x, pre[at + 1] = z.y;
                }
            }
        }
        x.issue(q + Ring::RING - 1, n + (Ring::RING - 1) * ROWS, count, real);
        dy.issue(q + Ring::RING - 1, n + (Ring::RING - 1) * ROWS, count, real);
        copies_commit();
        if (n + ROWS < count) read(n + ROWS);
        times_slope(d, pre, a.act);
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            float2 m1 = both(0.f), m2 = both(0.f);
            if (n + r < count) {
#pragma unroll
                for (int k = 0; k < NV; ++k) {
                    if (!real[k]) continue;
#pragma unroll
                    for (int i = 0; i < P; ++i) {
                        const int at = 2 * ((r * NV + k) * P + i);
                        float2 e = make_float2(d[at], d[at + 1]);
                        sum1[k][i] = __fadd2_rn(sum1[k][i], e);
                        sum2[k][i] = __ffma2_rn(e, xn[r][k][i], sum2[k][i]);
                        e = __fmul2_rn(e, gamma[k][i]);
                        m1 = __fadd2_rn(m1, e);
                        m2 = __ffma2_rn(e, xn[r][k][i], m2);
                        d[at] = e.x, d[at + 1] = e.y;
                    }
                }
            }
            m[2 * r] = V > 1 ? m1.x + m1.y : m1.x, m[2 * r + 1] = V > 1 ? m2.x + m2.y : m2.x;
        }
        lanes_sums(m, a.lanes);
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            if (n + r >= count) break;
            const float2 m1 = both(-m[2 * r] * inv), m2 = both(-m[2 * r + 1] * inv);
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                float2 w[P];
#pragma unroll
                for (int i = 0; i < P; ++i) {
                    const int at = 2 * ((r * NV + k) * P + i);
                    w[i] = __fmul2_rn(both(scale[r]), __ffma2_rn(xn[r][k][i], m2, __fadd2_rn(make_float2(d[at], d[at + 1]), m1)));
                }
                if (real[k]) store_pack(dx + k * apart, pack_of<T, V>(w));
            }
            dx += a.lddx;
        }
    }
    if (!a.channels) return;
    float* out = a.channels + (size_t)chunk * 2 * a.C + c;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        if (!real[k]) continue;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            out[k * apart + i] = i % 2 ? sum1[k][i / 2].y : sum1[k][i / 2].x;
            out[a.C + k * apart + i] = i % 2 ? sum2[k][i / 2].y : sum2[k][i / 2].x;
        }
    }
}

// ----------------------------------------------------------------------------------------------------- slab and stream

// What a block takes: `groups` groups of sample n from channel c0 on, rows r0 .. r1.  A thread keeps to one pack of channels (pack, of group `group`) and
// takes every `step`th row from `first` on, `count` in all; wider rows than the block has threads (one group then) are taken a block's
// width at a time, in `turns`.  The second kernel of a stream walks its rows backwards: what the first has read last is what L2 still holds (32 x 3136 x 512
// in bf16 forward 70.6 us, 68.6 so; no difference for tensors that fit).
template <typename T, int V, bool BACKWARDS>
struct Part {
    int part, groups, g0, c0, packs, ev, step, turns, r0, r1, pack, group, first, count;
    long long n;
    __device__ explicit Part(const NormArgs<T>& a)
    {
        unsigned bx = blockIdx.x;
        part = (int)(bx % a.parts);
        bx /= a.parts;
        const int tile = (int)(bx % a.tiles), tid = threadIdx.x;
        n = bx / a.tiles;
        g0 = tile * a.tile_groups;
        groups = min(a.tile_groups, a.G - g0);
        c0 = g0 * a.E;
        ev = a.ev;
        packs = groups * ev;
        r0 = min(part * a.part_rows, a.S), r1 = min(r0 + a.part_rows, a.S);
        step = 1, turns = 1, first = r0, pack = tid, group = 0;
        if (packs <= kThreads) {
            const int row = tid / packs;
            step = kThreads / packs;
            pack = tid - row * packs;
            group = pack / ev;
            first = r0 + row;
            if (row >= step) pack = -1;
        } else {
            turns = (packs + kThreads - 1) / kThreads;
        }
        count = pack >= 0 && first < r1 ? (r1 - first + step - 1) / step : 0;
        if (BACKWARDS && count) first += (count - 1) * step;
        if (V * sizeof(T) >= 4) first = min(first, a.S - 1);    // (a thread without rows, too, names addresses within the tensor: its copies of no bytes have one)
    }
    // rows from one of the thread's to its next
    __device__ long long stride() const { return BACKWARDS ? -step : step; }
    // the pack of this thread in turn q, or -1; and its rows then
    __device__ int pack_of(int q) const
    {
        const int p = turns == 1 ? pack : pack + q * kThreads;
        return p < packs ? p : -1;
    }
    __device__ int count_of(int q) const { return pack_of(q) >= 0 ? count : 0; }
};

// Sums over the threads that hold group gi of what `value` gives for a thread index, by one warp.
template <int N, typename P, typename F>
__device__ __forceinline__ void group_sums(const P& p, int gi, float (&s)[N], F value)
{
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int i = 0; i < N; ++i) s[i] = 0.f;
    if (p.turns == 1) {
        // lanes by packs of the group (the next power of two) and rows
        const int shift = p.ev >= 32 ? 5 : 32 - __clz(p.ev - 1), c0 = lane & ((1 << shift) - 1);
        for (int row = lane >> shift; row < p.step; row += 32 >> shift)
            for (int c = c0; c < p.ev; c += 1 << shift) value(row * p.packs + gi * p.ev + c, s);
    } else {
        for (int k = lane; k < kThreads; k += 32) value(k, s);
    }
    lanes_sums(s, 32);
}

enum { kSlab = 0, kStreamStats = 1, kStreamApply = 2 };

// Slots that a thread needs for its rows: whole groups of `group`.
__host__ __device__ constexpr int thread_slots(int rows, int group) { return (rows + group - 1) / group * group; }

// The packs of one tensor that a thread takes: rows first, first + step, .. of its channels.  A slab's stay in shared memory, all under way at once;
// a stream's go through a ring.
template <typename T, int V, bool KEEP>
struct ThreadRows {
    using Ring = RowRing<T, V, kThreads, kGroup<V>, kRing>;
    static constexpr int bytes = V * (int)sizeof(T);
    Ring ring;                          // (KEEP: mine is the first of all slots)
    int count;
    __device__ void begin() const
    {
        if (KEEP) {
            const T* from = ring.p;
            unsigned char* to = ring.mine;
#pragma unroll 4
            for (int i = 0; i < count; ++i, from += ring.ld, to += kThreads * bytes) {
                if (Ring::async) copy_async<Ring::async ? bytes : 4>(to, from, true);
                else store_pack(reinterpret_cast<T*>(to), load_pack<T, V>(from));
            }
        }
    }
    __device__ Pack<T, V> get(int q, int i, int j) const
    {
        // (slots are there for whole groups; what lies behind the last row is not used)
        if (KEEP) return *reinterpret_cast<const Pack<T, V>*>(ring.mine + i * (kThreads * bytes) + j * (kThreads * bytes));
        return ring.get(q, i, j, count);
    }
};
template <typename T, int V> constexpr size_t ring_bytes = RowRing<T, V, kThreads, kGroup<V>, kRing>::smem;

// Walks `count` rows of the thread in groups: `issue(q, i)` starts the copies of group q, `take(q, i, whole)` uses it.
template <bool KEEP, int GROUP, typename Issue, typename Take>
__device__ __forceinline__ void walk_rows(int count, Issue issue, Take take)
{
    if (!KEEP) {
#pragma unroll
        for (int q = 0; q < kRing - 1; ++q) {
            issue(q, q * GROUP);
            copies_commit();
        }
    }
    int q = 0;
#pragma unroll 1
    for (int i = 0; i + GROUP <= count; i += GROUP, ++q) {
        if (!KEEP) copies_wait<kRing - 2>();
        take(q, i, Whole());
        if (!KEEP) {
            issue(q + kRing - 1, i + (kRing - 1) * GROUP);
            copies_commit();
        }
    }
    if (!KEEP) copies_wait<0>();
    if (q * GROUP < count) take(q, q * GROUP, Cut());
}

template <typename T, int V, int MODE>
__global__ void __launch_bounds__(kThreads) norm_slab_fwd_kernel(const NormArgs<T> a)
{
    constexpr int P = kPairs<V>;
    constexpr bool KEEP = MODE == kSlab;
    ptx::grid_dep_wait();
    extern __shared__ float4 smem4[];
    __shared__ float ecount[kThreads], emean[kThreads], em2[kThreads];
    float4* gstat = smem4;                                   // [tile_groups] count, mean, sum of squares about it; then mean, rstd
    float2* gnorm = reinterpret_cast<float2*>(gstat + a.tile_groups);
    unsigned char* rows = reinterpret_cast<unsigned char*>(reinterpret_cast<float4*>(gnorm) + (a.tile_groups + 1) / 2);
    const Part<T, V, MODE == kStreamApply> p(a);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int g0 = p.g0;
    const T* x = a.x + (p.n * a.S + p.first) * a.ldx + p.c0;
    using Rows = ThreadRows<T, V, KEEP>;
    auto rows_of = [&](int q) {
        Rows r;
        r.count = p.count_of(q);
        // (turns take whole rows: a part's rows each)
        r.ring = {rows + ((KEEP ? q * thread_slots(a.part_rows, kGroup<V>) * kThreads : 0) + threadIdx.x) * Rows::bytes, x + (r.count ? p.pack_of(q) * V : 0), p.stride() * a.ldx};
        return r;
    };

    if (MODE != kStreamApply) {
        if (KEEP) {
            for (int q = 0; q < p.turns; ++q) rows_of(q).begin();
            copies_commit();
            copies_wait<0>();
        }
        float2 s1 = both(0.f), s2 = both(0.f);
        float shift = 0.f;
        int count = 0;
        for (int q = 0; q < p.turns; ++q) {
            const Rows r = rows_of(q);
            walk_rows<KEEP, kGroup<V>>(r.count, [&](int g, int i) { r.ring.issue(g, i, r.count); }, [&](int g, int i, auto whole) {
                float2 v[kGroup<V>][P];
#pragma unroll
                for (int j = 0; j < kGroup<V>; ++j) pairs<T, V>(r.get(g, i, j), v[j]);
                if (i == 0 && q == 0) shift = v[0][0].x;
#pragma unroll
                for (int j = 0; j < kGroup<V>; ++j) {
                    if (!decltype(whole)::value && i + j >= r.count) break;
#pragma unroll
                    for (int k = 0; k < P; ++k) {
                        const float2 d = __fadd2_rn(v[j][k], both(-shift));
                        s1 = __fadd2_rn(s1, d);
                        s2 = __ffma2_rn(d, d, s2);
                    }
                }
            });
            count += V * r.count;
        }
        if (V == 1) s1.y = s2.y = 0.f;
        const float cnt = (float)count, t1 = s1.x + s1.y, off = count ? t1 / cnt : 0.f;
        ecount[threadIdx.x] = cnt;
        emean[threadIdx.x] = shift + off;
        em2[threadIdx.x] = (s2.x + s2.y) - t1 * off;
        __syncthreads();
        for (int gi = warp; gi < p.groups; gi += kWarps) {
            float t[2], q[1];
            group_sums(p, gi, t, [&](int k, float (&o)[2]) { o[0] += ecount[k], o[1] = fmaf(ecount[k], emean[k], o[1]); });
            const float n = t[0], mean = n > 0.f ? t[1] / n : 0.f;
            group_sums(p, gi, q, [&](int k, float (&o)[1]) {
                const float d = emean[k] - mean;
                if (ecount[k] > 0.f) o[0] += fmaf(ecount[k] * d, d, em2[k]);
            });
            const float m2 = q[0];
            if (lane == 0) {
                const float4 st = make_float4(n, mean, m2, 0.f);
                if (KEEP) gstat[gi] = st;
                else a.part_stats[((size_t)p.n * a.G + g0 + gi) * a.parts + p.part] = st;
            }
        }
        if (MODE == kStreamStats) return;
    }
    if (KEEP) cg::this_cluster().sync();
    for (int gi = warp; gi < p.groups; gi += kWarps) {
        auto stat = [&](int k) {
            if (KEEP) return cg::this_cluster().map_shared_rank(gstat, k)[gi];
            return a.part_stats[((size_t)p.n * a.G + g0 + gi) * a.parts + k];
        };
        float n = 0.f, base = 0.f, m2 = 0.f;
        for (int k = lane; k < a.parts; k += 32) {
            const float4 st = stat(k);
            n += st.x;
            base = fmaf(st.x, st.y, base);
        }
        n = lanes_sum(n, 32);
        const float mean = lanes_sum(base, 32) / n;
        for (int k = lane; k < a.parts; k += 32) {
            const float4 st = stat(k);
            const float d = st.y - mean;
            if (st.x > 0.f) m2 += fmaf(st.x * d, d, st.z);
        }
        const float rstd = rsqrtf(lanes_sum(m2, 32) / n + a.eps);
        if (lane == 0) {
            gnorm[gi] = make_float2(mean, rstd);
            if (p.part == 0) {
                if (a.mean) a.mean[p.n * a.G + g0 + gi] = mean;
                if (a.rstd) a.rstd[p.n * a.G + g0 + gi] = rstd;
            }
        }
    }
    // the statistics stay readable until all blocks of the cluster have them
    if (KEEP) cg::this_cluster().sync();
    else __syncthreads();
    const long long ystep = p.stride() * a.ldy;
    for (int q = 0; q < p.turns; ++q) {
        const Rows r = rows_of(q);
        if (r.count == 0) continue;
        T* y = a.y + (p.n * a.S + p.first) * a.ldy + p.c0 + p.pack_of(q) * V;
        const int pk = p.pack_of(q);
        const float2 st = gnorm[p.group];
        float2 scale[P], add[P];
        load_scale<V>(a.gamma, a.beta, p.c0 + pk * V, true, scale, add);
#pragma unroll
        for (int k = 0; k < P; ++k) scale[k] = __fmul2_rn(scale[k], both(st.y));
        walk_rows<KEEP, kGroup<V>>(r.count, [&](int g, int i) { r.ring.issue(g, i, r.count); }, [&](int g, int i, auto whole) {
            float o[kGroup<V> * 2 * P];
#pragma unroll
            for (int j = 0; j < kGroup<V>; ++j) {
                float2 v[P];
                pairs<T, V>(r.get(g, i, j), v);
#pragma unroll
                for (int k = 0; k < P; ++k) {
                    v[k] = __ffma2_rn(__fadd2_rn(v[k], both(-st.x)), scale[k], add[k]);
                    o[2 * (j * P + k)] = v[k].x, o[2 * (j * P + k) + 1] = v[k].y;
                }
            }
            activate(o, a.act);
#pragma unroll
            for (int j = 0; j < kGroup<V>; ++j) {
                float2 v[P];
#pragma unroll
                for (int k = 0; k < P; ++k) v[k] = make_float2(o[2 * (j * P + k)], o[2 * (j * P + k) + 1]);
                if (decltype(whole)::value || i + j < r.count) store_pack(y, pack_of<T, V>(v));
                y += ystep;
            }
        });
    }
}

template <typename T, int V, int MODE>
__global__ void __launch_bounds__(kThreads, 2) norm_slab_bwd_kernel(const NormArgs<T> a)
{
    constexpr int P = kPairs<V>;
    constexpr bool KEEP = MODE == kSlab;
    ptx::grid_dep_wait();
    extern __shared__ float4 smem4[];
    __shared__ float e1[kThreads], e2[kThreads];
    float4* gsum = smem4;                                    // [tile_groups] sums over the part of gamma d and gamma d x^
    float2* gmean = reinterpret_cast<float2*>(gsum + a.tile_groups);
    float* csum = reinterpret_cast<float*>(reinterpret_cast<float4*>(gmean) + (a.tile_groups + 1) / 2);       // [2][kThreads * V]
    unsigned char* rows = reinterpret_cast<unsigned char*>(csum + (MODE == kStreamApply ? 0 : 2 * kThreads * V));
    const Part<T, V, MODE == kStreamApply> p(a);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int g0 = p.g0, width = p.packs * V, kept = KEEP ? thread_slots(p.turns == 1 ? (a.part_rows + p.step - 1) / p.step : a.part_rows, kGroup<V>) : 0;
    const T* x = a.x + (p.n * a.S + p.first) * a.ldx + p.c0;
    const T* dy = a.dy + (p.n * a.S + p.first) * a.lddy + p.c0;
    using Rows = ThreadRows<T, V, KEEP>;
    auto rows_of = [&](int q, bool second) {                 // of x, or of dy
        const size_t before = KEEP ? ((size_t)second * p.turns + q) * kept * kThreads * Rows::bytes : second * ring_bytes<T, V>;
        Rows r;
        r.count = p.count_of(q);
        r.ring = {rows + before + threadIdx.x * Rows::bytes, (second ? dy : x) + (r.count ? p.pack_of(q) * V : 0), p.stride() * (second ? a.lddy : a.ldx)};
        return r;
    };
    // x^ and d of the rows of a group
    struct Params { float2 gamma[P], beta[P]; float mean, rstd; };
    auto params_of = [&](int pk) {
        Params r;
        const int g = g0 + p.group;
        r.mean = a.mean[p.n * a.G + g], r.rstd = a.rstd[p.n * a.G + g];
        load_scale<V>(a.gamma, a.beta, p.c0 + pk * V, true, r.gamma, r.beta);
        return r;
    };
    auto terms = [&](const Params& m, const Rows& rx, const Rows& rg, int g, int i, float2 (&xn)[kGroup<V>][P], float (&d)[kGroup<V> * 2 * P]) {
        float pre[kGroup<V> * 2 * P];
#pragma unroll
        for (int j = 0; j < kGroup<V>; ++j) {
            float2 w[P];
            pairs<T, V>(rx.get(g, i, j), xn[j]);
            pairs<T, V>(rg.get(g, i, j), w);
#pragma unroll
            for (int k = 0; k < P; ++k) {
                xn[j][k] = __fmul2_rn(__fadd2_rn(xn[j][k], both(-m.mean)), both(m.rstd));
                const float2 v = __ffma2_rn(xn[j][k], m.gamma[k], m.beta[k]);
                pre[2 * (j * P + k)] = v.x, pre[2 * (j * P + k) + 1] = v.y;
                d[2 * (j * P + k)] = w[k].x, d[2 * (j * P + k) + 1] = w[k].y;
            }
        }
        times_slope(d, pre, a.act);
    };

    if (MODE != kStreamApply) {
        if (KEEP) {
            for (int q = 0; q < p.turns; ++q) rows_of(q, false).begin(), rows_of(q, true).begin();
            copies_commit();
            copies_wait<0>();
        }
        float m1 = 0.f, m2 = 0.f;
        for (int q = 0; q < p.turns; ++q) {
            const Rows rx = rows_of(q, false), rg = rows_of(q, true);
            const int pk = p.pack_of(q);
            float2 s1[P], s2[P];
#pragma unroll
            for (int k = 0; k < P; ++k) s1[k] = s2[k] = both(0.f);
            if (rx.count) {
                const Params m = params_of(pk);
                walk_rows<KEEP, kGroup<V>>(rx.count, [&](int g, int i) { rx.ring.issue(g, i, rx.count), rg.ring.issue(g, i, rx.count); }, [&](int g, int i, auto whole) {
                    float2 xn[kGroup<V>][P];
                    float d[kGroup<V> * 2 * P];
                    terms(m, rx, rg, g, i, xn, d);
#pragma unroll
                    for (int j = 0; j < kGroup<V>; ++j) {
                        if (!decltype(whole)::value && i + j >= rx.count) break;
#pragma unroll
                        for (int k = 0; k < P; ++k) {
                            const float2 e = make_float2(d[2 * (j * P + k)], d[2 * (j * P + k) + 1]);
                            s1[k] = __fadd2_rn(s1[k], e);
                            s2[k] = __ffma2_rn(e, xn[j][k], s2[k]);
                        }
                    }
                });
#pragma unroll
                for (int k = 0; k < P; ++k) {
                    m1 = fmaf(m.gamma[k].x, s1[k].x, m1), m2 = fmaf(m.gamma[k].x, s2[k].x, m2);
                    if (V > 1) m1 = fmaf(m.gamma[k].y, s1[k].y, m1), m2 = fmaf(m.gamma[k].y, s2[k].y, m2);
                }
            }
            if (a.channels) {
                float* out = a.channels + ((size_t)p.n * a.parts + p.part) * 2 * a.C + p.c0;
                if (p.step == 1) {
                    if (pk >= 0) {
#pragma unroll
                        for (int i = 0; i < V; ++i) {
                            out[pk * V + i] = i % 2 ? s1[i / 2].y : s1[i / 2].x;
                            out[a.C + pk * V + i] = i % 2 ? s2[i / 2].y : s2[i / 2].x;
                        }
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        csum[threadIdx.x * V + i] = i % 2 ? s1[i / 2].y : s1[i / 2].x;
                        csum[(kThreads + threadIdx.x) * V + i] = i % 2 ? s2[i / 2].y : s2[i / 2].x;
                    }
                    __syncthreads();
                    for (int k = threadIdx.x; k < 2 * width; k += kThreads) {
                        const int which = k / width, c = k % width;
                        float s = 0.f;
                        for (int j = 0; j < p.step; ++j) s += csum[which * kThreads * V + j * width + c];
                        out[which * a.C + c] = s;
                    }
                }
            }
        }
        e1[threadIdx.x] = m1, e2[threadIdx.x] = m2;
        __syncthreads();
        for (int gi = warp; gi < p.groups; gi += kWarps) {
            float t[2];
            group_sums(p, gi, t, [&](int k, float (&o)[2]) { o[0] += e1[k], o[1] += e2[k]; });
            const float t1 = t[0], t2 = t[1];
            if (lane == 0) {
                const float4 st = make_float4(t1, t2, 0.f, 0.f);
                if (KEEP) gsum[gi] = st;
                else a.part_stats[((size_t)p.n * a.G + g0 + gi) * a.parts + p.part] = st;
            }
        }
        if (MODE == kStreamStats) return;
    }
    if (KEEP) cg::this_cluster().sync();
    for (int gi = warp; gi < p.groups; gi += kWarps) {
        float t1 = 0.f, t2 = 0.f;
        for (int k = lane; k < a.parts; k += 32) {
            const float4 st = KEEP ? cg::this_cluster().map_shared_rank(gsum, k)[gi] : a.part_stats[((size_t)p.n * a.G + g0 + gi) * a.parts + k];
            t1 += st.x, t2 += st.y;
        }
        t1 = lanes_sum(t1, 32), t2 = lanes_sum(t2, 32);
        const float inv = 1.f / ((float)a.S * a.E);
        if (lane == 0) gmean[gi] = make_float2(t1 * inv, t2 * inv);
    }
    if (KEEP) cg::this_cluster().sync();
    else __syncthreads();
    const long long dxstep = p.stride() * a.lddx;
    for (int q = 0; q < p.turns; ++q) {
        const Rows rx = rows_of(q, false), rg = rows_of(q, true);
        if (rx.count == 0) continue;
        const int pk = p.pack_of(q);
        const float2 mm = gmean[p.group];
        const Params m = params_of(pk);
        T* dx = a.dx + (p.n * a.S + p.first) * a.lddx + p.c0 + pk * V;
        walk_rows<KEEP, kGroup<V>>(rx.count, [&](int g, int i) { rx.ring.issue(g, i, rx.count), rg.ring.issue(g, i, rx.count); }, [&](int g, int i, auto whole) {
            float2 xn[kGroup<V>][P];
            float d[kGroup<V> * 2 * P];
            terms(m, rx, rg, g, i, xn, d);
#pragma unroll
            for (int j = 0; j < kGroup<V>; ++j) {
                float2 o[P];
#pragma unroll
                for (int k = 0; k < P; ++k) {
                    const float2 e = __ffma2_rn(make_float2(d[2 * (j * P + k)], d[2 * (j * P + k) + 1]), m.gamma[k], both(-mm.x));
                    o[k] = __fmul2_rn(both(m.rstd), __ffma2_rn(xn[j][k], both(-mm.y), e));
                }
                if (decltype(whole)::value || i + j < rx.count) store_pack(dx, pack_of<T, V>(o));
                dx += dxstep;
            }
        });
    }
}

// --------------------------------------------------------------------------------------------------------------- plan

constexpr size_t kSlabBytes = 64 * 1024;      // rows that a block keeps: three blocks an SM
constexpr int kMaxCluster = 8, kSms = 148;

// Slots of 16 bytes (of an element, without packs) that the threads of a slab's block need, in bytes: threads that a row leaves over have some, too.
size_t slab_bytes(int part_rows, int packs, int pack_bytes, int group, bool bwd)
{
    const int step = packs <= kThreads ? kThreads / packs : 1, turns = packs <= kThreads ? 1 : (packs + kThreads - 1) / kThreads;
    return (size_t)thread_slots((part_rows + step - 1) / step, group) * turns * kThreads * pack_bytes * (bwd ? 2 : 1);
}

// How a call is cut.  The sizes decide, and whether rows can be moved in packs of 16 bytes; the workspace has room for either.
struct NormPlan {
    bool rows, slab;
    int lanes, nv, chunks, chunk;             // rows
    int tile_groups, tiles, parts, part_rows; // slab, stream
    size_t stats, channels;                   // floats of workspace
};

NormPlan make_norm_plan(int N, int S, int C, int G, int esize, int V, bool bwd)
{
    NormPlan p{};
    const int E = C / G, ev = E / V;
    int lanes = 1;
    while (lanes < 32 && lanes < ev) lanes *= 2;
    const int nv = (ev + lanes - 1) / lanes;
    if (S == 1 && nv <= 4) {
        p.rows = true;
        p.lanes = lanes;
        p.nv = nv <= 1 ? 1 : nv <= 2 ? 2 : 4;
        // as many chunks of samples as fill the machine (eight blocks an SM), at least four samples each
        const long long cols = ((long long)G * lanes + kRowThreads - 1) / kRowThreads;
        long long chunks = (8LL * kSms + cols - 1) / cols;
        if (chunks > (N + 3) / 4) chunks = (N + 3) / 4;
        p.chunk = (int)((N + chunks - 1) / chunks);
        p.chunks = (N + p.chunk - 1) / p.chunk;
        p.channels = bwd ? (size_t)p.chunks * 2 * C : 0;
        return p;
    }
    // groups of a tile: rows of 128 bytes or more, of 64 or 32 where the slab does not fit else, but not more packs than threads
    const auto tile = [&](int bytes) {
        int n = (bytes + E * esize - 1) / (E * esize);
        if (n > G) n = G;
        while (n > 1 && n * ev > kThreads) --n;
        return n;
    };
    int parts = 1;
    for (int bytes = 128; bytes >= 32; bytes /= 2) {
        p.tile_groups = tile(bytes);
        p.tiles = (G + p.tile_groups - 1) / p.tile_groups;
        // a cluster of the fewest blocks that hold the slab; more while there are SMs left and rows to share out
        const auto need = [&](int n) { return slab_bytes((S + n - 1) / n, p.tile_groups * ev, V * esize, V == 1 ? kGroup<1> : kGroup<2>, bwd); };
        parts = 1;
        while (parts < kMaxCluster && need(parts) > kSlabBytes) parts *= 2;
        p.slab = need(parts) <= kSlabBytes;
        if (p.slab) break;
    }
    while (p.slab && parts < kMaxCluster && (long long)N * p.tiles * parts < kSms && S / parts >= 64) parts *= 2;
    // Large tensors are faster as a stream (32 x 3136 x 256 in bf16, forward and backward: 92 us, as slabs 138), whose second reading L2
    // serves in part; slabs save a launch and the reading below that (4 x 1024 x 256: 8 us forward, 10 as a stream).
    const int choice = env_int("CONV2D_B200_NORM_STREAM", 0);
    if (choice == 0 ? (size_t)N * S * C * esize > (bwd ? 16u : 24u) << 20 : choice > 0) p.slab = false;
    if (!p.slab) {
        p.tile_groups = tile(128), p.tiles = (G + p.tile_groups - 1) / p.tile_groups;
        // two blocks an SM (one of the backward pass): more are more beginnings and endings
        const long long slabs = (long long)N * p.tiles, want = ((bwd ? 1LL : 2LL) * kSms + slabs - 1) / slabs;
        parts = (int)(want > 1024 ? 1024 : want);
        if (parts > (S + 15) / 16) parts = (S + 15) / 16;
    }
    p.part_rows = (S + parts - 1) / parts;
    p.parts = p.slab ? parts : (S + p.part_rows - 1) / p.part_rows;
    p.stats = p.slab ? 0 : (size_t)N * G * p.parts * 4;
    p.channels = bwd ? (size_t)N * p.parts * 2 * C : 0;
    return p;
}

// Every element type and pack width that the sizes allow.
size_t workspace_floats(int N, int S, int C, int G, bool bwd)
{
    size_t most = 0;
    for (int esize = 2; esize <= 4; esize += 2)
        for (int V = 1; V <= 16 / esize; V *= 2) {
            if ((C / G) % V) continue;
            const NormPlan p = make_norm_plan(N, S, C, G, esize, V, bwd);
            if (p.stats + p.channels > most) most = p.stats + p.channels;
        }
    return most;
}

// Column (which, c) of the partial sums [parts][2][C].
struct ParamStore {
    float *dgamma, *dbeta;
    int C;
    __device__ void operator()(long long col, float s) const
    {
        if (col < C) {
            if (dbeta) dbeta[col] = s;
        } else if (dgamma) {
            dgamma[col - C] = s;
        }
    }
};

template <typename T, int V>
NormArgs<T> make_args(const NormSeq& s, const NormPlan& p)
{
    NormArgs<T> a{};
    a.x = static_cast<const T*>(s.x), a.dy = static_cast<const T*>(s.dy), a.gamma = s.gamma, a.beta = s.beta;
    a.y = static_cast<T*>(s.y), a.dx = static_cast<T*>(s.dx), a.mean = s.mean, a.rstd = s.rstd;
    a.part_stats = reinterpret_cast<float4*>(s.ws);
    a.channels = s.dgamma || s.dbeta ? s.ws + p.stats : nullptr;
    a.N = s.N, a.S = s.S, a.C = s.C, a.G = s.G, a.E = s.C / s.G;
    a.ldx = s.ldx, a.ldy = s.ldy, a.lddy = s.lddy, a.lddx = s.lddx, a.eps = s.eps, a.act = s.act;
    a.lanes = p.lanes, a.chunks = p.chunks, a.chunk = p.chunk;
    a.tile_groups = p.tile_groups, a.tiles = p.tiles, a.parts = p.parts, a.part_rows = p.part_rows, a.ev = a.E / V;
    return a;
}

template <typename... KArgs, typename... Args>
conv2d_status_t launched(void (*kernel)(KArgs...), long long blocks, int threads, size_t smem, unsigned cluster, cudaStream_t stream, Args... args)
{
    if (blocks > 0x7fffffffLL) return CONV2D_ERR_SHAPE;
    const cudaError_t e = cluster > 1 ? launch_pdl_cluster(kernel, dim3((unsigned)blocks), dim3(threads), smem, stream, cluster, args...)
                                      : launch_pdl(kernel, dim3((unsigned)blocks), dim3(threads), smem, stream, args...);
    if (e != cudaSuccess) return CONV2D_ERR_CUDA;
    count_launch();
    return CONV2D_OK;
}

template <typename T, int V, int NV, int ROWS>
conv2d_status_t rows_fwd(const NormArgs<T>& a, cudaStream_t stream)
{
    constexpr size_t smem = SampleRing<T, V, NV, ROWS>::smem;
    static SmemLimit limit;
    if (raise_smem_limit(reinterpret_cast<const void*>(norm_rows_fwd_kernel<T, V, NV, ROWS>), smem, limit) != cudaSuccess) return CONV2D_ERR_CUDA;
    return launched(norm_rows_fwd_kernel<T, V, NV, ROWS>, (long long)ceil_div_u((long long)a.G * a.lanes, kRowThreads) * a.chunks, kRowThreads, smem, 1, stream, a);
}
template <typename T, int V, int NV, int ROWS>
conv2d_status_t rows_bwd(const NormArgs<T>& a, cudaStream_t stream)
{
    constexpr size_t smem = 2 * SampleRing<T, V, NV, ROWS>::smem;
    static SmemLimit limit;
    if (raise_smem_limit(reinterpret_cast<const void*>(norm_rows_bwd_kernel<T, V, NV, ROWS>), smem, limit) != cudaSuccess) return CONV2D_ERR_CUDA;
    return launched(norm_rows_bwd_kernel<T, V, NV, ROWS>, (long long)ceil_div_u((long long)a.G * a.lanes, kRowThreads) * a.chunks, kRowThreads, smem, 1, stream, a);
}

template <typename T, int V>
conv2d_status_t fwd(const NormSeq& s, cudaStream_t stream)
{
    const NormPlan p = make_norm_plan(s.N, s.S, s.C, s.G, sizeof(T), V, false);
    const NormArgs<T> a = make_args<T, V>(s, p);
    if (p.rows) {
        if (p.nv == 1) return rows_fwd<T, V, 1, 2>(a, stream);
        if (p.nv == 2) return rows_fwd<T, V, 2, 1>(a, stream);
        return rows_fwd<T, V, 4, 1>(a, stream);
    }
    const long long blocks = (long long)s.N * p.tiles * p.parts;
    const size_t fixed = (size_t)p.tile_groups * 16 + (p.tile_groups + 1) / 2 * 16;
    if (p.slab) {
        const size_t smem = fixed + slab_bytes(p.part_rows, p.tile_groups * (a.E / V), V * sizeof(T), kGroup<V>, false);
        static SmemLimit limit;
        if (raise_smem_limit(reinterpret_cast<const void*>(norm_slab_fwd_kernel<T, V, kSlab>), smem, limit) != cudaSuccess) return CONV2D_ERR_CUDA;
        return launched(norm_slab_fwd_kernel<T, V, kSlab>, blocks, kThreads, smem, p.parts, stream, a);
    }
    const size_t smem = fixed + ring_bytes<T, V>;
    static SmemLimit stats, apply;
    if (raise_smem_limit(reinterpret_cast<const void*>(norm_slab_fwd_kernel<T, V, kStreamStats>), smem, stats) != cudaSuccess
        || raise_smem_limit(reinterpret_cast<const void*>(norm_slab_fwd_kernel<T, V, kStreamApply>), smem, apply) != cudaSuccess) return CONV2D_ERR_CUDA;
    const conv2d_status_t st = launched(norm_slab_fwd_kernel<T, V, kStreamStats>, blocks, kThreads, smem, 1, stream, a);
    return st != CONV2D_OK ? st : launched(norm_slab_fwd_kernel<T, V, kStreamApply>, blocks, kThreads, smem, 1, stream, a);
}

template <typename T, int V>
conv2d_status_t bwd(const NormSeq& s, cudaStream_t stream)
{
    const NormPlan p = make_norm_plan(s.N, s.S, s.C, s.G, sizeof(T), V, true);
    const NormArgs<T> a = make_args<T, V>(s, p);
    conv2d_status_t st;
    long long parts = (long long)s.N * p.parts;
    if (p.rows) {
        parts = p.chunks;
        if (p.nv == 1) st = rows_bwd<T, V, 1, 2>(a, stream);
        else if (p.nv == 2) st = rows_bwd<T, V, 2, 1>(a, stream);
        else st = rows_bwd<T, V, 4, 1>(a, stream);
    } else {
        const long long blocks = (long long)s.N * p.tiles * p.parts;
        const size_t fixed = (size_t)p.tile_groups * 16 + (p.tile_groups + 1) / 2 * 16, sums = sizeof(float) * 2 * kThreads * V;
        if (p.slab) {
            const size_t smem = fixed + sums + slab_bytes(p.part_rows, p.tile_groups * (a.E / V), V * sizeof(T), kGroup<V>, true);
            static SmemLimit limit;
            if (raise_smem_limit(reinterpret_cast<const void*>(norm_slab_bwd_kernel<T, V, kSlab>), smem, limit) != cudaSuccess) return CONV2D_ERR_CUDA;
            st = launched(norm_slab_bwd_kernel<T, V, kSlab>, blocks, kThreads, smem, p.parts, stream, a);
        } else {
            const size_t first = fixed + sums + 2 * ring_bytes<T, V>, second = fixed + 2 * ring_bytes<T, V>;
            static SmemLimit stats, apply;
            if (raise_smem_limit(reinterpret_cast<const void*>(norm_slab_bwd_kernel<T, V, kStreamStats>), first, stats) != cudaSuccess
                || raise_smem_limit(reinterpret_cast<const void*>(norm_slab_bwd_kernel<T, V, kStreamApply>), second, apply) != cudaSuccess) return CONV2D_ERR_CUDA;
            st = launched(norm_slab_bwd_kernel<T, V, kStreamStats>, blocks, kThreads, first, 1, stream, a);
            if (st == CONV2D_OK) st = launched(norm_slab_bwd_kernel<T, V, kStreamApply>, blocks, kThreads, second, 1, stream, a);
        }
    }
    if (st != CONV2D_OK || !a.channels) return st;
    return launch_column_sums(a.channels, parts, 2LL * s.C, 2LL * s.C, ParamStore{s.dgamma, s.dbeta, s.C}, stream);
}

// The widest packs, up to 16 bytes, in which no pack crosses from one group to the next and every row of every tensor begins on a boundary of them.
template <typename T>
bool packs_of(const NormSeq& s, int V)
{
    constexpr int e = sizeof(T);
    return (s.C / s.G) % V == 0 && rows_aligned(s.x, s.ldx, e, V * e) && rows_aligned(s.y, s.ldy, e, V * e) && rows_aligned(s.dy, s.lddy, e, V * e)
        && rows_aligned(s.dx, s.lddx, e, V * e);
}

template <typename T>
conv2d_status_t fwd_typed(const NormSeq& s, cudaStream_t stream)
{
    if constexpr (sizeof(T) == 2)
        if (packs_of<T>(s, 8)) return fwd<T, 8>(s, stream);
    if (packs_of<T>(s, 4)) return fwd<T, 4>(s, stream);
    return packs_of<T>(s, 2) ? fwd<T, 2>(s, stream) : fwd<T, 1>(s, stream);
}
template <typename T>
conv2d_status_t bwd_typed(const NormSeq& s, cudaStream_t stream)
{
    if constexpr (sizeof(T) == 2)
        if (packs_of<T>(s, 8)) return bwd<T, 8>(s, stream);
    if (packs_of<T>(s, 4)) return bwd<T, 4>(s, stream);
    return packs_of<T>(s, 2) ? bwd<T, 2>(s, stream) : bwd<T, 1>(s, stream);
}

}  // namespace

size_t norm_fwd_workspace_bytes(int N, int S, int C, int G) { return sizeof(float) * workspace_floats(N, S, C, G, false); }
size_t norm_bwd_workspace_bytes(int N, int S, int C, int G) { return sizeof(float) * workspace_floats(N, S, C, G, true); }

conv2d_status_t launch_norm_fwd(const NormSeq& s, conv2d_operand_t type, cudaStream_t stream)
{
    if (type == CONV2D_OPERAND_BF16) return fwd_typed<bf16>(s, stream);
    if (type == CONV2D_OPERAND_FP16) return fwd_typed<fp16>(s, stream);
    return fwd_typed<float>(s, stream);
}
conv2d_status_t launch_norm_bwd(const NormSeq& s, conv2d_operand_t type, cudaStream_t stream)
{
    if (type == CONV2D_OPERAND_BF16) return bwd_typed<bf16>(s, stream);
    if (type == CONV2D_OPERAND_FP16) return bwd_typed<fp16>(s, stream);
    return bwd_typed<float>(s, stream);
}

}  // namespace conv2d_b200
