// Selective state space scan, backward.
//
//   g = dy silu(z),   e_t = C_t g_t + a_{t+1} e_{t+1}  with  a_t = exp(s_t A),   q_t = e_t a_t h_{t-1}
//   dC_t = sum_d g h_t,  dB_t = sum_d e s u,  dA = sum_t s q,  ds = sum_n A q + u sum_n e B,  du = s sum_n e B + Dskip g,
//   dz = dy v silu'(z),  dDskip = sum_t g u
//
// The forward pass keeps the state before every 16th row.  A block walks the tiles of 16 rows from the last to the first; in a tile the
// decays a and the states h of all 16 rows are computed again, from the kept one, into registers (a thread has four states of one
// channel: 128 registers), so that the walk back needs no exponential.  Sums over the states go over the lanes of a channel, sums
// over the channels (dB, dC) over the other lanes, the warps and the channel sets that the block takes in turn, and from there as one
// partial sum of the block into the workspace; those are added by a kernel of their own in a fixed order.
#pragma once

#include "scan_common.cuh"

namespace conv2d_b200 {

constexpr int kSpt = 4;                 // states of a thread

inline int bwd_lanes_for(int N)
{
    int nl = 1;
    while (nl * kSpt < N) nl *= 2;
    return nl;
}

template <typename T>
struct ScanBwdArgs {
    const T *u, *delta, *Bm, *Cm, *z, *dy;
    const float *A, *Dskip, *delta_bias, *states, *dstate_out;
    const int* lengths;
    T *du, *ddelta, *dz;
    float *local, *steps;               // [B][segs][D][NQ], [B][segs][D]: what segments begin with from the right (end with, in the first walk)
    float *per_channel;                 // [B][segs] times channel_floats: partial sums of dA, dDskip, ddelta_bias
    float *per_row;                     // [G][blocks_group][B * L][2][NP]: partial sums of dB, dC
    float *dstate_in;
    int B, L, D, N, G, E;
    int segs, seg_rows, blocks_group, sets;
    long long ldu, lddelta, ldB, ldC, ldz, lddy, lddu, ldddelta, lddz;
    bool softplus;
};

template <int NL>
struct ScanBwdTile {
    static constexpr int W = 4, TH = W * 32, CL = 32 / NL, CB = W * CL, NP = NL * kSpt, TT = kCheckpointRows, YS = CB + CL;
    // (s, s u, g) of the tile, B and C, three sums over states, the warps' sums over channels and the block's
    static constexpr size_t fixed_floats = 4 * TT * CB + 2 * TT * NP + 3 * TT * YS + W * TT * 2 * NP + TT * 2 * NP;
    // a set's carried gradient, dA and A of every thread, and its sums for dDskip and ddelta_bias
    template <int V> static constexpr size_t set_floats() { return TH * (3 * kSpt + 2 * V); }
};

// Loads of a tile: pack `pk` of the rows tid / PPR + i * (TH / PPR), and elements tid + i * TH of B and C.
template <typename T, int NL, int V>
__global__ void __launch_bounds__(128) scan_bwd_kernel(const ScanBwdArgs<T> a)
{
    using Tile = ScanBwdTile<NL>;
    constexpr int W = Tile::W, TH = Tile::TH, CL = Tile::CL, CB = Tile::CB, NP = Tile::NP, TT = Tile::TT, YS = Tile::YS;
    constexpr int PPR = CB / V, PK = (TT * PPR + TH - 1) / TH, BK = (TT * NP + TH - 1) / TH, RS = TH / PPR;
    ptx::grid_dep_wait();
    extern __shared__ float4 smem4[];
    float4* q4 = smem4;                                       // [TT][CB] (s, s u, g, -)
    float* Bs = reinterpret_cast<float*>(q4 + TT * CB);       // [TT][NP]
    float* Cs = Bs + TT * NP;
    float* vs = Cs + TT * NP;                                 // [TT][YS] sum_n C h, sum_n A2 q, sum_n e B
    float* s1 = vs + TT * YS;
    float* s2 = s1 + TT * YS;
    float* parts = s2 + TT * YS;                              // [W][TT][2][NP]
    float* acc = parts + W * TT * 2 * NP;                     // [TT][2][NP]
    float4* carry4 = reinterpret_cast<float4*>(acc + TT * 2 * NP);   // [sets][TH]
    float4* dA4 = carry4 + a.sets * TH;
    float4* A24 = dA4 + a.sets * TH;
    float* chan = reinterpret_cast<float*>(A24 + a.sets * TH);       // [sets][2][V][TH]

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    unsigned bx = blockIdx.x;
    const int cb = (int)(bx % a.blocks_group);
    bx /= a.blocks_group;
    const int g = (int)(bx % a.G);
    bx /= a.G;
    const int seg = (int)(bx % a.segs);
    const long long b = bx / a.segs;
    const int len = sequence_length(a.lengths, (int)b, a.L);
    const int t_begin = seg * a.seg_rows, t_end = min(t_begin + a.seg_rows, a.L), live = min(t_end, len);
    const long long row0 = b * a.L;
    const int ch = warp * CL + lane / NL, n0 = (lane % NL) * kSpt, NQ = round4(a.N);
    const int cks = (a.L + TT - 1) / TT;
    const int sets = min(a.sets, (a.E - cb * CB * a.sets + CB - 1) / CB);    // of this block, at least one
    const int pk = (tid % PPR) * V, prow = tid / PPR;

    for (int set = 0; set < sets; ++set) {
        const int c0 = (cb * a.sets + set) * CB, d = g * a.E + c0 + ch;
        const bool mine = c0 + ch < a.E;
        float av[kSpt], cv[kSpt];
#pragma unroll
        for (int i = 0; i < kSpt; ++i) {
            const bool real = mine && n0 + i < a.N;
            av[i] = real ? a.A[(size_t)d * a.N + n0 + i] * kLog2e : 0.f;
            cv[i] = 0.f;
            if (real && a.segs > 1) cv[i] = a.local[(((size_t)b * a.segs + seg) * a.D + d) * NQ + n0 + i];
            else if (real && a.dstate_out) cv[i] = a.dstate_out[((size_t)b * a.D + d) * a.N + n0 + i];
        }
        A24[set * TH + tid] = make_float4(av[0], av[1], av[2], av[3]);
        carry4[set * TH + tid] = make_float4(cv[0], cv[1], cv[2], cv[3]);
        dA4[set * TH + tid] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int i = 0; i < 2 * V; ++i) chan[(set * 2 * V + i) * TH + tid] = 0.f;
    }
    for (int i = tid; i < TT * 2 * NP; i += TH) acc[i] = 0.f;

    Pack<T, V> pu[PK], pd[PK], pz[PK], pg[PK];
    T pb[BK], pc[BK];
    auto fetch = [&](int t0, int set) {
        const int c = (cb * a.sets + set) * CB + pk, d = g * a.E + c;
#pragma unroll
        for (int i = 0; i < PK; ++i) {
            const int r = prow + i * RS, t = t0 + r;
            const bool real = c < a.E && r < TT && t < live;
            const long long row = row0 + t;
            pu[i] = real ? load_pack<T, V>(a.u + row * a.ldu + d) : zero_pack<T, V>();
            pd[i] = real ? load_pack<T, V>(a.delta + row * a.lddelta + d) : zero_pack<T, V>();
            pg[i] = real ? load_pack<T, V>(a.dy + row * a.lddy + d) : zero_pack<T, V>();
            pz[i] = real && a.z ? load_pack<T, V>(a.z + row * a.ldz + d) : zero_pack<T, V>();
        }
        if (set == 0) {
#pragma unroll
            for (int i = 0; i < BK; ++i) {
                const int e = tid + i * TH, t = t0 + e / NP, n = e % NP;
                const bool real = e < TT * NP && n < a.N && t < live;
                pb[i] = real ? a.Bm[(row0 + t) * a.ldB + g * a.N + n] : from_float<T>(0.f);
                pc[i] = real ? a.Cm[(row0 + t) * a.ldC + g * a.N + n] : from_float<T>(0.f);
            }
        }
    };

    const int tiles = live > t_begin ? (live - t_begin + TT - 1) / TT : 0;
    if (tiles) fetch(t_begin + (tiles - 1) * TT, 0);
    for (int tile = tiles - 1; tile >= 0; --tile) {
        const int t0 = t_begin + tile * TT;
        for (int set = 0; set < sets; ++set) {
            const int c0 = (cb * a.sets + set) * CB;
            const bool pk_real = c0 + pk < a.E;
            Pack<T, V> cu[PK], cd[PK], cz[PK], cg[PK];
#pragma unroll
            for (int i = 0; i < PK; ++i) {
                const int r = prow + i * RS;
                cu[i] = pu[i], cd[i] = pd[i], cz[i] = pz[i], cg[i] = pg[i];
                if (TT * PPR % TH != 0 && r >= TT) continue;
                float u[V], s[V], z[V], dy[V];
                unpack(pu[i], u);
                unpack(pd[i], s);
                unpack(pz[i], z);
                unpack(pg[i], dy);
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    if (a.delta_bias && pk_real) s[j] += a.delta_bias[g * a.E + c0 + pk + j];
                    if (a.softplus) s[j] = softplus(s[j]);
                    if (t0 + r >= live || !pk_real) s[j] = 0.f;
                    const float gate = a.z ? dy[j] * z[j] * sigmoid(z[j]) : dy[j];
                    q4[r * CB + pk + j] = make_float4(s[j], s[j] * u[j], gate, 0.f);
                }
            }
            if (set == 0) {
#pragma unroll
                for (int i = 0; i < BK; ++i) {
                    const int e = tid + i * TH;
                    if (TT * NP % TH != 0 && e >= TT * NP) continue;
                    Bs[e] = to_float(pb[i]);
                    Cs[e] = to_float(pc[i]);
                }
            }
            __syncthreads();
            if (set + 1 < sets) fetch(t0, set + 1);
            else if (tile > 0) fetch(t0 - TT, 0);

            const int d = g * a.E + c0 + ch;
            const bool mine = c0 + ch < a.E;
            const float4 A4 = A24[set * TH + tid];
            const float2 A2[2] = {make_float2(A4.x, A4.y), make_float2(A4.z, A4.w)};
            float4 h4 = make_float4(0.f, 0.f, 0.f, 0.f);
            if (mine && n0 < NQ) h4 = *reinterpret_cast<const float4*>(a.states + (((size_t)b * cks + t0 / TT) * a.D + d) * NQ + n0);
            const float2 h0[2] = {make_float2(h4.x, h4.y), make_float2(h4.z, h4.w)};
            float2 ea[TT][2], h[TT][2];
#pragma unroll
            for (int tq = 0; tq < TT; tq += 4) {
                float v[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int t = tq + j;
                    const float4 q = q4[t * CB + ch];
                    const float4 bv = *reinterpret_cast<const float4*>(Bs + t * NP + n0), cv = *reinterpret_cast<const float4*>(Cs + t * NP + n0);
                    const float2 s_2 = make_float2(q.x, q.x), su2 = make_float2(q.y, q.y);
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        float2 e = __fmul2_rn(s_2, A2[i]);
                        e.x = ex2(e.x), e.y = ex2(e.y);
                        ea[t][i] = e;
                        h[t][i] = __ffma2_rn(e, t ? h[t - 1][i] : h0[i], __fmul2_rn(su2, i ? make_float2(bv.z, bv.w) : make_float2(bv.x, bv.y)));
                    }
                    const float2 o = __ffma2_rn(h[t][1], make_float2(cv.z, cv.w), __fmul2_rn(h[t][0], make_float2(cv.x, cv.y)));
                    v[j] = o.x + o.y;
                }
                constexpr int left = NL >= 4 ? 1 : 4 / NL;
                const int first = sum_over_lanes<4, NL, 1>(v, lane);
                if (first_of_equals<4, NL, 1>(lane)) {
#pragma unroll
                    for (int j = 0; j < left; ++j) vs[(tq + first + j) * YS + ch] = v[j];
                }
            }
            const float4 c4 = carry4[set * TH + tid], w4 = dA4[set * TH + tid];
            float2 carry[2] = {make_float2(c4.x, c4.y), make_float2(c4.z, c4.w)}, dA[2] = {make_float2(w4.x, w4.y), make_float2(w4.z, w4.w)};
#pragma unroll
            for (int tq = TT - 4; tq >= 0; tq -= 4) {
                float n_sums[8];                              // sum_n A2 q of four rows, then sum_n e B
#pragma unroll
                for (int j = 3; j >= 0; --j) {
                    const int t = tq + j;
                    const float4 q = q4[t * CB + ch];
                    const float4 bv = *reinterpret_cast<const float4*>(Bs + t * NP + n0), cv = *reinterpret_cast<const float4*>(Cs + t * NP + n0);
                    const float2 s_2 = make_float2(q.x, q.x), su2 = make_float2(q.y, q.y), g2 = make_float2(q.z, q.z);
                    float2 Aq = make_float2(0.f, 0.f), eB = make_float2(0.f, 0.f);
                    float d_sums[8];                          // e s u, then g h, of the four states
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const float2 e = __ffma2_rn(i ? make_float2(cv.z, cv.w) : make_float2(cv.x, cv.y), g2, carry[i]);
                        const float2 qq = __fmul2_rn(e, __fmul2_rn(ea[t][i], t ? h[t - 1][i] : h0[i]));
                        dA[i] = __ffma2_rn(s_2, qq, dA[i]);
                        Aq = __ffma2_rn(A2[i], qq, Aq);
                        eB = __ffma2_rn(e, i ? make_float2(bv.z, bv.w) : make_float2(bv.x, bv.y), eB);
                        const float2 db = __fmul2_rn(e, su2), dc = __fmul2_rn(g2, h[t][i]);
                        d_sums[2 * i] = db.x, d_sums[2 * i + 1] = db.y, d_sums[4 + 2 * i] = dc.x, d_sums[5 + 2 * i] = dc.y;
                        carry[i] = __fmul2_rn(ea[t][i], e);
                    }
                    n_sums[j] = Aq.x + Aq.y;
                    n_sums[4 + j] = eB.x + eB.y;
                    constexpr int left = CL >= 8 ? 1 : 8 / CL;
                    const int first = sum_over_lanes<8, CL, NL>(d_sums, lane);
                    if (first_of_equals<8, CL, NL>(lane)) {
#pragma unroll
                        for (int k = 0; k < left; ++k) {
                            const int id = first + k;
                            parts[((warp * TT + t) * 2 + (id >> 2)) * NP + n0 + (id & 3)] = d_sums[k];
                        }
                    }
                }
                constexpr int left = NL >= 8 ? 1 : 8 / NL;
                const int first = sum_over_lanes<8, NL, 1>(n_sums, lane);
                if (first_of_equals<8, NL, 1>(lane)) {
#pragma unroll
                    for (int k = 0; k < left; ++k) {
                        const int id = first + k;
                        (id >> 2 ? s2 : s1)[(tq + (id & 3)) * YS + ch] = n_sums[k];
                    }
                }
            }
            carry4[set * TH + tid] = make_float4(carry[0].x, carry[0].y, carry[1].x, carry[1].y);
            dA4[set * TH + tid] = make_float4(dA[0].x, dA[0].y, dA[1].x, dA[1].y);
            __syncthreads();

            float sum_d[V] = {}, sum_b[V] = {};
#pragma unroll
            for (int i = 0; i < PK; ++i) {
                const int r = prow + i * RS;
                if (!pk_real || r >= TT || t0 + r >= live) continue;
                float u[V], raw[V], z[V], dy[V], du[V], dd[V], dz[V];
                unpack(cu[i], u);
                unpack(cd[i], raw);
                unpack(cz[i], z);
                unpack(cg[i], dy);
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const int c = g * a.E + c0 + pk + j, at = r * YS + pk + j;
                    const float4 q = q4[r * CB + pk + j];
                    const float skip = a.Dskip ? a.Dskip[c] : 0.f;
                    du[j] = fmaf(q.x, s2[at], skip * q.z);
                    dd[j] = fmaf(kLn2, s1[at], u[j] * s2[at]);
                    if (a.softplus) dd[j] *= sigmoid(a.delta_bias ? raw[j] + a.delta_bias[c] : raw[j]);
                    if (a.z) {
                        const float sg = sigmoid(z[j]);
                        dz[j] = dy[j] * fmaf(skip, u[j], vs[at]) * sg * fmaf(z[j], 1.f - sg, 1.f);
                    }
                    sum_d[j] = fmaf(q.z, u[j], sum_d[j]);
                    sum_b[j] += dd[j];
                }
                const long long row = row0 + t0 + r;
                store_pack(a.du + row * a.lddu + g * a.E + c0 + pk, pack<T, V>(du));
                store_pack(a.ddelta + row * a.ldddelta + g * a.E + c0 + pk, pack<T, V>(dd));
                if (a.z) store_pack(a.dz + row * a.lddz + g * a.E + c0 + pk, pack<T, V>(dz));
            }
#pragma unroll
            for (int j = 0; j < V; ++j) {
                chan[((set * 2) * V + j) * TH + tid] += sum_d[j];
                chan[((set * 2 + 1) * V + j) * TH + tid] += sum_b[j];
            }
            const bool out = set == sets - 1;
            for (int i = tid; i < TT * 2 * NP; i += TH) {
                float s = acc[i];
#pragma unroll
                for (int w = 0; w < W; ++w) s += parts[w * TT * 2 * NP + i];
                acc[i] = out ? 0.f : s;
                const int t = t0 + i / (2 * NP);
                if (out && t < live)
                    a.per_row[((((size_t)g * a.blocks_group + cb) * a.B * a.L) + row0 + t) * (2 * NP) + i % (2 * NP)] = s;
            }
        }
    }

    // rows of padding, and what a block has summed over its rows
    for (int set = 0; set < sets; ++set) {
        const int c0 = (cb * a.sets + set) * CB, d = g * a.E + c0 + ch;
        if (c0 + pk < a.E) {
            for (int t = max(t_begin, live) + prow; t < t_end; t += RS) {
                const long long row = row0 + t;
                store_pack(a.du + row * a.lddu + g * a.E + c0 + pk, zero_pack<T, V>());
                store_pack(a.ddelta + row * a.ldddelta + g * a.E + c0 + pk, zero_pack<T, V>());
                if (a.z) store_pack(a.dz + row * a.lddz + g * a.E + c0 + pk, zero_pack<T, V>());
            }
        }
        float* out = a.per_channel + ((size_t)b * a.segs + seg) * channel_floats(a.D, NQ);
        if (c0 + ch < a.E && n0 < NQ) *reinterpret_cast<float4*>(out + (size_t)d * NQ + n0) = dA4[set * TH + tid];
        if (a.dstate_in && a.segs == 1 && c0 + ch < a.E) {
            const float4 c4 = carry4[set * TH + tid];
            const float cv[kSpt] = {c4.x, c4.y, c4.z, c4.w};
#pragma unroll
            for (int i = 0; i < kSpt; ++i)
                if (n0 + i < a.N) a.dstate_in[((size_t)b * a.D + d) * a.N + n0 + i] = cv[i];
        }
    }
    __syncthreads();
    for (int i = tid; i < sets * 2 * CB; i += TH) {
        const int c = i % CB, which = i / CB % 2, set = i / (2 * CB), cc = (cb * a.sets + set) * CB + c;
        if (cc >= a.E) continue;
        float s = 0.f;
        for (int r = 0; r < RS; ++r) s += chan[((set * 2 + which) * V + c % V) * TH + r * PPR + c / V];
        float* out = a.per_channel + ((size_t)b * a.segs + seg) * channel_floats(a.D, NQ) + (size_t)a.D * NQ;
        out[(size_t)which * a.D + g * a.E + cc] = s;
    }
}

// What a segment hands to the one before it when it is walked from zero: carry <- a_t (C_t g_t + carry), and the sum of its steps.
template <typename T, int NL, int V>
__global__ void __launch_bounds__(128) scan_bwd_carry_kernel(const ScanBwdArgs<T> a, int blocks_group)
{
    using Tile = ScanBwdTile<NL>;
    constexpr int TH = Tile::TH, CL = Tile::CL, CB = Tile::CB, NP = Tile::NP, TT = Tile::TT;
    constexpr int PPR = CB / V, PK = (TT * PPR + TH - 1) / TH, BK = (TT * NP + TH - 1) / TH, RS = TH / PPR;
    ptx::grid_dep_wait();
    __shared__ __align__(16) float2 sg[TT * CB];
    __shared__ __align__(16) float Cs[TT * NP];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    unsigned bx = blockIdx.x;
    const int c0 = (int)(bx % blocks_group) * CB;
    bx /= blocks_group;
    const int g = (int)(bx % a.G);
    bx /= a.G;
    const int seg = (int)(bx % a.segs);
    const long long b = bx / a.segs;
    const int len = sequence_length(a.lengths, (int)b, a.L);
    const int t_begin = seg * a.seg_rows, live = min(min(t_begin + a.seg_rows, a.L), len);
    const long long row0 = b * a.L;
    const int ch = warp * CL + lane / NL, n0 = (lane % NL) * kSpt, NQ = round4(a.N), d = g * a.E + c0 + ch;
    const bool mine = c0 + ch < a.E;
    const int pk = (tid % PPR) * V, prow = tid / PPR;
    const bool pk_real = c0 + pk < a.E;
    float2 A2[2], carry[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
    float av[kSpt], bias[V], steps = 0.f;
#pragma unroll
    for (int i = 0; i < kSpt; ++i) av[i] = mine && n0 + i < a.N ? a.A[(size_t)d * a.N + n0 + i] * kLog2e : 0.f;
    A2[0] = make_float2(av[0], av[1]), A2[1] = make_float2(av[2], av[3]);
#pragma unroll
    for (int i = 0; i < V; ++i) bias[i] = a.delta_bias && pk_real ? a.delta_bias[g * a.E + c0 + pk + i] : 0.f;

    Pack<T, V> pd[PK], pz[PK], pg[PK];
    T pc[BK];
    auto fetch = [&](int t0) {
#pragma unroll
        for (int i = 0; i < PK; ++i) {
            const int r = prow + i * RS, t = t0 + r;
            const bool real = pk_real && r < TT && t < live;
            const long long row = row0 + t;
            pd[i] = real ? load_pack<T, V>(a.delta + row * a.lddelta + g * a.E + c0 + pk) : zero_pack<T, V>();
            pg[i] = real ? load_pack<T, V>(a.dy + row * a.lddy + g * a.E + c0 + pk) : zero_pack<T, V>();
            pz[i] = real && a.z ? load_pack<T, V>(a.z + row * a.ldz + g * a.E + c0 + pk) : zero_pack<T, V>();
        }
#pragma unroll
        for (int i = 0; i < BK; ++i) {
            const int e = tid + i * TH, t = t0 + e / NP, n = e % NP;
            pc[i] = e < TT * NP && n < a.N && t < live ? a.Cm[(row0 + t) * a.ldC + g * a.N + n] : from_float<T>(0.f);
        }
    };
    const int tiles = live > t_begin ? (live - t_begin + TT - 1) / TT : 0;
    if (tiles) fetch(t_begin + (tiles - 1) * TT);
    for (int tile = tiles - 1; tile >= 0; --tile) {
        const int t0 = t_begin + tile * TT;
#pragma unroll
        for (int i = 0; i < PK; ++i) {
            const int r = prow + i * RS;
            if (TT * PPR % TH != 0 && r >= TT) continue;
            float s[V], z[V], dy[V];
            unpack(pd[i], s);
            unpack(pz[i], z);
            unpack(pg[i], dy);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                s[j] += bias[j];
                if (a.softplus) s[j] = softplus(s[j]);
                if (t0 + r >= live) s[j] = 0.f;
                sg[r * CB + pk + j] = make_float2(s[j], a.z ? dy[j] * z[j] * sigmoid(z[j]) : dy[j]);
            }
        }
#pragma unroll
        for (int i = 0; i < BK; ++i) {
            const int e = tid + i * TH;
            if (TT * NP % TH != 0 && e >= TT * NP) continue;
            Cs[e] = to_float(pc[i]);
        }
        __syncthreads();
        if (tile > 0) fetch(t0 - TT);
#pragma unroll 4
        for (int t = TT - 1; t >= 0; --t) {
            const float2 q = sg[t * CB + ch];
            const float4 cv = *reinterpret_cast<const float4*>(Cs + t * NP + n0);
            const float2 s_2 = make_float2(q.x, q.x), g2 = make_float2(q.y, q.y);
            float2 e0 = __fmul2_rn(s_2, A2[0]), e1 = __fmul2_rn(s_2, A2[1]);
            e0.x = ex2(e0.x), e0.y = ex2(e0.y), e1.x = ex2(e1.x), e1.y = ex2(e1.y);
            carry[0] = __fmul2_rn(e0, __ffma2_rn(make_float2(cv.x, cv.y), g2, carry[0]));
            carry[1] = __fmul2_rn(e1, __ffma2_rn(make_float2(cv.z, cv.w), g2, carry[1]));
            steps += q.x;
        }
        __syncthreads();
    }
    if (mine && n0 < NQ) {
        const size_t at = ((size_t)b * a.segs + seg) * a.D + d;
        *reinterpret_cast<float4*>(a.local + at * NQ + n0) = make_float4(carry[0].x, carry[0].y, carry[1].x, carry[1].y);
        if (n0 == 0) a.steps[at] = steps;
    }
}

}  // namespace conv2d_b200
