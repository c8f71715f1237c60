// Selective state space scan, forward.
//
//   h_t = exp(s_t A) h_{t-1} + s_t u_t B_t,   v_t = C_t . h_t + Dskip u_t,   y_t = v_t silu(z_t)
//
// Every (row, channel, state) takes an exponential of its own, so the special-function units (16 a clock and SM) set the pace, not memory.
// A block takes CB channels of one sequence and walks its rows in tiles of TT: the tile's u, delta, z, B and C come in by wide loads
// one tile ahead; s and s u are computed once per row and channel and put into shared memory beside B and C; then every warp
// walks the tile with its states in registers, and the sums over the states go back through shared memory so that y is stored
// in rows.  Sequences that would leave the machine idle are cut into segments, whose end states are computed first, from zero
// (STATE_ONLY), joined, and given to the walk proper.
#pragma once

#include "scan_common.cuh"

namespace conv2d_b200 {

template <typename T>
struct ScanFwdArgs {
    const T *u, *delta, *Bm, *Cm, *z;
    const float *A, *Dskip, *delta_bias, *state_in;
    const int* lengths;
    T* y;
    float *state_out, *states, *local, *steps;     // local: [B][segs][D][NQ] states that segments begin with (end with, STATE_ONLY)
    int B, L, D, N, G, E;                          // E = D / G channels of a group
    int segs, seg_rows, blocks_group;              // seg_rows: a multiple of the tile; blocks_group: blocks of a group's channels
    long long ldu, lddelta, ldB, ldC, ldz, ldy;
    bool softplus;
};

template <int NL>
struct ScanFwdTile {
    static constexpr int W = NL >= 8 ? 8 : 4, CL = 32 / NL, CB = W * CL, NP = NL * kSpt, TT = NL <= 2 ? 16 : 32, YS = CB + CL;
    static constexpr size_t smem = sizeof(float) * (2 * TT * CB + 2 * TT * NP + TT * YS);
};

template <typename T, int NL, int V, bool STATE_ONLY>
__global__ void __launch_bounds__(ScanFwdTile<NL>::W * 32) scan_fwd_kernel(const ScanFwdArgs<T> a)
{
    using Tile = ScanFwdTile<NL>;
    constexpr int CL = Tile::CL, CB = Tile::CB, NP = Tile::NP, TT = Tile::TT, YS = Tile::YS, TH = Tile::W * 32;
    constexpr int PPR = CB / V, PK = (TT * PPR + TH - 1) / TH, BK = (TT * NP + TH - 1) / TH;
    ptx::grid_dep_wait();
    extern __shared__ float4 smem4[];
    float2* dd = reinterpret_cast<float2*>(smem4);            // [TT][CB] (s, s u)
    float* Bs = reinterpret_cast<float*>(dd + TT * CB);       // [TT][NP]
    float* Cs = Bs + TT * NP;
    float* ys = Cs + TT * NP;                                 // [TT][YS]

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    unsigned bx = blockIdx.x;
    const int cb = (int)(bx % a.blocks_group);
    bx /= a.blocks_group;
    const int g = (int)(bx % a.G);
    bx /= a.G;
    const int seg = (int)(bx % a.segs);
    const long long b = bx / a.segs;
    const int len = sequence_length(a.lengths, (int)b, a.L);
    const int c0 = cb * CB;                                   // first channel, counted within the group
    const int nch = min(CB, a.E - c0);
    const int d0 = g * a.E + c0;
    const int t_begin = seg * a.seg_rows, t_end = min(t_begin + a.seg_rows, a.L), live = min(t_end, len);
    const long long row0 = b * a.L;

    // the states of this thread
    const int ch = warp * CL + lane / NL, n0 = (lane % NL) * kSpt;
    const bool mine = ch < nch;
    const int d = d0 + ch, NQ = round4(a.N);
    float2 A2[kSpt / 2], h[kSpt / 2];
    {
        float av[kSpt], hv[kSpt];
#pragma unroll
        for (int i = 0; i < kSpt; ++i) {
            const bool real = mine && n0 + i < a.N;
            av[i] = real ? a.A[(size_t)d * a.N + n0 + i] * kLog2e : 0.f;
            hv[i] = 0.f;
            if (!STATE_ONLY && real) {
                if (a.segs > 1) hv[i] = a.local[(((size_t)b * a.segs + seg) * a.D + d) * NQ + n0 + i];
                else if (a.state_in) hv[i] = a.state_in[((size_t)b * a.D + d) * a.N + n0 + i];
            }
        }
        A2[0] = make_float2(av[0], av[1]), A2[1] = make_float2(av[2], av[3]);
        h[0] = make_float2(hv[0], hv[1]), h[1] = make_float2(hv[2], hv[3]);
    }
    float steps = 0.f;

    // loads of a tile: pack `pk` of the rows tid / PPR + i * (TH / PPR), and elements tid + i * TH of B and C
    const int pk = (tid % PPR) * V, prow = tid / PPR;
    const bool pk_real = pk < nch;                            // (V divides E: a pack lies inside or outside)
    float bias[V], skip[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        bias[i] = a.delta_bias && pk_real ? a.delta_bias[d0 + pk + i] : 0.f;
        skip[i] = !STATE_ONLY && a.Dskip && pk_real ? a.Dskip[d0 + pk + i] : 0.f;
    }
    Pack<T, V> pu[PK], pd[PK], pz[PK];
    T pb[BK], pc[BK];
    auto fetch = [&](int t0) {
#pragma unroll
        for (int i = 0; i < PK; ++i) {
            const int r = prow + i * (TH / PPR), t = t0 + r;
            const bool real = pk_real && r < TT && t < live;
            const long long row = row0 + t;
            pu[i] = real ? load_pack<T, V>(a.u + row * a.ldu + d0 + pk) : zero_pack<T, V>();
            pd[i] = real ? load_pack<T, V>(a.delta + row * a.lddelta + d0 + pk) : zero_pack<T, V>();
            if (!STATE_ONLY) pz[i] = real && a.z ? load_pack<T, V>(a.z + row * a.ldz + d0 + pk) : zero_pack<T, V>();
        }
#pragma unroll
        for (int i = 0; i < BK; ++i) {
            const int e = tid + i * TH, t = t0 + e / NP, n = e % NP;
            const bool real = e < TT * NP && n < a.N && t < live;
            pb[i] = real ? a.Bm[(row0 + t) * a.ldB + g * a.N + n] : from_float<T>(0.f);
            if (!STATE_ONLY) pc[i] = real ? a.Cm[(row0 + t) * a.ldC + g * a.N + n] : from_float<T>(0.f);
        }
    };

    if (t_begin < live) fetch(t_begin);
    for (int t0 = t_begin; t0 < live; t0 += TT) {
        Pack<T, V> cu[PK], cz[PK];
#pragma unroll
        for (int i = 0; i < PK; ++i) {
            const int r = prow + i * (TH / PPR);
            cu[i] = pu[i];
            if (!STATE_ONLY) cz[i] = pz[i];
            if (TT * PPR % TH != 0 && r >= TT) continue;
            float u[V], s[V];
            unpack(pu[i], u);
            unpack(pd[i], s);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                s[j] += bias[j];
                if (a.softplus) s[j] = softplus(s[j]);
                if (t0 + r >= live) s[j] = 0.f;               // padding: the state stays
                dd[r * CB + pk + j] = make_float2(s[j], s[j] * u[j]);
            }
        }
#pragma unroll
        for (int i = 0; i < BK; ++i) {
            const int e = tid + i * TH;
            if (TT * NP % TH != 0 && e >= TT * NP) continue;
            Bs[e] = to_float(pb[i]);
            if (!STATE_ONLY) Cs[e] = to_float(pc[i]);
        }
        __syncthreads();
        if (t0 + TT < live) fetch(t0 + TT);
#pragma unroll 1
        for (int tt = 0; tt < TT; tt += 4) {
            if (!STATE_ONLY && a.states && tt % kCheckpointRows == 0 && t0 + tt < live && mine && n0 < NQ) {
                const int cks = (a.L + kCheckpointRows - 1) / kCheckpointRows, ck = (t0 + tt) / kCheckpointRows;
                *reinterpret_cast<float4*>(a.states + (((size_t)b * cks + ck) * a.D + d) * NQ + n0) = make_float4(h[0].x, h[0].y, h[1].x, h[1].y);
            }
            float out[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float2 s = dd[(tt + j) * CB + ch];
                const float4 bv = *reinterpret_cast<const float4*>(Bs + (tt + j) * NP + n0);
                const float2 s2 = make_float2(s.x, s.x), su2 = make_float2(s.y, s.y);
                float2 e0 = __fmul2_rn(s2, A2[0]), e1 = __fmul2_rn(s2, A2[1]);
                e0.x = ex2(e0.x), e0.y = ex2(e0.y), e1.x = ex2(e1.x), e1.y = ex2(e1.y);
                h[0] = __ffma2_rn(e0, h[0], __fmul2_rn(su2, make_float2(bv.x, bv.y)));
                h[1] = __ffma2_rn(e1, h[1], __fmul2_rn(su2, make_float2(bv.z, bv.w)));
                if (STATE_ONLY) {
                    steps += s.x;
                } else {
                    const float4 cv = *reinterpret_cast<const float4*>(Cs + (tt + j) * NP + n0);
                    const float2 o = __ffma2_rn(h[1], make_float2(cv.z, cv.w), __fmul2_rn(h[0], make_float2(cv.x, cv.y)));
                    out[j] = o.x + o.y;
                }
            }
            if (!STATE_ONLY) {
                constexpr int left = NL >= 4 ? 1 : 4 / NL;
                const int first = sum_over_lanes<4, NL, 1>(out, lane);
                if (first_of_equals<4, NL, 1>(lane)) {
#pragma unroll
                    for (int j = 0; j < left; ++j) ys[(tt + first + j) * YS + ch] = out[j];
                }
            }
        }
        __syncthreads();
        if (!STATE_ONLY) {
#pragma unroll
            for (int i = 0; i < PK; ++i) {
                const int r = prow + i * (TH / PPR);
                if (!pk_real || r >= TT || t0 + r >= live) continue;
                float u[V], z[V], o[V];
                unpack(cu[i], u);
                unpack(cz[i], z);
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    o[j] = fmaf(skip[j], u[j], ys[r * YS + pk + j]);
                    if (a.z) o[j] *= z[j] * sigmoid(z[j]);
                }
                store_pack(a.y + (row0 + t0 + r) * a.ldy + d0 + pk, pack<T, V>(o));
            }
        }
    }
    if (!STATE_ONLY) {
        if (pk_real)
            for (int t = max(t_begin, live) + prow; t < t_end; t += TH / PPR) store_pack(a.y + (row0 + t) * a.ldy + d0 + pk, zero_pack<T, V>());
        if (a.state_out && seg == a.segs - 1 && mine) {
            const float hv[kSpt] = {h[0].x, h[0].y, h[1].x, h[1].y};
#pragma unroll
            for (int i = 0; i < kSpt; ++i)
                if (n0 + i < a.N) a.state_out[((size_t)b * a.D + d) * a.N + n0 + i] = hv[i];
        }
    } else if (mine && n0 < NQ) {
        const size_t at = ((size_t)b * a.segs + seg) * a.D + d;
        *reinterpret_cast<float4*>(a.local + at * NQ + n0) = make_float4(h[0].x, h[0].y, h[1].x, h[1].y);
        if (n0 == 0) a.steps[at] = steps;
    }
}

}  // namespace conv2d_b200
