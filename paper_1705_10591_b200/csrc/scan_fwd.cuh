// Selective state space scan, forward.
//
//   h_t = exp(s_t A) h_{t-1} + s_t u_t B_t,   v_t = C_t . h_t + Dskip u_t,   y_t = v_t silu(z_t)
//
// Every (row, channel, state) takes an exponential of its own, so the special-function units (16 a clock and SM) set the pace, not memory.
// A block takes the channels of its W scanning warps and walks the rows of a sequence in tiles of TT; four more warps do what is done once
// per row and channel, so that the scanning warps, of which a batch of a few thousand channels gives one or two to a scheduler, only scan: while
// tile k is scanned, they bring tile k + 3 in (asynchronous copies), put s and s u of tile k + 1 into shared memory beside its B and C in fp32,
// and gate and store the sums over the states of tile k - 1.  A scanning warp takes eight rows at a time: the exponentials and inputs of all
// eight first, independent of each other, then the recurrence over them.
// A batch of few channels has less than one warp for each scheduler.  Then sequences are cut into segments, whose end states are computed
// first, from zero (STATE_ONLY), joined, and given to the walk proper; every exponential is taken twice then.
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
    int ldu, lddelta, ldB, ldC, ldz, ldy;
    int u_unit, delta_unit, z_unit, B_unit, C_unit;   // bytes in which rows can be copied
    bool y_quads, softplus;                           // y_quads: y can be stored four elements at a time
};

template <int NL, int SPT>
struct ScanFwdTile {
    static constexpr int CL = 32 / NL, NP = NL * SPT, R = 8, W = NL >= 8 ? 8 : 4, CB = W * CL, TT = CB >= 64 || NP >= 64 ? 16 : 32;
    static constexpr int SCAN = 32 * W, HELP = 128, TH = SCAN + HELP, RAWS = 4;
    static constexpr int YS = CB + 4;                 // (the lanes that store a row's sums hit different banks)
    static constexpr size_t raw(size_t esize) { return esize * TT * (3 * CB + 2 * NP); }              // one tile as it lies in memory
    static constexpr size_t smem(size_t esize) { return RAWS * raw(esize) + sizeof(float) * 2 * (2 * TT * CB + 2 * TT * NP + TT * YS); }
};

template <typename T, int NL, int SPT, bool STATE_ONLY>
__global__ void __launch_bounds__(ScanFwdTile<NL, SPT>::TH) scan_fwd_kernel(const ScanFwdArgs<T> a)
{
    using Tile = ScanFwdTile<NL, SPT>;
    constexpr int CL = Tile::CL, CB = Tile::CB, NP = Tile::NP, R = Tile::R, TT = Tile::TT, HT = Tile::HELP, YS = Tile::YS, P = SPT / 2, ES = sizeof(T);
    constexpr int OWN = NL >= R ? 1 : R / NL, SHARE = NL > R ? NL / R : 1;      // rows of a lane after a sum; lanes that have the same row
    constexpr int UNITS = TT * CB / 4, UK = (UNITS + HT - 1) / HT, BUNITS = TT * NP / 4, BK = (BUNITS + HT - 1) / HT, UROWS = HT / (CB / 4);
    constexpr int DD = TT * CB, BC = 2 * TT * NP, YB = TT * YS, RAW = TT * (3 * CB + 2 * NP), RAWS = Tile::RAWS;
    ptx::grid_dep_wait();
    extern __shared__ float4 smem4[];
    float2* dd = reinterpret_cast<float2*>(smem4);            // [2][TT][CB] (s, s u)
    float* bc = reinterpret_cast<float*>(dd + 2 * DD);        // [2] of B, C [TT][NP]
    float* ys = bc + 2 * BC;                                  // [2][TT][YS]
    T* raw = reinterpret_cast<T*>(ys + 2 * YB);               // [RAWS] of u, delta, z [TT][CB], B, C [TT][NP]

    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
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
    const int d0 = g * a.E + c0, NQ = round4(a.N);
    const int t_begin = seg * a.seg_rows, t_end = min(t_begin + a.seg_rows, a.L), live = min(t_end, len);
    const int tiles = live > t_begin ? (live - t_begin + TT - 1) / TT : 0;
    const long long row0 = b * a.L;

    if (warp < Tile::W) {                                     // ---- the scanning warps
        const int ch = warp * CL + lane % CL, sl = lane / CL, n0 = sl * SPT;
        const bool mine = ch < nch;
        const int d = d0 + ch;
        float2 A2[P], h[P];
        {
            float av[SPT], hv[SPT];
#pragma unroll
            for (int i = 0; i < SPT; ++i) {
                const bool real = mine && n0 + i < a.N;
                av[i] = real ? decay_rate(a.A[(size_t)d * a.N + n0 + i]) : 0.f;
                hv[i] = 0.f;
                if (!STATE_ONLY && real) {
                    if (a.segs > 1) hv[i] = a.local[(((size_t)b * a.segs + seg) * a.D + d) * NQ + n0 + i];
                    else if (a.state_in) hv[i] = a.state_in[((size_t)b * a.D + d) * a.N + n0 + i];
                }
            }
#pragma unroll
            for (int k = 0; k < P; ++k) A2[k] = make_float2(av[2 * k], av[2 * k + 1]), h[k] = make_float2(hv[2 * k], hv[2 * k + 1]);
        }
        float steps = 0.f;
        auto keep = [&](float* p) {                           // the thread's states, at [..][NQ] of its channel
            if (!mine || n0 >= NQ) return;
#pragma unroll
            for (int k = 0; k < SPT / 4; ++k)
                if (n0 + 4 * k < NQ) *reinterpret_cast<float4*>(p + n0 + 4 * k) = make_float4(h[2 * k].x, h[2 * k].y, h[2 * k + 1].x, h[2 * k + 1].y);
        };
        // B or C of the thread's states, in pairs
        auto pairs = [&](const float* p, float2 (&v)[P]) {
#pragma unroll
            for (int k = 0; k < SPT / 4; ++k) {
                const float4 q = *reinterpret_cast<const float4*>(p + 4 * k);
                v[2 * k] = make_float2(q.x, q.y), v[2 * k + 1] = make_float2(q.z, q.w);
            }
        };
        __syncthreads();                                      // tile 0 is there
        for (int k = 0; k < tiles; ++k) {
            const int t0 = t_begin + k * TT;
            float* yb = ys + (k & 1) * YB;
#pragma unroll 1
            for (int r0 = 0; r0 < TT; r0 += R) {
                if (!STATE_ONLY && a.states && r0 % kCheckpointRows == 0 && t0 + r0 < live) {
                    const int cks = (a.L + kCheckpointRows - 1) / kCheckpointRows, ck = (t0 + r0) / kCheckpointRows;
                    keep(a.states + (((size_t)b * cks + ck) * a.D + d) * NQ);
                }
                const float2* sp = dd + (k & 1) * DD + r0 * CB + ch;
                const float *Bp = bc + (k & 1) * BC + r0 * NP + n0, *Cp = Bp + TT * NP;
                float2 e[R][P], in[R][P];
#pragma unroll
                for (int j = 0; j < R; ++j) {
                    const float2 s = sp[j * CB];
                    float2 bv[P];
                    pairs(Bp + j * NP, bv);
                    if (STATE_ONLY) steps += s.x;
#pragma unroll
                    for (int i = 0; i < P; ++i) e[j][i] = decay(both(s.x), A2[i]), in[j][i] = __fmul2_rn(both(s.y), bv[i]);
                }
                float out[R];
#pragma unroll
                for (int j = 0; j < R; ++j) {
                    float2 o = both(0.f), cv[P];
                    if (!STATE_ONLY) pairs(Cp + j * NP, cv);
#pragma unroll
                    for (int i = 0; i < P; ++i) {
                        h[i] = __ffma2_rn(e[j][i], h[i], in[j][i]);
                        if (!STATE_ONLY) o = i ? __ffma2_rn(h[i], cv[i], o) : __fmul2_rn(h[i], cv[i]);
                    }
                    out[j] = o.x + o.y;
                }
                if (!STATE_ONLY) {
                    sum_over_lanes<R, NL, CL>(out, lane);     // leaves rows OWN * (sl / SHARE) ..
                    if (sl % SHARE == 0) {
#pragma unroll
                        for (int i = 0; i < OWN; ++i) yb[(r0 + sl / SHARE * OWN + i) * YS + ch] = out[i];
                    }
                }
            }
            __syncthreads();
        }
        const size_t at = ((size_t)b * a.segs + seg) * a.D + d;
        if (STATE_ONLY) {
            keep(a.local + at * NQ);
            if (mine && sl == 0) a.steps[at] = steps;
        } else if (a.state_out && seg == a.segs - 1 && mine) {
#pragma unroll
            for (int i = 0; i < SPT; ++i)
                if (n0 + i < a.N) a.state_out[((size_t)b * a.D + d) * a.N + n0 + i] = i % 2 ? h[i / 2].y : h[i / 2].x;
        }
        return;
    }

    // ---- the helping warps: four adjacent channels of a row at a time, the channels are the thread's own for the whole call
    const int tid = threadIdx.x - Tile::SCAN, uc = tid % (CB / 4) * 4, ur = tid / (CB / 4);
    float bias[4], skip[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        bias[i] = a.delta_bias && uc + i < nch ? a.delta_bias[d0 + uc + i] : 0.f;
        skip[i] = !STATE_ONLY && a.Dskip && uc + i < nch ? a.Dskip[d0 + uc + i] : 0.f;
    }
    const T *ub = a.u + row0 * a.ldu + d0, *db = a.delta + row0 * a.lddelta + d0, *zb = a.z + row0 * a.ldz + d0;
    const T *Bb = a.Bm + row0 * a.ldB + (long long)g * a.N, *Cb = a.Cm + row0 * a.ldC + (long long)g * a.N;
    T* yb = a.y + row0 * a.ldy + d0 + uc;
    auto fetch = [&](int k) {
        if (k < tiles) {
            T* p = raw + k % RAWS * RAW;
            const int t = t_begin + k * TT, rows = live - t;
            copy_tile<TT, CB, HT>(p, ub + (long long)t * a.ldu, a.ldu, rows, nch, a.u_unit, tid);
            copy_tile<TT, CB, HT>(p + TT * CB, db + (long long)t * a.lddelta, a.lddelta, rows, nch, a.delta_unit, tid);
            if (!STATE_ONLY && a.z) copy_tile<TT, CB, HT>(p + 2 * TT * CB, zb + (long long)t * a.ldz, a.ldz, rows, nch, a.z_unit, tid);
            copy_tile<TT, NP, HT>(p + 3 * TT * CB, Bb + (long long)t * a.ldB, a.ldB, rows, a.N, a.B_unit, tid);
            if (!STATE_ONLY) copy_tile<TT, NP, HT>(p + 3 * TT * CB + TT * NP, Cb + (long long)t * a.ldC, a.ldC, rows, a.N, a.C_unit, tid);
        }
        copies_commit();
    };
    auto convert = [&](int k) {
        const T* rw = raw + k % RAWS * RAW;
        const int rows = live - t_begin - k * TT;
#pragma unroll
        for (int i = 0; i < UK; ++i) {
            const int r = ur + i * UROWS;
            if (UNITS % HT != 0 && r >= TT) continue;
            float u[4], s[4];
            load4(rw + r * CB + uc, u);
            load4(rw + TT * CB + r * CB + uc, s);
            float2 s2[2] = {make_float2(s[0] + bias[0], s[1] + bias[1]), make_float2(s[2] + bias[2], s[3] + bias[3])};
            if (a.softplus) s2[0] = softplus(s2[0]), s2[1] = softplus(s2[1]);
            if (r >= rows) s2[0] = s2[1] = both(0.f);         // padding: the state stays
            float4* to = reinterpret_cast<float4*>(dd + (k & 1) * DD + r * CB + uc);
            to[0] = make_float4(s2[0].x, s2[0].x * u[0], s2[0].y, s2[0].y * u[1]);
            to[1] = make_float4(s2[1].x, s2[1].x * u[2], s2[1].y, s2[1].y * u[3]);
        }
        float* to = bc + (k & 1) * BC;
#pragma unroll
        for (int i = 0; i < BK; ++i) {
            const int e = (tid + i * HT) * 4;
            if (BUNITS % HT != 0 && e >= TT * NP) continue;
            float v[4];
            load4(rw + 3 * TT * CB + e, v);
            *reinterpret_cast<float4*>(to + e) = make_float4(v[0], v[1], v[2], v[3]);
            if (!STATE_ONLY) {
                load4(rw + 3 * TT * CB + TT * NP + e, v);
                *reinterpret_cast<float4*>(to + TT * NP + e) = make_float4(v[0], v[1], v[2], v[3]);
            }
        }
    };
    auto finish = [&](int k) {
        const T* rw = raw + k % RAWS * RAW;
        const float* yk = ys + (k & 1) * YB;
        const int rows = live - t_begin - k * TT;
#pragma unroll
        for (int i = 0; i < UK; ++i) {
            const int r = ur + i * UROWS;
            if (uc >= nch || r >= TT || r >= rows) continue;
            float u[4], o[4];
            load4(rw + r * CB + uc, u);
            const float4 y4 = *reinterpret_cast<const float4*>(yk + r * YS + uc);
            o[0] = fmaf(skip[0], u[0], y4.x), o[1] = fmaf(skip[1], u[1], y4.y), o[2] = fmaf(skip[2], u[2], y4.z), o[3] = fmaf(skip[3], u[3], y4.w);
            if (a.z) {
                float z[4];
                load4(rw + 2 * TT * CB + r * CB + uc, z);
#pragma unroll
                for (int j = 0; j < 4; ++j) o[j] *= z[j] * sigmoid(z[j]);
            }
            T* to = yb + (long long)(t_begin + k * TT + r) * a.ldy;
            if (a.y_quads) {
                store_pack(to, pack<T, 4>(o));
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (uc + j < nch) to[j] = from_float<T>(o[j]);
            }
        }
    };
    fetch(0);
    fetch(1);
    fetch(2);
    copies_wait<2>();
    helpers_sync<HT>();                                       // (every helper's copies have arrived)
    if (tiles) convert(0);
    __syncthreads();
    for (int k = 0; k < tiles; ++k) {
        // the buffer of tile k + 3 is that of tile k - 1, whose u and z `finish` still reads: it comes first
        if (!STATE_ONLY && k > 0) finish(k - 1);
        copies_wait<1>();
        helpers_sync<HT>();
        fetch(k + 3);
        if (k + 1 < tiles) convert(k + 1);
        __syncthreads();
    }
    if (STATE_ONLY) return;
    if (tiles) finish(tiles - 1);
    for (int t = max(t_begin, live) + ur; t < t_end; t += UROWS)
        for (int j = 0; j < 4 && uc + j < nch; ++j) yb[(long long)t * a.ldy + j] = from_float<T>(0.f);
}

}  // namespace conv2d_b200
