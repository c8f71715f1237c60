// Selective state space scan, forward.
//
//   h_t = exp(s_t A) h_{t-1} + s_t u_t B_t,   v_t = C_t . h_t + Dskip u_t,   y_t = v_t silu(z_t)
//
// Every (row, channel, state) takes an exponential of its own, so the special-function units (16 a clock and SM) set the pace, not memory:
// 16384 x 4096 channels of 16 states take 239 us of them on all SMs, 276 on the 128 that such a call has blocks for, and 605 in all;
// without the helpers' work beside it the scan alone takes 495, so the rest is what two warps of a scheduler take from each other.
// A block takes the channels of its W scanning warps and walks the rows of a sequence in tiles of TT; four more warps do what is done once
// per row and channel, so that the scanning warps, of which a batch of a few thousand channels gives one or two to a scheduler, only scan: while
// tile k is scanned, they bring tile k + 3 in (asynchronous copies), put s and s u of tile k + 1 into shared memory beside its B and C in fp32,
// and gate and store the sums over the states of tile k - 1.  A scanning warp waits for nothing if it can help it (see the loop): 684 us with the
// exponentials of eight rows together before the recurrence over them.
// Two blocks an SM: 128 registers (80 with eight scanning warps, which spill 5 to 9 registers and are still 12 % faster than one block).
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
    bool wide, y_quads, softplus;                     // wide: all of them 16; y_quads: y can be stored four elements at a time
};

template <int NL, int SPT>
struct ScanFwdTile {
    static constexpr int CL = 32 / NL, NP = NL * SPT, R = 8, W = NL >= 16 ? 8 : 4, CB = W * CL, TT = CB >= 64 || NP >= 64 ? 16 : 32;
    static constexpr int SCAN = 32 * W, HELP = 128, TH = SCAN + HELP, RAWS = 4;
    static constexpr int YS = CB + 4;                 // (the lanes that store a row's sums hit different banks)
    static constexpr size_t raw(size_t esize) { return esize * TT * (3 * CB + 2 * NP); }              // one tile as it lies in memory
    static constexpr size_t smem(size_t esize) { return RAWS * raw(esize) + sizeof(float) * 2 * (2 * TT * CB + 2 * TT * NP + TT * YS); }
};

template <typename T, int NL, int SPT, bool STATE_ONLY>
__global__ void __launch_bounds__(ScanFwdTile<NL, SPT>::TH, 2) scan_fwd_kernel(const ScanFwdArgs<T> a)
{
    using Tile = ScanFwdTile<NL, SPT>;
    constexpr int CL = Tile::CL, CB = Tile::CB, NP = Tile::NP, R = Tile::R, TT = Tile::TT, HT = Tile::HELP, YS = Tile::YS, P = SPT / 2;
    constexpr bool WIDE = CB * sizeof(T) >= 16 && NP * sizeof(T) >= 16;
    constexpr int OWN = NL >= R ? 1 : R / NL, SHARE = NL > R ? NL / R : 1;      // rows of a lane after a sum; lanes that have the same row
    constexpr int UNITS = TT * CB / 4, UK = (UNITS + HT - 1) / HT, BUNITS = TT * NP / 4, BK = (BUNITS + HT - 1) / HT, UROWS = HT / (CB / 4);
    constexpr int DD = TT * CB, BC = 2 * TT * NP, YB = TT * YS, RAW = TT * (3 * CB + 2 * NP), RAWS = Tile::RAWS, AHEAD = 2;
    using Yes = std::true_type;
    using No = std::false_type;
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
            const float2* sp = dd + (k & 1) * DD + ch;
            const float *Bp = bc + (k & 1) * BC + n0, *Cp = Bp + TT * NP;
            // A warp issues in order, so what it waits for has to be spread by hand: the exponentials and inputs are taken AHEAD rows before they are
            // used, their operands are read a row before that, and a group's sums over the lanes are joined between the rows of the next one.
            float2 e[AHEAD][P], in[AHEAD][P];
            struct Row { float2 s, b[P]; };
            auto read = [&](int r) {
                Row v;
                v.s = sp[r * CB];
                pairs(Bp + r * NP, v.b);
                return v;
            };
            auto prepare = [&](const Row& v, int j) {
                if (STATE_ONLY) steps += v.s.x;
#pragma unroll
                for (int i = 0; i < P; ++i) e[j][i] = decay(both(v.s.x), A2[i]), in[j][i] = __fmul2_rn(both(v.s.y), v.b[i]);
            };
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) prepare(read(j), j);
            Row next = read(AHEAD);
            float2 cv[P], cn[P];
            if (!STATE_ONLY) pairs(Cp, cn);
            float out[R], sums[R];
            auto store = [&](int r0) {                        // rows OWN * (sl / SHARE) ..
                if (sl % SHARE == 0) {
#pragma unroll
                    for (int i = 0; i < OWN; ++i) yb[(r0 + sl / SHARE * OWN + i) * YS + ch] = sums[i];
                }
            };
            auto group = [&](int r0, auto first, auto last) {
                if (!STATE_ONLY && a.states && r0 % kCheckpointRows == 0 && t0 + r0 < live) {
                    const int cks = (a.L + kCheckpointRows - 1) / kCheckpointRows, ck = (t0 + r0) / kCheckpointRows;
                    keep(a.states + (((size_t)b * cks + ck) * a.D + d) * NQ);
                }
#pragma unroll
                for (int j = 0; j < R; ++j) {
                    float2 o = both(0.f);
#pragma unroll
                    for (int i = 0; i < P; ++i) cv[i] = cn[i];
                    if (!STATE_ONLY && !(decltype(last)::value && j == R - 1)) pairs(Cp + (r0 + j + 1) * NP, cn);
#pragma unroll
                    for (int i = 0; i < P; ++i) {
                        h[i] = __ffma2_rn(e[j % AHEAD][i], h[i], in[j % AHEAD][i]);
                        if (!STATE_ONLY) o = i ? __ffma2_rn(h[i], cv[i], o) : __fmul2_rn(h[i], cv[i]);
                    }
                    out[j] = o.x + o.y;
                    if (!decltype(last)::value || j + AHEAD < R) {
                        const Row now = next;
                        if (!decltype(last)::value || j + AHEAD + 1 < R) next = read(r0 + AHEAD + j + 1);
                        prepare(now, j % AHEAD);
                    }
                    if (!STATE_ONLY && !decltype(first)::value && j % 2 == 1) sum_stage<R, NL, CL>(sums, lane, j / 2);
                }
                if (!STATE_ONLY) {
                    if (!decltype(first)::value) store(r0 - R);
#pragma unroll
                    for (int j = 0; j < R; ++j) sums[j] = out[j];
                }
            };
            group(0, Yes(), No());
#pragma unroll 1
            for (int r0 = R; r0 < TT - R; r0 += R) group(r0, No(), No());
            group(TT - R, No(), Yes());
            if (!STATE_ONLY) {
#pragma unroll
                for (int stage = 0; stage < R / 2; ++stage) sum_stage<R, NL, CL>(sums, lane, stage);
                store(TT - R);
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
            const T *u = ub + (long long)t * a.ldu, *s = db + (long long)t * a.lddelta, *z = zb + (long long)t * a.ldz;
            const T *Bt = Bb + (long long)t * a.ldB, *Ct = Cb + (long long)t * a.ldC;
            if (WIDE && a.wide) {
                copy_tile_by<TT, CB, 16, HT>(p, u, a.ldu, rows, nch, tid);
                copy_tile_by<TT, CB, 16, HT>(p + TT * CB, s, a.lddelta, rows, nch, tid);
                copy_tile_by<TT, NP, 16, HT>(p + 3 * TT * CB, Bt, a.ldB, rows, a.N, tid);
                if (!STATE_ONLY) {
                    if (a.z) copy_tile_by<TT, CB, 16, HT>(p + 2 * TT * CB, z, a.ldz, rows, nch, tid);
                    copy_tile_by<TT, NP, 16, HT>(p + 3 * TT * CB + TT * NP, Ct, a.ldC, rows, a.N, tid);
                }
            } else {
                copy_tile<TT, CB, HT>(p, u, a.ldu, rows, nch, a.u_unit, tid);
                copy_tile<TT, CB, HT>(p + TT * CB, s, a.lddelta, rows, nch, a.delta_unit, tid);
                copy_tile<TT, NP, HT>(p + 3 * TT * CB, Bt, a.ldB, rows, a.N, a.B_unit, tid);
                if (!STATE_ONLY) {
                    if (a.z) copy_tile<TT, CB, HT>(p + 2 * TT * CB, z, a.ldz, rows, nch, a.z_unit, tid);
                    copy_tile<TT, NP, HT>(p + 3 * TT * CB + TT * NP, Ct, a.ldC, rows, a.N, a.C_unit, tid);
                }
            }
        }
        copies_commit();
    };
    // (branches are taken once for all units of a thread: their operations stay side by side)
    auto row_of = [&](int i) { return UNITS % HT != 0 ? min(ur + i * UROWS, TT - 1) : ur + i * UROWS; };
    auto convert = [&](int k) {
        const T* rw = raw + k % RAWS * RAW;
        const int rows = live - t_begin - k * TT;
        float u[UK][4], b[BK][4], c[BK][4];
        float2 s2[UK][2];
#pragma unroll
        for (int i = 0; i < UK; ++i) {
            float s[4];
            load4(rw + row_of(i) * CB + uc, u[i]);
            load4(rw + TT * CB + row_of(i) * CB + uc, s);
            s2[i][0] = make_float2(s[0] + bias[0], s[1] + bias[1]), s2[i][1] = make_float2(s[2] + bias[2], s[3] + bias[3]);
        }
#pragma unroll
        for (int i = 0; i < BK; ++i) {
            const int e = BUNITS % HT != 0 ? min((tid + i * HT) * 4, TT * NP - 4) : (tid + i * HT) * 4;
            load4(rw + 3 * TT * CB + e, b[i]);
            if (!STATE_ONLY) load4(rw + 3 * TT * CB + TT * NP + e, c[i]);
        }
        if (a.softplus) {
#pragma unroll
            for (int i = 0; i < UK; ++i) s2[i][0] = softplus(s2[i][0]), s2[i][1] = softplus(s2[i][1]);
        }
#pragma unroll
        for (int i = 0; i < UK; ++i) {
            const int r = ur + i * UROWS;
            if (UNITS % HT != 0 && r >= TT) continue;
            if (r >= rows) s2[i][0] = s2[i][1] = both(0.f);   // padding: the state stays
            float4* to = reinterpret_cast<float4*>(dd + (k & 1) * DD + r * CB + uc);
            to[0] = make_float4(s2[i][0].x, s2[i][0].x * u[i][0], s2[i][0].y, s2[i][0].y * u[i][1]);
            to[1] = make_float4(s2[i][1].x, s2[i][1].x * u[i][2], s2[i][1].y, s2[i][1].y * u[i][3]);
        }
        float* to = bc + (k & 1) * BC;
#pragma unroll
        for (int i = 0; i < BK; ++i) {
            const int e = (tid + i * HT) * 4;
            if (BUNITS % HT != 0 && e >= TT * NP) continue;
            *reinterpret_cast<float4*>(to + e) = make_float4(b[i][0], b[i][1], b[i][2], b[i][3]);
            if (!STATE_ONLY) *reinterpret_cast<float4*>(to + TT * NP + e) = make_float4(c[i][0], c[i][1], c[i][2], c[i][3]);
        }
    };
    auto finish = [&](int k) {
        const T* rw = raw + k % RAWS * RAW;
        const float* yk = ys + (k & 1) * YB;
        const int rows = live - t_begin - k * TT;
        float o[UK][4];
#pragma unroll
        for (int i = 0; i < UK; ++i) {
            float u[4];
            load4(rw + row_of(i) * CB + uc, u);
            const float4 y4 = *reinterpret_cast<const float4*>(yk + row_of(i) * YS + uc);
            o[i][0] = fmaf(skip[0], u[0], y4.x), o[i][1] = fmaf(skip[1], u[1], y4.y), o[i][2] = fmaf(skip[2], u[2], y4.z), o[i][3] = fmaf(skip[3], u[3], y4.w);
        }
        if (a.z) {
#pragma unroll
            for (int i = 0; i < UK; ++i) {
                float z[4];
                load4(rw + 2 * TT * CB + row_of(i) * CB + uc, z);
#pragma unroll
                for (int j = 0; j < 4; ++j) o[i][j] *= z[j] * sigmoid(z[j]);
            }
        }
#pragma unroll
        for (int i = 0; i < UK; ++i) {
            const int r = ur + i * UROWS;
            if (uc >= nch || r >= TT || r >= rows) continue;
            T* to = yb + (long long)(t_begin + k * TT + r) * a.ldy;
            if (a.y_quads) {
                store_pack(to, pack<T, 4>(o[i]));
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (uc + j < nch) to[j] = from_float<T>(o[i][j]);
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
