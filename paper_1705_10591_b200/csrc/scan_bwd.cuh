// Selective state space scan, backward.
//
//   g = dy silu(z),   e_t = C_t g_t + a_{t+1} e_{t+1}  with  a_t = exp(s_t A),   q_t = e_t a_t h_{t-1}
//   dC_t = sum_d g h_t,  dB_t = sum_d e s u,  dA = sum_t s q,  ds = sum_n A q + u sum_n e B,  du = s sum_n e B + Dskip g,
//   dz = dy v silu'(z),  dDskip = sum_t g u
//
// The forward pass keeps the state before every 16th row.  A block walks the tiles of 16 rows from the last to the first; in a tile the
// states h of all 16 rows are computed again, from the kept one, into registers (a thread has four states of one channel: 64
// registers; the decays beside them would make it one block an SM, so those are taken twice).  Sums over the states go over the lanes of a channel.
// Sums over the channels (dB, dC) are the larger part, eight values a row: two lanes join theirs, one going on with dB and one with dC (going
// on over all lanes took 32 of 95 instructions a row), and the rest is added through shared memory, over the warps and the channel sets that the block
// takes in turn, and goes into the workspace as one partial sum of the block; those are added by a kernel of their own in a fixed order.
// 4 x 2048 x 2048 of 16 states: about 433 us of the training step's 573.  The exponentials, twice, take 120 of them; shared memory is busy for two thirds of the
// time on the SMs that have two blocks (256 blocks are not a multiple of 148), eight of its 20 cycles a row and warp for the sums over channels.
// As in the forward pass four helping warps do what is done once per row and channel while the four scanning warps scan: copies, step sizes and
// gates of the next tile, outputs and sums over the warps of the last one.
#pragma once

#include "scan_common.cuh"

namespace conv2d_b200 {

constexpr int kSpt = 4;                 // states of a thread

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
    int ldu, lddelta, ldB, ldC, ldz, lddy, lddu, ldddelta, lddz;
    int u_unit, delta_unit, z_unit, dy_unit, B_unit, C_unit;         // bytes in which rows can be copied
    bool out_quads, softplus;                                         // out_quads: du, ddelta, dz can be stored four elements at a time
};

template <int NL>
struct ScanBwdTile {
    static constexpr int W = NL == 1 ? 2 : 4, SCAN = 32 * W, HELP = 128, TH = SCAN + HELP, RAWS = 4;
    static constexpr int CL = 32 / NL, CB = W * CL, NP = NL * kSpt, TT = kCheckpointRows, YS = CB + 4;
    static constexpr int PV = CL > 1 ? 1 : 2;                 // quads of a row that a lane leaves for the sums over channels
    static constexpr size_t raw(size_t esize) { return esize * TT * (4 * CB + 2 * NP); }
    // tiles as they lie in memory; twice (s, s u) and g of a tile, B and C, and three sums over states; the warps' sums over channels, and the block's
    static constexpr size_t fixed(size_t esize)
    {
        return RAWS * raw(esize) + sizeof(float) * (2 * (3 * TT * CB + 2 * TT * NP + 3 * TT * YS) + W * TT * PV * 128 + TT * 2 * NP);
    }
    // of a channel set: the carried gradient, dA and A of every scanning thread, and the helpers' sums for dDskip and ddelta_bias
    static constexpr size_t set_bytes = sizeof(float) * (SCAN * 3 * kSpt + HELP * 8);
};

template <typename T, int NL>
__global__ void __launch_bounds__(ScanBwdTile<NL>::TH, 2) scan_bwd_kernel(const ScanBwdArgs<T> a)
{
    using Tile = ScanBwdTile<NL>;
    constexpr int W = Tile::W, HT = Tile::HELP, CL = Tile::CL, CB = Tile::CB, NP = Tile::NP, TT = Tile::TT, YS = Tile::YS, RAWS = Tile::RAWS, ES = sizeof(T);
    constexpr int UNITS = TT * CB / 4, UK = (UNITS + HT - 1) / HT, UROWS = HT / (CB / 4), BUNITS = TT * NP / 4, BK = (BUNITS + HT - 1) / HT;
    constexpr int QQ = TT * CB, BC = 2 * TT * NP, SB = 3 * TT * YS, RAW = TT * (4 * CB + 2 * NP), SETS_TH = Tile::SCAN, PV = Tile::PV;
    ptx::grid_dep_wait();
    extern __shared__ float4 smem4[];
    float2* dd = reinterpret_cast<float2*>(smem4);            // [2][TT][CB] (s, s u)
    float* gg = reinterpret_cast<float*>(dd + 2 * QQ);        // [2][TT][CB] g
    float* bc = gg + 2 * QQ;                                  // [2] of B, C [TT][NP]
    float* sums = bc + 2 * BC;                                // [2] of sum_n C h, sum_n A2 q, sum_n e B [TT][YS]
    float4* parts = reinterpret_cast<float4*>(sums + 2 * SB); // [W][TT][PV][32]: of four states, dB in the lower channel lanes and dC in the upper
    float4* acc = parts + W * TT * PV * 32;                   // [TT][2][NP / 4]
    float4* carry4 = acc + TT * 2 * NP / 4;                   // [sets][SCAN]
    float4* dA4 = carry4 + a.sets * SETS_TH;
    float4* A24 = dA4 + a.sets * SETS_TH;
    float* chan = reinterpret_cast<float*>(A24 + a.sets * SETS_TH);  // [sets][8][HELP]: dDskip, ddelta_bias of the helper's four channels
    T* raw = reinterpret_cast<T*>(chan + a.sets * 8 * HT);           // [RAWS] of u, delta, z, dy [TT][CB], B, C [TT][NP]

    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
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
    const int NQ = round4(a.N), cks = (a.L + TT - 1) / TT;
    const int c_base = cb * CB * a.sets, sets = min(a.sets, (a.E - c_base + CB - 1) / CB);      // at least one
    const int tiles = live > t_begin ? (live - t_begin + TT - 1) / TT : 0, jobs = tiles * sets;
    // job k: set k % sets of the tile tiles - 1 - k / sets
    float* per_channel = a.per_channel + ((size_t)b * a.segs + seg) * channel_floats(a.D, NQ);

    if (warp < W) {                                           // ---- the scanning warps
        const int tid = threadIdx.x, chl = warp * CL + lane % CL, n0 = lane / CL * kSpt;
        for (int set = 0; set < sets; ++set) {
            const int c = c_base + set * CB + chl, d = g * a.E + c;
            float av[kSpt], cv[kSpt];
#pragma unroll
            for (int i = 0; i < kSpt; ++i) {
                const bool real = c < a.E && n0 + i < a.N;
                av[i] = real ? decay_rate(a.A[(size_t)d * a.N + n0 + i]) : 0.f;
                cv[i] = 0.f;
                if (real && a.segs > 1) cv[i] = a.local[(((size_t)b * a.segs + seg) * a.D + d) * NQ + n0 + i];
                else if (real && a.dstate_out) cv[i] = a.dstate_out[((size_t)b * a.D + d) * a.N + n0 + i];
            }
            A24[set * SETS_TH + tid] = make_float4(av[0], av[1], av[2], av[3]);
            carry4[set * SETS_TH + tid] = make_float4(cv[0], cv[1], cv[2], cv[3]);
            dA4[set * SETS_TH + tid] = make_float4(0.f, 0.f, 0.f, 0.f);
        }
        float4 kept = make_float4(0.f, 0.f, 0.f, 0.f);        // the state that the forward pass kept, loaded one job ahead
        auto load_kept = [&](int tile, int set) {
            const int c = c_base + set * CB + chl, d = g * a.E + c;
            if (c < a.E && n0 < NQ) kept = *reinterpret_cast<const float4*>(a.states + (((size_t)b * cks + t_begin / TT + tile) * a.D + d) * NQ + n0);
            else kept = make_float4(0.f, 0.f, 0.f, 0.f);
        };
        if (jobs) load_kept(tiles - 1, 0);
        int tile = tiles - 1, set = 0;
        __syncthreads();                                      // job 0 is there
#pragma unroll 1
        for (int k = 0; k < jobs; ++k) {
            const float4 A4 = A24[set * SETS_TH + tid];
            const float2 A2[2] = {make_float2(A4.x, A4.y), make_float2(A4.z, A4.w)};
            const float2 h0[2] = {make_float2(kept.x, kept.y), make_float2(kept.z, kept.w)};
            const int next_set = set + 1 < sets ? set + 1 : 0, next_tile = next_set ? tile : tile - 1;
            if (k + 1 < jobs) load_kept(next_tile, next_set);
            const float2* sp = dd + (k & 1) * QQ + chl;
            const float* gp = gg + (k & 1) * QQ + chl;
            const float *Bp = bc + (tile & 1) * BC + n0, *Cp = Bp + TT * NP;
            float *vs = sums + (k & 1) * SB + chl, *s1 = vs + TT * YS, *s2 = s1 + TT * YS;
            float4* pp = parts + warp * TT * PV * 32 + lane;
            float2 h[TT][2];
#pragma unroll
            for (int t = 0; t < TT; ++t) {
                const float2 q = sp[t * CB];
                const float4 bv = *reinterpret_cast<const float4*>(Bp + t * NP);
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    h[t][i] = __ffma2_rn(decay(both(q.x), A2[i]), t ? h[t - 1][i] : h0[i],
                                         __fmul2_rn(both(q.y), i ? make_float2(bv.z, bv.w) : make_float2(bv.x, bv.y)));
            }
            __syncthreads();                                  // the helpers have added the last job's sums over channels
            const float4 c4 = carry4[set * SETS_TH + tid], w4 = dA4[set * SETS_TH + tid];
            float2 carry[2] = {make_float2(c4.x, c4.y), make_float2(c4.z, c4.w)}, dA[2] = {make_float2(w4.x, w4.y), make_float2(w4.z, w4.w)};
            // (a row's operands are read before the sums of the row before are stored: the compiler may not move them across)
            struct Row { float2 q; float g; float4 b, c; };
            auto read = [&](int t) {
                return Row{sp[t * CB], gp[t * CB], *reinterpret_cast<const float4*>(Bp + t * NP), *reinterpret_cast<const float4*>(Cp + t * NP)};
            };
            Row next_row = read(TT - 1);
            // The sums over the lanes of four rows are joined between the next four rows: a warp issues in order, and would wait for each exchange
            float n_prev[8], v_prev[4];
            auto join = [&](int stage) {
                sum_stage<4, NL, CL>(v_prev, lane, stage);
                sum_stage<8, NL, CL>(n_prev, lane, stage);
            };
            auto store = [&](int tq) {
                constexpr int v_left = NL >= 4 ? 1 : 4 / NL, n_left = NL >= 8 ? 1 : 8 / NL;
                if (first_of_equals<4, NL, CL>(lane)) {
#pragma unroll
                    for (int i = 0; i < v_left; ++i) vs[(tq + first_value<4, NL, CL>(lane) + i) * YS] = v_prev[i];
                }
                if (first_of_equals<8, NL, CL>(lane)) {
#pragma unroll
                    for (int i = 0; i < n_left; ++i) {
                        const int id = first_value<8, NL, CL>(lane) + i;
                        (id >> 2 ? s2 : s1)[(tq + (id & 3)) * YS] = n_prev[i];
                    }
                }
            };
#pragma unroll
            for (int tq = TT - 4; tq >= 0; tq -= 4) {
                float n_sums[8], v[4];                        // sum_n A2 q of four rows, then sum_n e B; sum_n C h
#pragma unroll
                for (int j = 3; j >= 0; --j) {
                    const int t = tq + j;
                    const float2 q = next_row.q, s_2 = both(q.x), su2 = both(q.y), g2 = both(next_row.g);
                    const float4 bv = next_row.b, cv = next_row.c;
                    if (t > 0) next_row = read(t - 1);
                    float2 Aq, eB, o;
                    float db[4], dc[4];                       // e s u and g h of the four states
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const float2 e = __ffma2_rn(i ? make_float2(cv.z, cv.w) : make_float2(cv.x, cv.y), g2, carry[i]);
                        carry[i] = __fmul2_rn(decay_again(s_2, A2[i]), e);
                        const float2 qq = __fmul2_rn(carry[i], t ? h[t - 1][i] : h0[i]), bi = i ? make_float2(bv.z, bv.w) : make_float2(bv.x, bv.y);
                        dA[i] = __ffma2_rn(s_2, qq, dA[i]);
                        Aq = i ? __ffma2_rn(A2[i], qq, Aq) : __fmul2_rn(A2[i], qq);
                        eB = i ? __ffma2_rn(e, bi, eB) : __fmul2_rn(e, bi);
                        const float2 x = __fmul2_rn(e, su2), y = __fmul2_rn(g2, h[t][i]), ci = i ? make_float2(cv.z, cv.w) : make_float2(cv.x, cv.y);
                        o = i ? __ffma2_rn(h[t][i], ci, o) : __fmul2_rn(h[t][i], ci);
                        db[2 * i] = x.x, db[2 * i + 1] = x.y, dc[2 * i] = y.x, dc[2 * i + 1] = y.y;
                    }
                    n_sums[j] = Aq.x + Aq.y;
                    n_sums[4 + j] = eB.x + eB.y;
                    v[j] = o.x + o.y;
                    if (CL > 1) {
                        const bool upper = lane & (CL / 2);
                        float r[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) r[i] = (upper ? dc[i] : db[i]) + __shfl_xor_sync(0xffffffffu, upper ? db[i] : dc[i], CL / 2);
                        pp[t * 32] = make_float4(r[0], r[1], r[2], r[3]);
                    } else {
                        pp[t * 64] = make_float4(db[0], db[1], db[2], db[3]);
                        pp[t * 64 + 32] = make_float4(dc[0], dc[1], dc[2], dc[3]);
                    }
                    if (tq < TT - 4) {
                        join(3 - j);
                        if (j == 0) join(4), store(tq + 4);
                    }
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) n_prev[i] = n_sums[i];
#pragma unroll
                for (int i = 0; i < 4; ++i) v_prev[i] = v[i];
            }
#pragma unroll
            for (int stage = 0; NL >> (stage + 1); ++stage) join(stage);
            store(0);
            carry4[set * SETS_TH + tid] = make_float4(carry[0].x, carry[0].y, carry[1].x, carry[1].y);
            dA4[set * SETS_TH + tid] = make_float4(dA[0].x, dA[0].y, dA[1].x, dA[1].y);
            set = next_set, tile = next_tile;
            __syncthreads();
        }
        for (int set = 0; set < sets; ++set) {
            const int c = c_base + set * CB + chl, d = g * a.E + c;
            if (c >= a.E) continue;
            if (n0 < NQ) *reinterpret_cast<float4*>(per_channel + (size_t)d * NQ + n0) = dA4[set * SETS_TH + tid];
            if (a.dstate_in && a.segs == 1) {
                const float4 c4 = carry4[set * SETS_TH + tid];
                const float cv[kSpt] = {c4.x, c4.y, c4.z, c4.w};
#pragma unroll
                for (int i = 0; i < kSpt; ++i)
                    if (n0 + i < a.N) a.dstate_in[((size_t)b * a.D + d) * a.N + n0 + i] = cv[i];
            }
        }
        return;
    }

    // ---- the helping warps: four adjacent channels of a row at a time, the same of every set
    const int tid = threadIdx.x - Tile::SCAN, uc = tid % (CB / 4) * 4, ur = tid / (CB / 4);
    for (int i = tid; i < sets * 8 * HT; i += HT) chan[i] = 0.f;
    // job k of each of three streams (copies, conversions, outputs), counted along
    struct Job { int k, tile, set; };
    auto next = [&](Job& j) {
        ++j.k;
        if (++j.set == sets) j.set = 0, --j.tile;
    };
    float bias[4], skip[4], sum_d[4] = {}, sum_b[4] = {};
    auto params = [&](int set) {                              // of the helper's four channels
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int c = c_base + set * CB + uc + j;
            bias[j] = a.delta_bias && c < a.E ? a.delta_bias[g * a.E + c] : 0.f;
            skip[j] = a.Dskip && c < a.E ? a.Dskip[g * a.E + c] : 0.f;
        }
    };
    params(0);
    const int db0 = g * a.E + c_base;
    const T *ub = a.u + row0 * a.ldu + db0, *db = a.delta + row0 * a.lddelta + db0, *zb = a.z + row0 * a.ldz + db0, *gb = a.dy + row0 * a.lddy + db0;
    const T *Bb = a.Bm + row0 * a.ldB + (long long)g * a.N, *Cb = a.Cm + row0 * a.ldC + (long long)g * a.N;
    T *dub = a.du + row0 * a.lddu + db0 + uc, *ddb = a.ddelta + row0 * a.ldddelta + db0 + uc, *dzb = a.dz + row0 * a.lddz + db0 + uc;
    auto fetch = [&](const Job& job) {
        const int tile = job.tile, set = job.set;
        if (job.k < jobs) {
            T* p = raw + job.k % RAWS * RAW;
            const int c0 = set * CB, nch = min(CB, a.E - c_base - c0), t = t_begin + tile * TT, rows = live - t;
            copy_tile<TT, CB, HT>(p, ub + (long long)t * a.ldu + c0, a.ldu, rows, nch, a.u_unit, tid);
            copy_tile<TT, CB, HT>(p + QQ, db + (long long)t * a.lddelta + c0, a.lddelta, rows, nch, a.delta_unit, tid);
            if (a.z) copy_tile<TT, CB, HT>(p + 2 * QQ, zb + (long long)t * a.ldz + c0, a.ldz, rows, nch, a.z_unit, tid);
            copy_tile<TT, CB, HT>(p + 3 * QQ, gb + (long long)t * a.lddy + c0, a.lddy, rows, nch, a.dy_unit, tid);
            if (set == 0) {
                copy_tile<TT, NP, HT>(p + 4 * QQ, Bb + (long long)t * a.ldB, a.ldB, rows, a.N, a.B_unit, tid);
                copy_tile<TT, NP, HT>(p + 4 * QQ + TT * NP, Cb + (long long)t * a.ldC, a.ldC, rows, a.N, a.C_unit, tid);
            }
        }
        copies_commit();
    };
    auto convert = [&](const Job& job) {
        const int k = job.k, tile = job.tile, set = job.set, c0 = c_base + set * CB, rows = live - t_begin - tile * TT;
        const T* rw = raw + k % RAWS * RAW;
        if (sets > 1) params(set);
#pragma unroll
        for (int i = 0; i < UK; ++i) {
            const int r = ur + i * UROWS;
            if (UNITS % HT != 0 && r >= TT) continue;
            float u[4], s[4], gr[4];
            load4(rw + r * CB + uc, u);
            load4(rw + QQ + r * CB + uc, s);
            load4(rw + 3 * QQ + r * CB + uc, gr);
            float2 s2[2], g2[2] = {make_float2(gr[0], gr[1]), make_float2(gr[2], gr[3])};
            s2[0] = make_float2(s[0] + bias[0], s[1] + bias[1]), s2[1] = make_float2(s[2] + bias[2], s[3] + bias[3]);
            if (a.softplus) s2[0] = softplus(s2[0]), s2[1] = softplus(s2[1]);
            if (r >= rows) s2[0] = s2[1] = both(0.f);
            if (a.z) {
                float z[4];
                load4(rw + 2 * QQ + r * CB + uc, z);
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const float2 zz = make_float2(z[2 * j], z[2 * j + 1]);
                    g2[j] = __fmul2_rn(g2[j], __fmul2_rn(zz, sigmoid(zz)));
                }
            }
            const float sv[4] = {s2[0].x, s2[0].y, s2[1].x, s2[1].y}, gv[4] = {g2[0].x, g2[0].y, g2[1].x, g2[1].y};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float sj = c0 + uc + j < a.E ? sv[j] : 0.f;
                dd[(k & 1) * QQ + r * CB + uc + j] = make_float2(sj, sj * u[j]);
            }
            *reinterpret_cast<float4*>(gg + (k & 1) * QQ + r * CB + uc) = make_float4(gv[0], gv[1], gv[2], gv[3]);
        }
        if (set == 0) {
            float* to = bc + (tile & 1) * BC;
#pragma unroll
            for (int i = 0; i < BK; ++i) {
                const int e = (tid + i * HT) * 4;
                if (BUNITS % HT != 0 && e >= TT * NP) continue;
                float v[4];
                load4(rw + 4 * QQ + e, v);
                *reinterpret_cast<float4*>(to + e) = make_float4(v[0], v[1], v[2], v[3]);
                load4(rw + 4 * QQ + TT * NP + e, v);
                *reinterpret_cast<float4*>(to + TT * NP + e) = make_float4(v[0], v[1], v[2], v[3]);
            }
        }
    };
    // sums over channels of a job: a thread takes four states of dB or dC of a row, their RL lanes of every warp
    constexpr int RL = CL > 1 ? CL / 2 : 1, TASKS = TT * 2 * NL;
    float* per_row = a.per_row + (((size_t)g * a.blocks_group + cb) * a.B * a.L + row0) * (2 * NP);
    auto add_parts = [&](const Job& job) {
        const int t0 = t_begin + job.tile * TT;
        const bool out = job.set == sets - 1;
        float4* to = reinterpret_cast<float4*>(per_row + (size_t)t0 * (2 * NP));
#pragma unroll
        for (int i = 0; i < (TASKS + HT - 1) / HT; ++i) {
            const int task = tid + i * HT, t = task / (2 * NL), sl = task / 2 % NL, which = task % 2;
            if (TASKS % HT != 0 && task >= TASKS) continue;
            const float4* p = parts + t * PV * 32 + (CL > 1 ? sl * CL + which * RL : which * 32 + sl);
            float2 lo = both(0.f), hi = both(0.f);
#pragma unroll
            for (int w = 0; w < W; ++w)
#pragma unroll
                for (int r = 0; r < RL; ++r) {                // (begun at different lanes, in different banks)
                    const float4 v = p[w * TT * PV * 32 + ((r + task / 2) & (RL - 1))];
                    lo = __fadd2_rn(lo, make_float2(v.x, v.y)), hi = __fadd2_rn(hi, make_float2(v.z, v.w));
                }
            const int at = (t * 2 + which) * (NP / 4) + sl;
            if (sets > 1) {
                const float4 v = acc[at];
                if (job.set > 0) lo = __fadd2_rn(lo, make_float2(v.x, v.y)), hi = __fadd2_rn(hi, make_float2(v.z, v.w));
                acc[at] = make_float4(lo.x, lo.y, hi.x, hi.y);
            }
            if (out && t0 + t < live) to[at] = make_float4(lo.x, lo.y, hi.x, hi.y);
        }
    };
    auto finish = [&](const Job& job) {
        const int k = job.k, tile = job.tile, set = job.set, c0 = c_base + set * CB, rows = live - t_begin - tile * TT, nch = a.E - c0;
        const T* rw = raw + k % RAWS * RAW;
        const float *vs = sums + (k & 1) * SB, *s1 = vs + TT * YS, *s2 = s1 + TT * YS;
        float* mine = chan + set * 8 * HT + tid;
        if (sets > 1) {
            params(set);
#pragma unroll
            for (int j = 0; j < 4; ++j) sum_d[j] = mine[j * HT], sum_b[j] = mine[(4 + j) * HT];
        }
#pragma unroll
        for (int i = 0; i < UK; ++i) {
            const int r = ur + i * UROWS;
            if (uc >= nch || r >= TT || r >= rows) continue;
            float u[4], rd[4], gy[4], du[4], ds[4];
            load4(rw + r * CB + uc, u);
            load4(rw + QQ + r * CB + uc, rd);
            load4(rw + 3 * QQ + r * CB + uc, gy);
            const float4 v4 = *reinterpret_cast<const float4*>(vs + r * YS + uc), a4 = *reinterpret_cast<const float4*>(s1 + r * YS + uc),
                         e4 = *reinterpret_cast<const float4*>(s2 + r * YS + uc);
            const float v[4] = {v4.x, v4.y, v4.z, v4.w}, sa[4] = {a4.x, a4.y, a4.z, a4.w}, se[4] = {e4.x, e4.y, e4.z, e4.w};
            const int t = t_begin + tile * TT + r;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float sj = dd[(k & 1) * QQ + r * CB + uc + j].x, gj = gg[(k & 1) * QQ + r * CB + uc + j];
                du[j] = fmaf(sj, se[j], skip[j] * gj);
                ds[j] = fmaf(kLn2, sa[j], u[j] * se[j]);
                if (a.softplus) ds[j] *= sigmoid(rd[j] + bias[j]);
                sum_d[j] = fmaf(gj, u[j], sum_d[j]);
                sum_b[j] += ds[j];
            }
            T* to_u = dub + (long long)t * a.lddu + set * CB;
            T* to_d = ddb + (long long)t * a.ldddelta + set * CB;
            if (a.out_quads) {
                store_pack(to_u, pack<T, 4>(du));
                store_pack(to_d, pack<T, 4>(ds));
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (uc + j < nch) to_u[j] = from_float<T>(du[j]), to_d[j] = from_float<T>(ds[j]);
            }
            if (a.z) {
                float z[4];
                load4(rw + 2 * QQ + r * CB + uc, z);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float sg = sigmoid(z[j]);
                    z[j] = gy[j] * fmaf(skip[j], u[j], v[j]) * sg * fmaf(z[j], 1.f - sg, 1.f);
                }
                T* to_z = dzb + (long long)t * a.lddz + set * CB;
                if (a.out_quads) {
                    store_pack(to_z, pack<T, 4>(z));
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (uc + j < nch) to_z[j] = from_float<T>(z[j]);
                }
            }
        }
        if (sets > 1) {
#pragma unroll
            for (int j = 0; j < 4; ++j) mine[j * HT] = sum_d[j], mine[(4 + j) * HT] = sum_b[j];
        }
    };
    Job in{0, tiles - 1, 0}, mid = in, last = in;
    for (int i = 0; i < 3; ++i, next(in)) fetch(in);
    copies_wait<2>();
    helpers_sync<HT>();                                       // (every helper's copies have arrived)
    if (jobs) convert(mid);
    next(mid);
    __syncthreads();
    for (int k = 0; k < jobs; ++k) {
        if (k > 0) add_parts(last);
        __syncthreads();
        // the buffer of job k + 3 is that of job k - 1, which `finish` still reads, as it does the (s, s u) and g that job k + 1 replaces
        if (k > 0) {
            finish(last);
            next(last);
        }
        copies_wait<1>();
        helpers_sync<HT>();
        fetch(in);
        next(in);
        if (k + 1 < jobs) convert(mid);
        next(mid);
        __syncthreads();
    }
    if (jobs) {
        add_parts(last);
        finish(last);
    }
    if (sets == 1) {
#pragma unroll
        for (int j = 0; j < 4; ++j) chan[j * HT + tid] = sum_d[j], chan[(4 + j) * HT + tid] = sum_b[j];
    }
    for (int set = 0; set < sets; ++set) {                    // rows of padding
        const int c = c_base + set * CB + uc;
        for (int t = max(t_begin, live) + ur; t < t_end; t += UROWS)
            for (int j = 0; j < 4 && c + j < a.E; ++j) {
                const int at = set * CB + j;
                dub[(long long)t * a.lddu + at] = ddb[(long long)t * a.ldddelta + at] = from_float<T>(0.f);
                if (a.z) dzb[(long long)t * a.lddz + at] = from_float<T>(0.f);
            }
    }
    helpers_sync<HT>();
    for (int i = tid; i < sets * 2 * CB; i += HT) {
        const int c = i % CB, which = i / CB % 2, set = i / (2 * CB), cc = c_base + set * CB + c;
        if (cc >= a.E) continue;
        float s = 0.f;
        for (int r = 0; r < UROWS; ++r) s += chan[(set * 8 + which * 4 + c % 4) * HT + r * (CB / 4) + c / 4];
        per_channel[(size_t)a.D * NQ + (size_t)which * a.D + g * a.E + cc] = s;
    }
}

// What a segment hands to the one before it when it is walked from zero: carry <- a_t (C_t g_t + carry), and the sum of its steps.
template <typename T, int NL, int V>
__global__ void __launch_bounds__(ScanBwdTile<NL>::SCAN) scan_bwd_carry_kernel(const ScanBwdArgs<T> a, int blocks_group)
{
    using Tile = ScanBwdTile<NL>;
    constexpr int TH = Tile::SCAN, CL = Tile::CL, CB = Tile::CB, NP = Tile::NP, TT = Tile::TT;
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
    const int ch = warp * CL + lane % CL, n0 = lane / CL * kSpt, NQ = round4(a.N), d = g * a.E + c0 + ch;
    const bool mine = c0 + ch < a.E;
    const int pk = (tid % PPR) * V, prow = tid / PPR;
    const bool pk_real = c0 + pk < a.E;
    float2 A2[2], carry[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
    float av[kSpt], bias[V], steps = 0.f;
#pragma unroll
    for (int i = 0; i < kSpt; ++i) av[i] = mine && n0 + i < a.N ? decay_rate(a.A[(size_t)d * a.N + n0 + i]) : 0.f;
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
            const float2 e0 = decay(s_2, A2[0]), e1 = decay(s_2, A2[1]);
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
