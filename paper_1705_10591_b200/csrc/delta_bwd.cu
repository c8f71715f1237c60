// Gated delta rule, backward.  With dS the gradient of the state behind a piece (D_ij = e^(G_i - G_j); E, t and P' as in the forward pass):
//   X = diag(e^(G_63 - G)) K dS,   W = X + [-t; P']^T [beta X; scale dO],   dV = beta W,   dbeta = rows of W . E,
//   dS <- e^(G_63) dS + [K; Q]^T [-e^G dV; scale e^G dO]
// walks the pieces from the last one back; then every piece by itself:
//   p = D o (scale dO (beta E)^T), j <= i;   y = -D o (dV (beta E)^T), j < i;
//   dq = scale e^G dO S^T + p K;   dk = a + c,  a = y K - e^G dV S^T,  c = p^T Q + y^T K + e^(G_63 - G) beta E dS^T,
//   dG_i = q_i.dq_i + k_i.a_i - k_i.c_i,   dg_t = sum of dG_i, i >= t, + <S after the piece, dS>  or  <S, dS before the piece> - sum of dG_i, i < t
// (every exponential of G stands beside a query or key: what scales them says what the exponent would have done).  The first half of a piece's tokens takes the second
// form: it adds fewer numbers there, and where there is no state to decay nothing is left of it, where the first form leaves the gradient of a sequence's first gate, which is
// zero without state_in, as what rounding makes of it.  (It takes 0.8 % of a training step of 4 x 2048 x 16 heads.)
#include "delta_walk.cuh"

namespace conv2d_b200 {
namespace {

template <typename T, int KD, int NV, bool WIDE>
__global__ void __launch_bounds__(kWalkThreads, 1) delta_bwd_walk_kernel(const DeltaArgs a, int across)
{
    using W = Walk<T, KD, NV, 2 * kPiece>;
    constexpr int IN = W::IN, C = W::C, STAGES = W::stages;
    extern __shared__ unsigned char unaligned[];
    unsigned char* raw = unaligned + ((1024 - (ptx::smem_u32(unaligned) & 1023)) & 1023);
    unsigned char *squares = raw + STAGES * W::keys, *values = squares + W::at_values, *rows = values - kSum * W::rows_part, *state = rows - W::state;
    unsigned char* outputs = values + W::values;
    WalkBars* bars = reinterpret_cast<WalkBars*>(squares + W::squares);
    volatile uint32_t* abort_flag = &bars->abort;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int v0 = (int)(blockIdx.x % across) * NV, bh = blockIdx.x / across, h = bh % a.H, b = bh / a.H, hk = h / a.share;
    if (tid == 0) {
        bars->abort = 0;
        ptx::mbar_init(&bars->keys[0], 1), ptx::mbar_init(&bars->keys[1], 1), ptx::mbar_init(&bars->squares, 1);
        for (int i = 0; i < 3; ++i) ptx::mbar_init(&bars->done[i], 1);
        ptx::mbar_init(&bars->settled, 1);
        ptx::fence_mbar_init();
    }
    if (warp == kWorkers / 32) {
        ptx::tmem_alloc(&bars->tmem, W::cols);
        ptx::tmem_relinquish();
    }
    ptx::tc_fence_before_sync();
    __syncthreads();
    ptx::tc_fence_after_sync();
    const uint32_t tmem = bars->tmem;
    ptx::grid_dep_wait();
    const int len = sequence_length(a.lengths, b, a.L), pieces = (len + kPiece - 1) / kPiece;
    const size_t unit0 = (size_t)bh * a.pieces;

    int keys_copied = 0, squares_copied = 0;                   // pieces whose copies have been started
    if (warp == kWorkers / 32) {
        const uint32_t elected = ptx::elect_one();
        const unsigned char* key_tiles = a.keys + ((size_t)b * a.Hk + hk) * a.pieces * W::keys;
        auto load_keys = [&](int s) {                          // the s-th piece from the end
            if (s >= pieces) return;
            ++keys_copied;
            if (!elected) return;
            uint64_t* bar = &bars->keys[STAGES == 2 ? s & 1 : 0];
            ptx::mbar_arrive_expect_tx(bar, W::keys);
            ptx::bulk_g2s(raw + (STAGES == 2 ? s & 1 : 0) * W::keys, key_tiles + (size_t)(pieces - 1 - s) * W::keys, W::keys, bar);
        };
        auto load_squares = [&](int s) {
            if (s >= pieces) return;
            ++squares_copied;
            if (!elected) return;
            ptx::mbar_arrive_expect_tx(&bars->squares, W::squares);
            ptx::bulk_g2s(squares, a.prepared + (unit0 + pieces - 1 - s) * kPrepared, W::squares, &bars->squares);
        };
        const uint32_t s_squares = ptx::smem_u32(squares), s_state = ptx::smem_u32(state), s_rows = ptx::smem_u32(rows);
        load_keys(0), load_squares(0);
        if (STAGES == 2) load_keys(1);
        bool alive = true;
        for (int s = 0; s < pieces; ++s) {
            const uint32_t keys = ptx::smem_u32(raw) + (STAGES == 2 ? s & 1 : 0) * W::keys;
            alive = alive && ptx::mbar_wait_bounded_warp(&bars->keys[STAGES == 2 ? s & 1 : 0], (STAGES == 2 ? s >> 1 : s) & 1, abort_flag, a.max_polls);
            __syncthreads();                                   // dS is there
            ptx::tc_fence_after_sync();
            if (alive) {
                multiply_digits<NV, false, true>(tmem, IN, KD / 16, elected,
                                                 [&](int p, int k) { return rows_as_m(keys + p * W::key_part + (k >> 2) * W::HALF + (k & 3) * 32); },
                                                 [&](int k) { return rows_as_k<NV>(s_state + k * 16 * NV * 2, W::state_part); });
                ptx::mma_commit(&bars->done[0], elected);
                if (STAGES == 2 && s > 0) load_keys(s + 1);
            }
            alive = alive && ptx::mbar_wait_bounded_warp(&bars->squares, s & 1, abort_flag, a.max_polls);
            __syncthreads();                                   // beta X and scale dO are there, dO has been read
            ptx::tc_fence_after_sync();
            if (alive) {                                       // (64 rows; the other 64 of the result are of whatever lies behind, and not read)
                multiply_digits<NV, false, true>(tmem + 3 * NV, kSum, 2 * kPiece / 16, elected,
                                                 [&](int p, int k) { return rows_as_m(s_squares + p * W::square_part + (k >> 2) * (W::square_part / 2) + (k & 3) * 32); },
                                                 [&](int k) { return rows_as_k<NV>(s_rows + k * 16 * NV * 2, W::rows_part); });
                ptx::mma_commit(&bars->done[1], elected);
            }
            __syncthreads();                                   // -e^G dV and scale e^G dO are there, in their place
            ptx::tc_fence_after_sync();
            if (alive) {
                multiply_digits<NV, true, true>(tmem, IN, 2 * kPiece / 16, elected, [&](int p, int k) { return columns_as_m(keys + p * W::key_part + k * 16 * 128, W::HALF); },
                                                [&](int k) { return rows_as_k<NV>(s_rows + k * 16 * NV * 2, W::rows_part); });
                ptx::mma_commit(&bars->done[2], elected);
                load_squares(s + 1);
                if (STAGES == 1) {
                    alive = ptx::mbar_wait_bounded_warp(&bars->done[2], s & 1, abort_flag, a.max_polls);
                    if (alive) load_keys(s + 1);
                }
            }
        }
    } else if (warp < kWorkers / 32) {
        const int quarter = warp & 3, row = quarter * 32 + lane, col0 = (warp >> 2) * C, token = row & (kPiece - 1), v = v0 + col0;
        const bool is_key = row < kPiece;                      // a token of K (its E and dV), or of Q (its dO); and row `row` of dS
        const uint32_t at = tmem + ((uint32_t)quarter << 21) + col0;
        const int there = a.V - v, saved = a.VP - v;
        float S[C], X[C], y[C];
        const size_t state0 = ((size_t)bh * a.K + row) * a.V + v;
#pragma unroll
        for (int j = 0; j < C; ++j) S[j] = a.dstate_out && row < a.K && j < there ? a.dstate_out[state0 + j] : 0.f;
        const float* factors = reinterpret_cast<const float*>(squares + kSquares);
        SavedRow<C> update;                                    // E
        auto fetch = [&](int i) {
            if (i >= 0 && is_key) update.load(a.updates + quad_at(unit0 + i, a.VP, kPiece, v, token), kPiece, saved);
        };
        auto put_state = [&](int i) {                          // dS behind piece i
            if (row < KD) {
                put_row<NV, C>(state, W::state_part, row, col0, S);
                save_row<C>(a.dstates + quad_at(unit0 + i, a.VP, KD, v, row), KD, saved, S);
            }
            ptx::fence_proxy_async_smem();
        };
        if (pieces > 0) put_state(pieces - 1);
        fetch(pieces - 1);
        for (int i = pieces - 1; i >= 0; --i) {
            const uint32_t parity = (pieces - 1 - i) & 1;
            ptx::tc_fence_before_sync();
            __syncthreads();
            ptx::mbar_wait_bounded(&bars->squares, parity, abort_flag, a.max_polls);
            const float eg = factors[token], ed = factors[kPiece + token], beta = factors[2 * kPiece + token], whole = factors[kPiece - 1];
            if (!is_key) {
                Tile<T, NV>::get(values, token, col0, y);
                scaled(y, a.scale, y);
                put_row<NV, C>(rows, W::rows_part, row, col0, y);
            }
            // D1: K dS
            ptx::mbar_wait_bounded(&bars->done[0], parity, abort_flag, a.max_polls);
            ptx::tc_fence_after_sync();
            if (is_key) {
                tmem_digits<C>(at, NV, X);
                scaled(X, ed, X);
                scaled(y, beta, X);
                put_row<NV, C>(rows, W::rows_part, row, col0, y);
            }
            ptx::fence_proxy_async_smem();
            ptx::tc_fence_before_sync();
            __syncthreads();
            // D2: W - X
            ptx::mbar_wait_bounded(&bars->done[1], parity, abort_flag, a.max_polls);
            ptx::tc_fence_after_sync();
            float sum = 0.f;
            if (is_key) {
                tmem_digits<C>(at + 3 * NV, NV, y);
                add_scaled(y, 1.f, X);
#pragma unroll
                for (int j = 0; j < C; ++j) sum = fmaf(y[j], update.q[j / 4].e[j % 4], sum);
                scaled(X, beta, y);
                scaled(y, -eg, X);
            } else {
                scaled(y, eg, y);
            }
            put_row<NV, C>(rows, W::rows_part, row, col0, y);
            ptx::fence_proxy_async_smem();
            ptx::tc_fence_before_sync();
            __syncthreads();
            if (is_key) {
                const size_t unit = unit0 + i;
                save_row<C>(a.dupdates + quad_at(unit, a.VP, kPiece, v, token), kPiece, saved, X);
                Tile<T, NV>::put(outputs, token, col0, X);
                if (saved > 0) {                               // (a sum over 32 columns stands for two of 16)
                    float* part = a.dbeta_parts + (unit * (a.VP / 16) + v / 16) * kPiece + token;
                    part[0] = sum;
                    if (C == 32 && saved > 16) part[kPiece] = 0.f;
                }
            }
            fetch(i - 1);
            // D3: dS <- e^G_63 dS + ..
            ptx::mbar_wait_bounded(&bars->done[2], parity, abort_flag, a.max_polls);
            ptx::tc_fence_after_sync();
            tmem_digits<C>(at, NV, y);
            add_scaled(y, whole, S);
#pragma unroll
            for (int j = 0; j < C; ++j) S[j] = y[j];
            if (i > 0) put_state(i - 1);
        }
        if (a.dstate_in && row < a.K) {
#pragma unroll
            for (int j = 0; j < C; ++j)
                if (j < there) a.dstate_in[state0 + j] = S[j];
        }
        zero_rows(static_cast<T*>(a.dv) + (long long)b * a.L * a.lddv + (long long)h * a.V + v0, a.lddv, len, a.L, min(NV, a.V - v0), tid, kWorkers);
    } else {
        const long long row0 = (long long)b * a.L, first = (long long)h * a.V + v0;
        move_values<T, NV, WIDE, true>(static_cast<const T*>(a.dout) + row0 * a.lddo + first, a.lddo, static_cast<T*>(a.dv) + row0 * a.lddv + first, a.lddv, values, outputs, len,
                                       pieces, a.V - v0, tid - kPieceThreads);
        return;
    }
    ptx::tc_fence_before_sync();
    __syncthreads();
    if (warp == kWorkers / 32) {
        ptx::tc_fence_after_sync();
        if (*abort_flag) {
            settle(&bars->keys[0], STAGES == 2 ? (keys_copied + 1) / 2 : keys_copied), settle(&bars->keys[1], STAGES == 2 ? keys_copied / 2 : 0);
            settle(&bars->squares, squares_copied);
            settle_products(&bars->settled, ptx::elect_one());
            if (lane == 0) atomicExch(a.timeout, 1u);
        }
        ptx::tmem_dealloc(tmem, W::cols);
    }
}

// One block for one piece of one value head: products over V in blocks of 32 columns, two in turn (while one's products run, the threads split the next one's numbers, and
// those of the one after it are under way), then products over tokens.
//   D1 [dV; dO] S^T,   D2 [dV; dO] E^T,   D3 E dS^T (64 rows),   then of D2 [y; p],
//   D4 [y; p] K,   D5 [y; p]^T [K; Q] (64 rows likewise).
// In the last step a thread has a quarter of a row of a and c (keys) or of dq (queries).  What bounds it: the MMAs of 128 rows, of which those of keys alone are half, six for
// every pair of numbers in three parts, are a half of its time; the rest is one thing after the other, since tensor memory has room for one piece.
template <typename T, int KD>
struct Piecewise {
    static constexpr int IN = Parts<T>::in, NB = 32, HALF = 2 * kPiece * 128, WORKERS = 512, THREADS = WORKERS + 32;
    static constexpr int rows_part = 2 * kPiece * NB * 2, half = kPiece * NB * 2, state_part = KD * NB * 2;
    // E lies as [zeros, E0, E1, zeros, E2], 64 rows each
    static constexpr int at_e = kSum * rows_part, at_s = at_e + 5 * half, at_ds = at_s + kSum * state_part, block = at_ds + kSum * state_part;
    static constexpr int keys = IN * (KD / 64) * HALF, key_part = (KD / 64) * HALF, square_part = 2 * kPiece * 128;
    // over V: two blocks; over tokens: keys and queries, [y; p], in whose place the results are collected; (the 64 rows more reach as far as one tile
    // behind the last one)
    static constexpr int over_v = 2 * block, over_tokens = keys + kSum * square_part + square_part, results = keys + 2 * kPiece * KD * 4;
    static constexpr int at_small3 = over_tokens > results ? over_tokens : results, behind = at_small3 + kPiece * KD * 4;
    static constexpr int smem = (over_v > behind ? over_v : behind) + 1024;       // (1024 to the first boundary of the swizzle)
    static_assert(smem + 4096 <= 232448, "a piece does not fit");                 // (4096: what else a block keeps)
    // Columns of tensor memory.  Products of first parts have a sum of their own: an MMA cuts what it adds off at the last digit of its sum, of small terms nearly all
    // (dq of 128 and 256 columns of V 0.8e-6 and 1.6e-6 off with one sum, 0.3e-6 so).  The small sums of D1 and D2 lie where D4 and D5 come later; those of D3
    // are its rows 64 and on, of E1 beside E0 and of E0 and E2 behind 64 rows of zeros, and are handed over through shared memory.
    static constexpr uint32_t d1 = 0, d3 = KD, d4 = 2 * KD, d2 = 3 * KD, d5 = 3 * KD, small1 = d4, small2 = d2 + kPiece, cols = 512;
};
struct PieceBars {
    uint64_t done[2], keys, last, settled;
    uint32_t tmem, abort;
    alignas(16) float factors[kFactors * kPiece];              // (read in fours)
    float dots[8][kPiece], inner[16], sums[2][16];
};
// A piece of a head, as one block finds it.
struct Place {
    int b, h, live, there;                                     // tokens of the sequence, rows of the tensors
    long long row0;
    size_t unit;
    __device__ Place(const DeltaArgs& a, unsigned id)
    {
        const int piece = id % a.pieces, bh = id / a.pieces;
        h = bh % a.H, b = bh / a.H, unit = id, row0 = (long long)b * a.L + (long long)piece * kPiece;
        live = min(sequence_length(a.lengths, b, a.L) - piece * kPiece, kPiece), there = min(a.L - piece * kPiece, kPiece);
    }
};
// What a thread has under way of 32 columns of V: quads.  Of what the passes kept two lanes have the two of a unit of 16 bytes and the next two the next row, so that
// half a warp reads whole lines and fills every bank once; of dO eight threads have a row.
template <typename T, int KD, bool WIDE>
struct Quads {
    static constexpr int ACROSS = Piecewise<T, KD>::WORKERS / KD, N = 8 / ACROSS;        // quads of a row of S at once, of a thread
    static __device__ __forceinline__ int quad(int tid, int rows) { return (tid & 1) + 2 * (tid / (2 * rows)); }
    static __device__ __forceinline__ int row(int tid, int rows) { return (tid >> 1) % rows; }
    SavedRow<4> s[N], ds[N], dv, e;
    Row<T, 4> dout;
    __device__ __forceinline__ void fetch(const DeltaArgs& a, const Place& at, int v0, int tid)
    {
        const int k = row(tid, KD), q = quad(tid, KD), t = row(tid, kPiece), p = quad(tid, kPiece), r = tid >> 3, c = (tid & 7) * 4;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int v = v0 + 4 * (q + ACROSS * i);
            s[i].load(a.states + quad_at(at.unit, a.VP, KD, v, k), KD, a.VP - v), ds[i].load(a.dstates + quad_at(at.unit, a.VP, KD, v, k), KD, a.VP - v);
        }
        const int v = v0 + 4 * p;
        dv.load(a.dupdates + quad_at(at.unit, a.VP, kPiece, v, t), kPiece, a.VP - v), e.load(a.updates + quad_at(at.unit, a.VP, kPiece, v, t), kPiece, a.VP - v);
        dout.template load<WIDE>(static_cast<const T*>(a.dout) + (at.row0 + r) * a.lddo + (long long)at.h * a.V + v0 + c, r < at.live ? a.V - v0 - c : 0);
    }
};
// Their places in a block's tiles.
template <typename T, int KD>
struct QuadPlaces {
    using W = Piecewise<T, KD>;
    using Q = Quads<T, KD, true>;
    int s[Q::N], row, dout;
    __device__ explicit QuadPlaces(int tid)
    {
#pragma unroll
        for (int i = 0; i < Q::N; ++i) s[i] = four_at<W::NB>(Q::row(tid, KD), 4 * (Q::quad(tid, KD) + Q::ACROSS * i));
        row = four_at<W::NB>(Q::row(tid, kPiece), 4 * Q::quad(tid, kPiece)), dout = four_at<W::NB>(kPiece + (tid >> 3), (tid & 7) * 4);
    }
    template <bool WIDE>
    __device__ __forceinline__ void put(unsigned char* at, const Quads<T, KD, WIDE>& x, float& inner) const
    {
#pragma unroll
        for (int i = 0; i < Q::N; ++i) {
            put_four<kSum>(at + W::at_s + s[i], W::state_part, x.s[i].q[0].e);
            put_four<kSum>(at + W::at_ds + s[i], W::state_part, x.ds[i].q[0].e);
#pragma unroll
            for (int n = 0; n < 4; ++n) inner = fmaf(x.s[i].q[0].e[n], x.ds[i].q[0].e[n], inner);
        }
        float f[4];
        x.dout.get(f);
        put_four<kSum>(at + row, W::rows_part, x.dv.q[0].e);
        uint32_t w[2][kSum];
        split<kSum>(x.e.q[0].e[0], x.e.q[0].e[1], w[0]);
        split<kSum>(x.e.q[0].e[2], x.e.q[0].e[3], w[1]);
#pragma unroll
        for (int p = 0; p < kSum; ++p) *reinterpret_cast<uint2*>(at + W::at_e + (p == 2 ? 4 : 1 + p) * W::half + row) = make_uint2(w[0][p], w[1][p]);
        put_four<W::IN>(at + dout, W::rows_part, f);
    }
};

// A block takes pieces gridDim.x apart; the next one's first numbers are under way while this one's results go out, the others come to the L2 cache meanwhile.  (A block for
// each piece: 240 us of a training step of 2048 of them, 17 us each, of which four pass between two blocks.)
template <typename T, int KD, bool WIDE>
__global__ void __launch_bounds__(Piecewise<T, KD>::THREADS, 1) delta_bwd_pieces_kernel(const DeltaArgs a, unsigned total)
{
    using W = Piecewise<T, KD>;
    constexpr int IN = W::IN, NB = W::NB;
    extern __shared__ unsigned char unaligned[];
    __shared__ PieceBars bars;
    unsigned char* raw = unaligned + ((1024 - (ptx::smem_u32(unaligned) & 1023)) & 1023);
    volatile uint32_t* abort_flag = &bars.abort;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const bool works = warp < W::WORKERS / 32, shared_key = a.dq_parts != nullptr;
    if (tid == 0) {
        bars.abort = 0;
        ptx::mbar_init(&bars.done[0], 1), ptx::mbar_init(&bars.done[1], 1), ptx::mbar_init(&bars.keys, 1), ptx::mbar_init(&bars.last, 1), ptx::mbar_init(&bars.settled, 1);
        ptx::fence_mbar_init();
    }
    if (!works) {
        ptx::tmem_alloc(&bars.tmem, W::cols);
        ptx::tmem_relinquish();
    }
    ptx::tc_fence_before_sync();
    __syncthreads();
    ptx::tc_fence_after_sync();
    const uint32_t tmem = bars.tmem, base = ptx::smem_u32(raw), keys = base, squares = base + W::keys;
    const int blocks = (a.VP + NB - 1) / NB;
    ptx::grid_dep_wait();

    // padding of all its pieces; from then on only pieces with tokens
    for (unsigned id = blockIdx.x; id < total; id += gridDim.x) {
        const Place at(a, id);
        if (at.live >= at.there) continue;
        const int first = max(at.live, 0), hk = at.h / a.share;
        for (int i = tid; i < (at.there - first) * a.K; i += W::THREADS) {
            const long long r = at.row0 + first + i / a.K;
            const int col = i % a.K;
            if (shared_key) a.dq_parts[(r * a.H + at.h) * a.K + col] = 0.f, a.dk_parts[(r * a.H + at.h) * a.K + col] = 0.f;
            else static_cast<T*>(a.dq)[r * a.lddq + (long long)hk * a.K + col] = from_float<T>(0.f), static_cast<T*>(a.dk)[r * a.lddk + (long long)hk * a.K + col] = from_float<T>(0.f);
        }
        for (int i = first + tid; i < at.there; i += W::THREADS) a.dg[(at.row0 + i) * a.lddg + at.h] = 0.f, a.dbeta[(at.row0 + i) * a.lddbeta + at.h] = 0.f;
    }
    auto following = [&](unsigned id) {
        while (id < total && Place(a, id).live <= 0) id += gridDim.x;
        return id;
    };
    // completions of done[0] and done[1] in a piece, and so far
    const int first_of = (blocks + 1) / 2, second_of = blocks / 2;
    int first_so_far = 0, second_so_far = 0, parity = 0;
    const unsigned begin = following(blockIdx.x);

    if (!works) {
        const uint32_t elected = ptx::elect_one();
        constexpr uint32_t idk = ptx::idesc_b16(128, KD, false);
        // tiles of rows of 32 numbers, K-major: 64-byte swizzle
        auto narrow = [](uint32_t at) { return rows_as_k<32>(at, 512); };
        bool alive = true;
        int copied = 0;
        for (unsigned id = begin; id < total; id = following(id + gridDim.x), parity ^= 1) {
            const Place here(a, id);
            for (int j = 0; j < blocks; ++j) {
                __syncthreads();
                ptx::tc_fence_after_sync();
                const uint32_t at = base + (j & 1) * W::block;
                auto rows = [&](int p, int k) { return narrow(at + p * W::rows_part + k * 32); };
                auto e = [&](int p, int k) { return narrow(at + W::at_e + (p == 2 ? 4 : 1 + p) * W::half + k * 32); };
                auto s = [&](int p, int k) { return narrow(at + W::at_s + p * W::state_part + k * 32); };
                auto ds = [&](int p, int k) { return narrow(at + W::at_ds + p * W::state_part + k * 32); };
                constexpr uint32_t id64 = ptx::idesc_b16(128, kPiece, false);
                multiply_first(tmem + W::d1, NB / 16, idk, elected, j > 0, rows, s);
                multiply_small(tmem + W::small1, NB / 16, idk, elected, j > 0, rows, s);
                multiply_first(tmem + W::d2, NB / 16, id64, elected, j > 0, rows, e);
                multiply_small(tmem + W::small2, NB / 16, id64, elected, j > 0, rows, e);
                // (of rows 0 to 63 and 64 on: zeros and E0 dS2, zeros and E2 dS0, zeros and E0 dS1, E1 dS1 and zeros, E0 dS0 and E1 dS0)
                auto third = [&](int half, int part, bool more) {
#pragma unroll
                    for (int k = 0; k < NB / 16; ++k) ptx::mma_b16(tmem + W::d3, narrow(at + W::at_e + half * W::half + k * 32), ds(part, k), idk, more || k > 0, elected);
                };
                third(0, 2, j > 0), third(3, 0, true), third(0, 1, true);
                third(2, 1, true), third(1, 0, true);
                ptx::mma_commit(&bars.done[j & 1], elected);
            }
            first_so_far += first_of, second_so_far += second_of;
            alive = alive && ptx::mbar_wait_bounded_warp(&bars.done[(blocks - 1) & 1], (((blocks - 1) & 1 ? second_so_far : first_so_far) - 1) & 1, abort_flag, a.max_polls);
            copied += alive;
            if (alive && elected) {                            // (the tiles over V are done with)
                ptx::mbar_arrive_expect_tx(&bars.keys, W::keys);
                ptx::bulk_g2s(raw, a.keys + (((size_t)here.b * a.Hk + here.h / a.share) * a.pieces + id % a.pieces) * W::keys, W::keys, &bars.keys);
            }
            alive = alive && ptx::mbar_wait_bounded_warp(&bars.keys, parity, abort_flag, a.max_polls);
            __syncthreads();                                   // [y; p] is there
            ptx::tc_fence_after_sync();
            if (alive) {
                auto tokens = [&](int p, int k) { return columns_as_m(keys + p * W::key_part + k * 16 * 128, W::HALF); };
                multiply(tmem + W::d4, kSum, IN, kPiece / 16, idk | ptx::kIdescBMajorMN, elected, false,
                         [&](int p, int k) { return rows_as_m(squares + p * W::square_part + k * 32); }, tokens);
                multiply(tmem + W::d5, kSum, IN, 2 * kPiece / 16, idk | ptx::kIdescBMajorMN | kIdescAMajorM, elected, false,
                         [&](int p, int k) { return columns_as_m(squares + p * W::square_part + k * 16 * 128, W::square_part); }, tokens);
                ptx::mma_commit(&bars.last, elected);
            }
            __syncthreads();                                   // (results are collected)
            __syncthreads();                                   // (and out)
        }
        ptx::tc_fence_after_sync();
        if (*abort_flag) {
            settle(&bars.keys, copied);
            settle_products(&bars.settled, elected);
            if (lane == 0) atomicExch(a.timeout, 1u);
        }
        ptx::tmem_dealloc(tmem, W::cols);
        return;
    }

    const int quarter = warp & 3, row = quarter * 32 + lane, side = warp >> 2, token = row & (kPiece - 1);
    const bool is_key = row < kPiece;
    const uint32_t lanes = tmem + ((uint32_t)quarter << 21);
    const float *eg = bars.factors, *ed = eg + kPiece, *be = eg + 2 * kPiece, *high = eg + 3 * kPiece, *low = eg + 4 * kPiece;
    const QuadPlaces<T, KD> places(tid);
    Quads<T, KD, WIDE> next;
    float factor = 0.f;
    auto fetch = [&](unsigned id) {                            // a piece's first block and factors
        if (id >= total) return;
        const Place at(a, id);
        next.fetch(a, at, 0, tid);
        factor = load_masked<float, 1>(reinterpret_cast<const float*>(a.prepared + at.unit * kPrepared + kSquares) + tid, tid < kFactors * kPiece).e[0];
    };
    auto ready = [&] {                                         // for the products
        ptx::fence_proxy_async_smem();
        ptx::tc_fence_before_sync();
        __syncthreads();
    };
    constexpr int SHARE = KD / 4;                              // columns of a thread
    // D3's small sums, [64][KD] in units of 16 bytes spread over the banks
    auto small3_at = [&](int col) { return reinterpret_cast<float4*>(raw + W::at_small3) + token * (KD / 4) + ((col >> 2) ^ (token & 7)); };
    fetch(begin);
    for (unsigned id = begin; id < total; parity ^= 1) {
        const Place here(a, id);
        const unsigned then = following(id + gridDim.x);
        float inner = 0.f;                                     // <S, dS>
        if (tid < kFactors * kPiece) bars.factors[tid] = factor;
        if (tid < 4 && then < total) {
            const size_t state = (size_t)KD * a.VP * 4, update = (size_t)kPiece * a.VP * 4;
            const char* from = tid == 0 ? reinterpret_cast<const char*>(a.states) + then * state : tid == 1 ? reinterpret_cast<const char*>(a.dstates) + then * state
                             : tid == 2 ? reinterpret_cast<const char*>(a.updates) + then * update : reinterpret_cast<const char*>(a.dupdates) + then * update;
            asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(from), "r"((unsigned)(tid < 2 ? state : update)) : "memory");
        }
        for (int j = 0; j < blocks; ++j) {
            if (j >= 2) ptx::mbar_wait_bounded(&bars.done[j & 1], ((j & 1 ? second_so_far : first_so_far) + (j >> 1) - 1) & 1, abort_flag, a.max_polls);
            places.put(raw + (j & 1) * W::block, next, inner);
            // (the rows of zeros: tiles of other products have lain there)
            if (j < 2) {
                static_assert(2 * W::half / 16 == W::WORKERS, "a unit a thread");
                const int z = tid < W::WORKERS / 2 ? tid : tid + 2 * W::WORKERS / 2;         // units of the first and of the fourth 64 rows
                *reinterpret_cast<uint4*>(raw + j * W::block + W::at_e + z * 16) = make_uint4(0u, 0u, 0u, 0u);
            }
            if (j + 1 < blocks) next.fetch(a, here, (j + 1) * NB, tid);
            ready();
        }
#pragma unroll
        for (int d = 1; d < 32; d *= 2) inner += __shfl_xor_sync(0xffffffffu, inner, d);
        if (lane == 0) bars.inner[warp] = inner;               // (while the last products run)
        if (warp == 4 || warp == 5) {                          // dbeta, a sum over the walk's columns
            const int r = (warp - 4) * 32 + lane, tiles = a.VP / 16;
            const float* from = a.dbeta_parts + here.unit * tiles * kPiece + r;
            float s = 0.f;
            for (int i = 0; i < tiles; ++i) s += from[i * kPiece];
            if (r < here.live) a.dbeta[(here.row0 + r) * a.lddbeta + here.h] = s;
        }
        first_so_far += first_of, second_so_far += second_of;
        ptx::mbar_wait_bounded(&bars.done[(blocks - 1) & 1], (((blocks - 1) & 1 ? second_so_far : first_so_far) - 1) & 1, abort_flag, a.max_polls);
        ptx::tc_fence_after_sync();
        {
            float x[16];
            {
                float y[16];
                tmem_row(lanes + W::d2 + side * 16, x);
                tmem_row(lanes + W::small2 + side * 16, y);
#pragma unroll
                for (int n = 0; n < 16; ++n) x[n] += y[n];
            }
#pragma unroll
            for (int i = 0; i < SHARE; i += 16) {
                const int col = side * SHARE + i;
                uint32_t v[16], w[16];
                ptx::tmem_ld16(lanes + W::d1 + col, v), ptx::tmem_ld16(lanes + W::small1 + col, w);
                ptx::tmem_ld_wait();
#pragma unroll
                for (int n = 0; n < 16; ++n) v[n] = __float_as_uint(__uint_as_float(v[n]) + __uint_as_float(w[n]));
                ptx::tmem_st16(lanes + W::d1 + col, v);
                if (is_key) continue;                          // (whole warps)
                float y[16];
                tmem_row(lanes + W::d3 + col, y);
#pragma unroll
                for (int u = 0; u < 4; ++u) *small3_at(col + 4 * u) = make_float4(y[4 * u], y[4 * u + 1], y[4 * u + 2], y[4 * u + 3]);
            }
            ptx::tmem_st_wait();
            const float hi = high[token], lo = low[token], by = is_key ? -1.f : a.scale;
            const int last = is_key ? token - 1 : token;       // (keys: j < i, queries: j <= i)
#pragma unroll
            for (int j = 0; j < 16; j += 4) {
                const int other = side * 16 + j;
                const float4 h4 = *reinterpret_cast<const float4*>(high + other), l4 = *reinterpret_cast<const float4*>(low + other),
                             b4 = *reinterpret_cast<const float4*>(be + other);
                const float hs[4] = {h4.x, h4.y, h4.z, h4.w}, ls[4] = {l4.x, l4.y, l4.z, l4.w}, bs[4] = {b4.x, b4.y, b4.z, b4.w};
#pragma unroll
                for (int n = 0; n < 4; ++n) {
                    const float d = ex2(((hi - hs[n]) + (lo - ls[n])) * kLog2e) * bs[n] * by;
                    x[j + n] = other + n <= last ? d * x[j + n] : 0.f;
                }
            }
            put_row<64, 16>(raw + W::keys, W::square_part, row, side * 16, x);
        }
        ready();
        ptx::mbar_wait_bounded(&bars.keys, parity, abort_flag, a.max_polls);
        ptx::mbar_wait_bounded(&bars.last, parity, abort_flag, a.max_polls);
        ptx::tc_fence_after_sync();
        // <S after, dS> = e^G_63 <S, dS> + sum over tokens of k . (e^(G_63 - G) beta E dS^T);
        // <S, dS before> = e^G_63 <S, dS> + sum of q . (scale e^G dO S^T) - k . (e^G dV S^T)
        float after = 0.f, before = 0.f, dot = 0.f;
        const float x1 = is_key ? -eg[token] : a.scale * eg[token], x3 = ed[token] * be[token];
        unsigned char* collected = raw + W::keys;              // [128 rows][KD] of what goes out, fp32 for shared keys
        const int bytes = shared_key ? 4 : (int)sizeof(T), units = KD * bytes / 16;
        // unit u of row r, spread over the banks
        auto collect_at = [&](int r, int u) { return (r * units + (u ^ (r & 7))) * 16; };
#pragma unroll
        for (int i = 0; i < SHARE; i += 16) {
            const int col = side * SHARE + i;
            float x[16], z[16];
            uint32_t v[16], w[16];
            ptx::tmem_ld16(lanes + W::d1 + col, v), ptx::tmem_ld16(lanes + W::d4 + col, w);
#pragma unroll
            for (int j = 0; j < 16; ++j) z[j] = 0.f;
#pragma unroll
            for (int p = IN - 1; p >= 0; --p)
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    float f[8];
                    unpack(*reinterpret_cast<const Pack<bf16, 8>*>(raw + unit_at<64>(p * W::key_part + (col >> 6) * W::HALF, row, ((col & 63) >> 3) + u)), f);
#pragma unroll
                    for (int j = 0; j < 8; ++j) z[8 * u + j] += f[j];
                }
            ptx::tmem_ld_wait();
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                before = fmaf(z[j], __uint_as_float(v[j]), before), dot = fmaf(z[j], __uint_as_float(w[j]), dot);
                x[j] = fmaf(x1, __uint_as_float(v[j]), __uint_as_float(w[j]));
            }
            if (is_key) {
                ptx::tmem_ld16(lanes + W::d3 + col, v), ptx::tmem_ld16(lanes + W::d5 + col, w);
                float rest[16];
#pragma unroll
                for (int u = 0; u < 4; ++u) *reinterpret_cast<float4*>(rest + 4 * u) = *small3_at(col + 4 * u);
                ptx::tmem_ld_wait();
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    float y = x3 * (__uint_as_float(v[j]) + rest[j]);
                    after = fmaf(z[j], y, after);
                    y += __uint_as_float(w[j]), dot = fmaf(-z[j], y, dot);
                    x[j] += y;
                }
            }
            if (shared_key) {
#pragma unroll
                for (int u = 0; u < 4; ++u) *reinterpret_cast<float4*>(collected + collect_at(row, col / 4 + u)) = make_float4(x[4 * u], x[4 * u + 1], x[4 * u + 2], x[4 * u + 3]);
            } else {
                constexpr int PER = 16 / (int)sizeof(T);
#pragma unroll
                for (int u = 0; u < 16 / PER; ++u) {
                    float f[PER];
#pragma unroll
                    for (int j = 0; j < PER; ++j) f[j] = x[u * PER + j];
                    store_pack<T, PER>(reinterpret_cast<T*>(collected + collect_at(row, col / PER + u)), pack<T, PER>(f));
                }
            }
        }
        before *= x1;
        bars.dots[side * 2 + (is_key ? 0 : 1)][token] = dot + before;
        // both are summed over the warp at once, one in either half of the lanes
        const bool upper = lane >= 16;
        float both_sums = (upper ? after : before) + __shfl_xor_sync(0xffffffffu, upper ? before : after, 16);
#pragma unroll
        for (int d = 1; d < 16; d *= 2) both_sums += __shfl_xor_sync(0xffffffffu, both_sums, d);
        if ((lane & 15) == 0) bars.sums[lane >> 4][warp] = both_sums;
        id = then;
        fetch(id);
        ptx::tc_fence_before_sync();
        __syncthreads();
        // rows of dk, then of dq, whole lines at a time
        const int hk = here.h / a.share;
        T *dq = static_cast<T*>(a.dq) + here.row0 * a.lddq + (long long)hk * a.K, *dk = static_cast<T*>(a.dk) + here.row0 * a.lddk + (long long)hk * a.K;
        const long long part0 = (here.row0 * a.H + here.h) * a.K;
        if (WIDE) {
            for (int i = tid; i < 2 * kPiece * units; i += W::WORKERS) {
                const int r = i / units, u = i % units, t = r & (kPiece - 1), col = u * 16 / bytes;
                if (t >= here.live || col >= a.K) continue;
                const uint4 v = *reinterpret_cast<const uint4*>(collected + collect_at(r, u));
                if (shared_key) *reinterpret_cast<uint4*>((r < kPiece ? a.dk_parts : a.dq_parts) + part0 + (long long)t * a.H * a.K + col) = v;
                else *reinterpret_cast<uint4*>(r < kPiece ? dk + t * a.lddk + col : dq + t * a.lddq + col) = v;
            }
        } else {
            for (int i = tid; i < 2 * kPiece * KD; i += W::WORKERS) {
                const int r = i / KD, col = i % KD, t = r & (kPiece - 1);
                if (t >= here.live || col >= a.K) continue;
                const unsigned char* from = collected + collect_at(r, col * bytes / 16) + col * bytes % 16;
                if (shared_key) (r < kPiece ? a.dk_parts : a.dq_parts)[part0 + (long long)t * a.H * a.K + col] = *reinterpret_cast<const float*>(from);
                else *(r < kPiece ? dk + t * a.lddk + col : dq + t * a.lddq + col) = *reinterpret_cast<const T*>(from);
            }
        }
        if (warp == 0) {                                       // sums from the last token back and from the first on, two tokens a lane
            float front = fmaf(eg[kPiece - 1], bars.inner[lane & 15], bars.sums[lane >> 4][lane & 15]);
#pragma unroll
            for (int d = 1; d < 16; d *= 2) front += __shfl_xor_sync(0xffffffffu, front, d);
            const float last = __shfl_sync(0xffffffffu, front, 31);
            front = __shfl_sync(0xffffffffu, front, 0);
            auto sum = [&](int i) {
                float s = 0.f;
#pragma unroll
                for (int j = 0; j < 8; ++j) s += bars.dots[j][i];
                return s;
            };
            const float g1 = sum(63 - 2 * lane), g0 = sum(62 - 2 * lane);
            float s = g0 + g1, p = s;                          // with those behind them, with those before them
#pragma unroll
            for (int d = 1; d < 32; d *= 2) {
                const float y = __shfl_up_sync(0xffffffffu, s, d), z = __shfl_down_sync(0xffffffffu, p, d);
                if (lane >= d) s += y;
                if (lane + d < 32) p += z;
            }
            p = __shfl_down_sync(0xffffffffu, p, 1);
            if (lane == 31) p = 0.f;
            const int first = 62 - 2 * lane;
            if (first < here.live) a.dg[(here.row0 + first) * a.lddg + here.h] = 2 * first < here.live ? front - p : s + last;
            if (first + 1 < here.live) a.dg[(here.row0 + first + 1) * a.lddg + here.h] = 2 * first + 2 < here.live ? front - (p + g0) : (s - g0) + last;
        }
        __syncthreads();
    }
}

// Gradients of a key head from those of its value heads.
template <typename T>
__global__ void __launch_bounds__(256) delta_bwd_shared_kernel(const DeltaArgs a)
{
    ptx::grid_dep_wait();
    const long long n = (long long)a.B * a.L * a.Hk * a.K;
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n; i += (long long)gridDim.x * 256) {
        const int col = (int)(i % a.K), hk = (int)(i / a.K % a.Hk);
        const long long row = i / ((long long)a.K * a.Hk), at = (row * a.H + (long long)hk * a.share) * a.K + col;
        float q = 0.f, k = 0.f;
        for (int r = 0; r < a.share; ++r) q += a.dq_parts[at + (long long)r * a.K], k += a.dk_parts[at + (long long)r * a.K];
        static_cast<T*>(a.dq)[row * a.lddq + (long long)hk * a.K + col] = from_float<T>(q);
        static_cast<T*>(a.dk)[row * a.lddk + (long long)hk * a.K + col] = from_float<T>(k);
    }
}

template <typename T, int KD, int NV, bool WIDE>
conv2d_status_t backward_walk(const DeltaArgs& a, cudaStream_t stream)
{
    using W = Walk<T, KD, NV, 2 * kPiece>;
    static SmemLimit limit;
    const int across = (int)ceil_div_u(a.V, NV);
    if (raise_smem_limit((const void*)delta_bwd_walk_kernel<T, KD, NV, WIDE>, W::smem, limit) != cudaSuccess) return CONV2D_ERR_CUDA;
    if (launch_pdl(delta_bwd_walk_kernel<T, KD, NV, WIDE>, dim3((unsigned)(a.B * a.H) * across), dim3(kWalkThreads), W::smem, stream, a, across) != cudaSuccess)
        return CONV2D_ERR_CUDA;
    count_launch();
    return CONV2D_OK;
}

template <typename T, int KD, bool WIDE>
conv2d_status_t backward_pieces(const DeltaArgs& a, cudaStream_t stream)
{
    using W = Piecewise<T, KD>;
    static SmemLimit limit;
    if (raise_smem_limit((const void*)delta_bwd_pieces_kernel<T, KD, WIDE>, W::smem, limit) != cudaSuccess) return CONV2D_ERR_CUDA;
    const unsigned total = (unsigned)(a.B * a.H) * (unsigned)a.pieces, most = (unsigned)sm_count();
    if (launch_pdl(delta_bwd_pieces_kernel<T, KD, WIDE>, dim3(total < most ? total : most), dim3(W::THREADS), W::smem, stream, a, total) != cudaSuccess)
        return CONV2D_ERR_CUDA;
    count_launch();
    return CONV2D_OK;
}

template <typename T, int KD>
conv2d_status_t backward_wide(const DeltaArgs& a, cudaStream_t stream)
{
    const int per = 16 / (int)sizeof(T);
    const bool wide_v = a.V % per == 0 && rows_aligned(a.dout, a.lddo, sizeof(T), 16) && rows_aligned(a.dv, a.lddv, sizeof(T), 16);
    const bool wide = wide_v && a.K % 8 == 0 && rows_aligned(a.q, a.ldq, sizeof(T), 16) && rows_aligned(a.k, a.ldk, sizeof(T), 16) &&
                      rows_aligned(a.dq, a.lddq, sizeof(T), 16) && rows_aligned(a.dk, a.lddk, sizeof(T), 16);
    conv2d_status_t st = CONV2D_ERR_UNSUPPORTED;
    if constexpr (sizeof(T) == 2 || KD == 64) {
        if (delta_columns<T, KD, 2 * kPiece>(a, wide_v) == 64) st = backward_walk<T, KD, 64, true>(a, stream);
    }
    if (st == CONV2D_ERR_UNSUPPORTED) st = wide_v ? backward_walk<T, KD, 32, true>(a, stream) : backward_walk<T, KD, 32, false>(a, stream);
    if (st != CONV2D_OK) return st;
    return wide ? backward_pieces<T, KD, true>(a, stream) : backward_pieces<T, KD, false>(a, stream);
}

template <typename T>
conv2d_status_t backward_typed(const DeltaArgs& a, cudaStream_t stream)
{
    const conv2d_status_t st = a.K <= 64 ? backward_wide<T, 64>(a, stream) : backward_wide<T, 128>(a, stream);
    if (st != CONV2D_OK || a.share == 1) return st;
    const long long blocks = ((long long)a.B * a.L * a.Hk * a.K + 255) / 256, most = 16LL * sm_count();
    if (launch_pdl(delta_bwd_shared_kernel<T>, dim3((unsigned)(blocks < most ? blocks : most)), dim3(256), 0, stream, a) != cudaSuccess) return CONV2D_ERR_CUDA;
    count_launch();
    return CONV2D_OK;
}

size_t up16(size_t n) { return (n + 15) / 16 * 16; }
size_t dbeta_bytes(const DeltaLayout& l) { return l.units * (l.VP / 16) * kPiece * 4; }
size_t shared_bytes(const DeltaLayout& l) { return l.H > l.Hk ? up16((size_t)l.B * l.L * l.H * l.K * 4) : 0; }

}  // namespace

size_t delta_bwd_workspace_bytes(const DeltaLayout& l) { return l.saved_bytes() + l.keys_bytes() + dbeta_bytes(l) + 2 * shared_bytes(l); }

conv2d_status_t launch_delta_bwd(DeltaArgs a, conv2d_operand_t type, const void* states, void* workspace, cudaStream_t stream)
{
    const DeltaLayout l(a.B, a.L, a.Hk, a.H, a.K, a.V, type);
    a.share = a.H / a.Hk, a.pieces = l.pieces, a.VP = l.VP;
    if (device_timeout_word(&a.timeout) != cudaSuccess) return CONV2D_ERR_CUDA;
    a.max_polls = (unsigned)env_int("CONV2D_B200_DELTA_MAX_POLLS", 1 << 22);
    unsigned char* kept = const_cast<unsigned char*>(static_cast<const unsigned char*>(states));      // (only read)
    a.prepared = kept;
    a.states = reinterpret_cast<float*>(kept + l.prepared_bytes());
    a.updates = reinterpret_cast<float*>(kept + l.prepared_bytes() + l.units * l.state());
    unsigned char* at = static_cast<unsigned char*>(workspace);
    a.dstates = reinterpret_cast<float*>(at), at += l.units * l.state();
    a.dupdates = reinterpret_cast<float*>(at), at += l.units * l.update();
    a.keys = at, at += l.keys_bytes();
    a.dbeta_parts = reinterpret_cast<float*>(at), at += dbeta_bytes(l);
    if (a.share > 1) a.dq_parts = reinterpret_cast<float*>(at), a.dk_parts = reinterpret_cast<float*>(at + shared_bytes(l));
    const conv2d_status_t st = launch_delta_prepare(a, type, false, stream);
    if (st != CONV2D_OK) return st;
    if (type == CONV2D_OPERAND_BF16) return backward_typed<bf16>(a, stream);
    if (type == CONV2D_OPERAND_FP16) return backward_typed<fp16>(a, stream);
    return backward_typed<float>(a, stream);
}

}  // namespace conv2d_b200
