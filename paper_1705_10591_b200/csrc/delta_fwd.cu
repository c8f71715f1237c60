// Gated delta rule, forward.
#include "delta_walk.cuh"

namespace conv2d_b200 {
namespace {

template <typename T, int KD, int NV, bool WIDE>
__global__ void __launch_bounds__(kWalkThreads, 1) delta_fwd_kernel(const DeltaArgs a, int across)
{
    using W = Walk<T, KD, NV, kPiece>;
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
        auto load_keys = [&](int i) {
            if (i >= pieces) return;
            ++keys_copied;
            if (!elected) return;
            uint64_t* bar = &bars->keys[STAGES == 2 ? i & 1 : 0];
            ptx::mbar_arrive_expect_tx(bar, W::keys);
            ptx::bulk_g2s(raw + (STAGES == 2 ? i & 1 : 0) * W::keys, key_tiles + (size_t)i * W::keys, W::keys, bar);
        };
        auto load_squares = [&](int i) {
            if (i >= pieces) return;
            ++squares_copied;
            if (!elected) return;
            ptx::mbar_arrive_expect_tx(&bars->squares, W::squares);
            ptx::bulk_g2s(squares, a.prepared + (unit0 + i) * kPrepared, W::squares, &bars->squares);
        };
        const uint32_t s_squares = ptx::smem_u32(squares), s_state = ptx::smem_u32(state), s_rows = ptx::smem_u32(rows);
        load_keys(0), load_squares(0);
        if (STAGES == 2) load_keys(1);
        bool alive = true;
        for (int i = 0; i < pieces; ++i) {
            const uint32_t keys = ptx::smem_u32(raw) + (STAGES == 2 ? i & 1 : 0) * W::keys;
            alive = alive && ptx::mbar_wait_bounded_warp(&bars->keys[STAGES == 2 ? i & 1 : 0], (STAGES == 2 ? i >> 1 : i) & 1, abort_flag, a.max_polls);
            __syncthreads();                                   // S is there
            ptx::tc_fence_after_sync();
            if (alive) {
                multiply_digits<NV, false, true>(tmem, IN, KD / 16, elected,
                                                 [&](int p, int k) { return rows_as_m(keys + p * W::key_part + (k >> 2) * W::HALF + (k & 3) * 32); },
                                                 [&](int k) { return rows_as_k<NV>(s_state + k * 16 * NV * 2, W::state_part); });
                ptx::mma_commit(&bars->done[0], elected);
                // (everything of the piece before is done with)
                if (STAGES == 2 && i > 0) load_keys(i + 1);
            }
            alive = alive && ptx::mbar_wait_bounded_warp(&bars->squares, i & 1, abort_flag, a.max_polls);
            __syncthreads();                                   // beta R is there, the values have been read
            ptx::tc_fence_after_sync();
            if (alive) {
                multiply_digits<NV, true, true>(tmem + 3 * NV, kSum, kPiece / 16, elected,
                                                [&](int p, int k) { return columns_as_m(s_squares + p * W::square_part + k * 16 * 128, W::square_part / 2); },
                                                [&](int k) { return rows_as_k<NV>(s_rows + k * 16 * NV * 2, W::rows_part); });
                ptx::mma_commit(&bars->done[1], elected);
            }
            __syncthreads();                                   // what updates S is there, in the place of beta R
            ptx::tc_fence_after_sync();
            if (alive) {
                multiply_digits<NV, true, true>(tmem, IN, kPiece / 16, elected, [&](int p, int k) { return columns_as_m(keys + p * W::key_part + k * 16 * 128, W::HALF); },
                                                [&](int k) { return rows_as_k<NV>(s_rows + k * 16 * NV * 2, W::rows_part); });
                ptx::mma_commit(&bars->done[2], elected);
                load_squares(i + 1);
                if (STAGES == 1) {
                    alive = ptx::mbar_wait_bounded_warp(&bars->done[2], i & 1, abort_flag, a.max_polls);
                    if (alive) load_keys(i + 1);
                }
            }
        }
    } else if (warp < kWorkers / 32) {
        const int quarter = warp & 3, row = quarter * 32 + lane, col0 = (warp >> 2) * C, token = row & (kPiece - 1), v = v0 + col0;
        const bool is_key = row < kPiece;                      // a token of K, or of Q; and row `row` of S
        const uint32_t at = tmem + ((uint32_t)quarter << 21) + col0;
        const int there = a.V - v, saved = a.VP - v;           // columns of this thread that there are
        float S[C], X[C];
        const size_t state0 = ((size_t)bh * a.K + row) * a.V + v;
#pragma unroll
        for (int j = 0; j < C; ++j) S[j] = a.state_in && row < a.K && j < there ? a.state_in[state0 + j] : 0.f;
        const float* factors = reinterpret_cast<const float*>(squares + kSquares);
        auto put_state = [&](int i) {                          // S before piece i, for its product and for the backward pass
            if (row < KD) {
                put_row<NV, C>(state, W::state_part, row, col0, S);
                if (a.states) save_row<C>(a.states + quad_at(unit0 + i, a.VP, KD, v, row), KD, saved, S);
            }
            ptx::fence_proxy_async_smem();
        };
        if (pieces > 0) put_state(0);
        for (int i = 0; i < pieces; ++i) {
            const uint32_t parity = i & 1;
            ptx::tc_fence_before_sync();
            __syncthreads();
            // D1: of keys R = v - e^G k S, of queries e^G q S
            ptx::mbar_wait_bounded(&bars->squares, parity, abort_flag, a.max_polls);
            const float eg = factors[token], ed = factors[kPiece + token], beta = factors[2 * kPiece + token], whole = factors[kPiece - 1];
            ptx::mbar_wait_bounded(&bars->done[0], parity, abort_flag, a.max_polls);
            ptx::tc_fence_after_sync();
            tmem_digits<C>(at, NV, X);
            if (is_key) {
                float y[C];
                Tile<T, NV>::get(values, token, col0, y);
                add_scaled(y, -eg, X);
#pragma unroll
                for (int j = 0; j < C; ++j) X[j] = y[j];
                scaled(y, beta, X);
                put_row<NV, C>(rows, W::rows_part, row, col0, y);
                ptx::fence_proxy_async_smem();
            } else {
                scaled(X, eg, X);
            }
            ptx::tc_fence_before_sync();
            __syncthreads();
            // D2: of keys E - R, of queries P' beta R
            ptx::mbar_wait_bounded(&bars->done[1], parity, abort_flag, a.max_polls);
            ptx::tc_fence_after_sync();
            float y[C];
            tmem_digits<C>(at + 3 * NV, NV, y);
            add_scaled(X, 1.f, y);
            if (is_key) {
                scaled(y, ed * beta, X);
                put_row<NV, C>(rows, W::rows_part, row, col0, y);
                ptx::fence_proxy_async_smem();
            }
            ptx::tc_fence_before_sync();
            __syncthreads();
            if (is_key) {
                if (a.updates) save_row<C>(a.updates + quad_at(unit0 + i, a.VP, kPiece, v, token), kPiece, saved, X);
            } else {
                scaled(X, a.scale, X);
                Tile<T, NV>::put(outputs, token, col0, X);
            }
            // D3, in D1's place: S <- e^G_63 S + K^T (..)
            ptx::mbar_wait_bounded(&bars->done[2], parity, abort_flag, a.max_polls);
            ptx::tc_fence_after_sync();
            tmem_digits<C>(at, NV, y);
            add_scaled(y, whole, S);
#pragma unroll
            for (int j = 0; j < C; ++j) S[j] = y[j];
            if (i + 1 < pieces) put_state(i + 1);
        }
        if (a.state_out && row < a.K) {
#pragma unroll
            for (int j = 0; j < C; ++j)
                if (j < there) a.state_out[state0 + j] = S[j];
        }
        zero_rows(static_cast<T*>(a.o) + (long long)b * a.L * a.ldo + (long long)h * a.V + v0, a.ldo, len, a.L, min(NV, a.V - v0), tid, kWorkers);
    } else {
        const long long row0 = (long long)b * a.L, col0 = (long long)h * a.V + v0;
        move_values<T, NV, WIDE, false>(static_cast<const T*>(a.v) + row0 * a.ldv + col0, a.ldv, static_cast<T*>(a.o) + row0 * a.ldo + col0, a.ldo, values, outputs, len, pieces,
                                        a.V - v0, tid - kPieceThreads);
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

template <typename T, int KD, int NV, bool WIDE>
conv2d_status_t walk(const DeltaArgs& a, cudaStream_t stream)
{
    using W = Walk<T, KD, NV, kPiece>;
    static SmemLimit limit;
    const int across = (int)ceil_div_u(a.V, NV);
    if (raise_smem_limit((const void*)delta_fwd_kernel<T, KD, NV, WIDE>, W::smem, limit) != cudaSuccess) return CONV2D_ERR_CUDA;
    if (launch_pdl(delta_fwd_kernel<T, KD, NV, WIDE>, dim3((unsigned)(a.B * a.H) * across), dim3(kWalkThreads), W::smem, stream, a, across) != cudaSuccess)
        return CONV2D_ERR_CUDA;
    count_launch();
    return CONV2D_OK;
}

template <typename T, int KD>
conv2d_status_t walk_wide(const DeltaArgs& a, cudaStream_t stream)
{
    const bool wide = a.V % (16 / sizeof(T)) == 0 && rows_aligned(a.v, a.ldv, sizeof(T), 16) && rows_aligned(a.o, a.ldo, sizeof(T), 16);
    if constexpr (sizeof(T) == 2 || KD == 64) {
        if (delta_columns<T, KD, kPiece>(a, wide) == 64) return walk<T, KD, 64, true>(a, stream);
    }
    return wide ? walk<T, KD, 32, true>(a, stream) : walk<T, KD, 32, false>(a, stream);
}

template <typename T>
conv2d_status_t walk_typed(const DeltaArgs& a, cudaStream_t stream)
{
    return a.K <= 64 ? walk_wide<T, 64>(a, stream) : walk_wide<T, 128>(a, stream);
}

}  // namespace

size_t delta_states_bytes(const DeltaLayout& l) { return l.prepared_bytes() + l.saved_bytes(); }
size_t delta_fwd_workspace_bytes(const DeltaLayout& l) { return l.prepared_bytes() + l.keys_bytes(); }

conv2d_status_t launch_delta_fwd(DeltaArgs a, conv2d_operand_t type, void* states, void* workspace, cudaStream_t stream)
{
    const DeltaLayout l(a.B, a.L, a.Hk, a.H, a.K, a.V, type);
    a.share = a.H / a.Hk, a.pieces = l.pieces, a.VP = l.VP;
    if (device_timeout_word(&a.timeout) != cudaSuccess) return CONV2D_ERR_CUDA;
    a.max_polls = (unsigned)env_int("CONV2D_B200_DELTA_MAX_POLLS", 1 << 22);
    // (sections of whole multiples of 16 bytes)
    unsigned char* at = static_cast<unsigned char*>(states ? states : workspace);
    a.prepared = at;
    if (states) {
        a.states = reinterpret_cast<float*>(at + l.prepared_bytes());
        a.updates = reinterpret_cast<float*>(at + l.prepared_bytes() + l.units * l.state());
    }
    a.keys = static_cast<unsigned char*>(workspace) + l.prepared_bytes();
    const conv2d_status_t st = launch_delta_prepare(a, type, true, stream);
    if (st != CONV2D_OK) return st;
    if (type == CONV2D_OPERAND_BF16) return walk_typed<bf16>(a, stream);
    if (type == CONV2D_OPERAND_FP16) return walk_typed<fp16>(a, stream);
    return walk_typed<float>(a, stream);
}

}  // namespace conv2d_b200
