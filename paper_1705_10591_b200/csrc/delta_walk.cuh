// What the two kernels that walk a sequence's pieces share: tensor-core products of tiles in shared memory, the threads' places in them, loads.
//
// A block walks one head of one sequence for NV columns of V.  A piece is three tcgen05 products with accumulators of 128 rows in tensor memory, each waiting for
// what threads make of the one before: with 32 columns a piece is all latency, and registers, not memory, hand S and E on.
//   D1 [128] = [K; Q] S            rows of K as they lie (K-major), S written by its threads, a row a thread (N-major)
//   D2 [128] = [-t; P'] (beta R)   both lie transposed, as rows of tokens j with 64 numbers each: M-major
//   D3 [128] = K^T (..)            the tile of K read the other way (M-major)
// Eight warps own a quarter of the 128 rows and one half of the columns each: a thread has one row of D1 and D2 (a token of K or of Q) and of S (a number of
// K).  A ninth warp issues the products and the copies of the next piece's tiles, and three more move values and outputs between their tensors and shared memory, whole
// lines at a time.  (Threads that fetched and stored their rows themselves, 32 lines an access, held the memory pipe for 600 cycles of a piece; a bulk
// copy for each row took twice as long again.)
#pragma once

#include "delta_common.cuh"

namespace conv2d_b200 {

constexpr int kWorkers = 256, kMovers = 96, kPieceThreads = kWorkers + 32, kWalkThreads = kPieceThreads + kMovers;

template <typename T, int KD, int NV, int ROWS>
struct Walk {
    static constexpr int IN = Parts<T>::in, HALF = 2 * kPiece * 128;              // bytes of 64 numbers of [K; Q]
    static constexpr int keys = IN * (KD / 64) * HALF, key_part = (KD / 64) * HALF, square_part = 2 * kPiece * 128;
    static constexpr int state_part = KD * NV * 2, rows_part = ROWS * NV * 2;     // S, and the ROWS rows of what D2 and D3 are products with
    static constexpr int state = kSum * state_part, values = kPiece * NV * (int)sizeof(T);
    // squares with their factors (and the barriers, to the next boundary of the swizzle), S, rows, values that come and go
    static constexpr int squares = (int)kPrepared, at_values = (squares + 128 + 1023) / 1024 * 1024 + state + kSum * rows_part;
    static constexpr int rest = at_values + 2 * values;
    static constexpr int stages = 2 * keys + rest <= 232448 - 1024 ? 2 : 1;
    static constexpr int smem = stages * keys + rest + 1024;                      // (1024: to the first boundary of the swizzle)
    static constexpr int cols = NV == 32 ? 256 : 512;                             // of tensor memory: twice three times NV, to a power of two
    static constexpr int C = NV / 2;                                              // columns of a thread
    static_assert(smem <= 232448, "a piece does not fit");
};

// Descriptors: [K; Q] and [-t^T | P'^T] have rows of 128 bytes, atoms of 8 rows.
__device__ __forceinline__ uint64_t rows_as_m(uint32_t at) { return ptx::smem_desc_sw128(at, 16, 1024); }
// columns as M, rows as K; `next`: distance to the following 64 columns
__device__ __forceinline__ uint64_t columns_as_m(uint32_t at, uint32_t next) { return ptx::smem_desc_sw128(at, next, 1024); }
// rows as K, their NV numbers as N; `next`: distance to the following NV
template <int NV>
__device__ __forceinline__ uint64_t rows_as_k(uint32_t at, uint32_t next)
{
    if (NV == 64) return ptx::smem_desc_sw128(at, next, 1024);
    // 64-byte swizzle: atoms of 8 rows x 64 bytes
    return (uint64_t)((at >> 4) & 0x3FFFu) | ((uint64_t)(next >> 4) << 16) | ((uint64_t)(512 >> 4) << 32) | (1ull << 46) | (4ull << 61);
}
constexpr uint32_t kIdescAMajorM = 1u << 15;

__device__ __forceinline__ void tmem_row(uint32_t at, float (&f)[16])
{
    uint32_t v[16];
    ptx::tmem_ld16(at, v);
    ptx::tmem_ld_wait();
#pragma unroll
    for (int i = 0; i < 16; ++i) f[i] = __uint_as_float(v[i]);
}
// The sum of products whose digits lie in three places, `step` columns apart.
template <int N> __device__ __forceinline__ void tmem_digits(uint32_t at, uint32_t step, float (&f)[N])
{
#pragma unroll
    for (int c = 0; c < N; c += 16) {
        uint32_t v[kSum][16];
#pragma unroll
        for (int p = 0; p < kSum; ++p) ptx::tmem_ld16(at + p * step + c, v[p]);
        ptx::tmem_ld_wait();
#pragma unroll
        for (int i = 0; i < 16; i += 2) {
            auto pair = [&](int p) { return make_float2(__uint_as_float(v[p][i]), __uint_as_float(v[p][i + 1])); };
            const float2 sum = __fadd2_rn(__fadd2_rn(pair(2), pair(1)), pair(0));
            f[c + i] = sum.x, f[c + i + 1] = sum.y;
        }
    }
}

// y <- a x + y, and x <- a x, two numbers at a time.
template <int N> __device__ __forceinline__ void add_scaled(float (&y)[N], float a, const float (&x)[N])
{
#pragma unroll
    for (int j = 0; j < N; j += 2) {
        const float2 r = __ffma2_rn(both(a), make_float2(x[j], x[j + 1]), make_float2(y[j], y[j + 1]));
        y[j] = r.x, y[j + 1] = r.y;
    }
}
template <int N> __device__ __forceinline__ void scaled(float (&y)[N], float a, const float (&x)[N])
{
#pragma unroll
    for (int j = 0; j < N; j += 2) {
        const float2 r = __fmul2_rn(both(a), make_float2(x[j], x[j + 1]));
        y[j] = r.x, y[j + 1] = r.y;
    }
}

// N numbers of row `row` from column `col` on (a multiple of 8), as parts, into a tile of rows of NV.
template <int NV, int N>
__device__ __forceinline__ void put_row(unsigned char* tile, int part_bytes, int row, int col, const float (&f)[N])
{
#pragma unroll
    for (int u = 0; u < N / 8; ++u) {
        uint32_t w[4][kSum];
#pragma unroll
        for (int j = 0; j < 4; ++j) split<kSum>(f[8 * u + 2 * j], f[8 * u + 2 * j + 1], w[j]);
#pragma unroll
        for (int p = 0; p < kSum; ++p) *reinterpret_cast<uint4*>(tile + p * part_bytes + unit_at<NV>(0, row, col / 8 + u)) = make_uint4(w[0][p], w[1][p], w[2][p], w[3][p]);
    }
}

// Four numbers, of which the first PARTS parts are not zero, likewise at place four_at() of a tile.
template <int NV> __device__ __forceinline__ int four_at(int row, int col) { return (int)unit_at<NV>(0, row, col / 8) + (col & 4) * 2; }
template <int PARTS>
__device__ __forceinline__ void put_four(unsigned char* at, int part_bytes, const float (&f)[4])
{
    uint32_t w[2][PARTS];
    split<PARTS>(f[0], f[1], w[0]);
    split<PARTS>(f[2], f[3], w[1]);
#pragma unroll
    for (int p = 0; p < kSum; ++p)
        *reinterpret_cast<uint2*>(at + p * part_bytes) = p < PARTS ? make_uint2(w[0][p < PARTS ? p : 0], w[1][p < PARTS ? p : 0]) : make_uint2(0u, 0u);
}

// What a pass keeps of a piece lies as [V/4][rows][4], so that the lanes of a warp, a row each, write and read whole lines (rows of V as they come: every
// access of a warp touched 32 lines, and a training step's walks waited twice as long for their stores as for everything else).
__device__ __forceinline__ size_t quad_at(size_t unit, int VP, int rows, int v, int row) { return unit * ((size_t)rows * VP) + ((size_t)(v >> 2) * rows + row) * 4; }
template <int N>
__device__ __forceinline__ void save_row(float* to, int rows, int there, const float (&f)[N])
{
#pragma unroll
    for (int i = 0; i < N; i += 4)
        if (i < there) *reinterpret_cast<float4*>(to + (size_t)i * rows) = make_float4(f[i], f[i + 1], f[i + 2], f[i + 3]);
}
template <int N>
struct SavedRow {
    Pack<float, 4> q[N / 4];
    __device__ __forceinline__ void load(const float* from, int rows, int there)
    {
#pragma unroll
        for (int i = 0; i < N / 4; ++i) q[i] = load_masked<float, 4>(from + (size_t)i * 4 * rows, 4 * i < there);
    }
};

// Rows of zeros behind a sequence: columns 0 .. cols - 1 of rows first .. L - 1.
template <typename T>
__device__ __forceinline__ void zero_rows(T* to, long long ld, int first, int L, int cols, int id, int threads)
{
    for (long long i = id; i < (long long)(L - first) * cols; i += threads) to[(first + i / cols) * ld + i % cols] = from_float<T>(0.f);
}

// Barriers of a block, 128 bytes at most.
struct WalkBars {
    uint64_t keys[2], squares, done[3], settled;
    uint32_t tmem, abort;
};
// Behind a wait that gave up: before a block ends, its copies (`issued` onto a barrier, the last of which may be under way) and its products are waited for, with a limit.
__device__ __forceinline__ void settle(uint64_t* bar, int issued)
{
    for (uint32_t i = 0; issued > 0 && i < (1u << 22); ++i)
        if (ptx::mbar_try_wait(bar, (issued - 1) & 1)) return;
}
__device__ __forceinline__ void settle_products(uint64_t* unused, uint32_t elected)
{
    ptx::mma_commit(unused, elected);
    settle(unused, 1);
}

// Tiles of 64 tokens x NV elements as they lie in their tensor, in units of 16 bytes swizzled like the operands.
template <typename T, int NV>
struct Tile {
    static constexpr int PER = 16 / (int)sizeof(T), UNITS = NV / PER, EACH = (kPiece * UNITS + kMovers - 1) / kMovers;
    static __device__ __forceinline__ uint32_t at(int row, int unit) { return unit_at<8 * UNITS>(0, row, unit); }
    // N elements of a row
    template <int N>
    static __device__ __forceinline__ void get(const unsigned char* tile, int row, int col, float (&f)[N])
    {
#pragma unroll
        for (int j = 0; j < N; j += PER) {
            float z[PER];
            unpack(load_pack<T, PER>(reinterpret_cast<const T*>(tile + at(row, (col + j) / PER))), z);
#pragma unroll
            for (int e = 0; e < PER; ++e) f[j + e] = z[e];
        }
    }
    template <int N>
    static __device__ __forceinline__ void put(unsigned char* tile, int row, int col, const float (&f)[N])
    {
#pragma unroll
        for (int j = 0; j < N; j += PER) {
            float z[PER];
#pragma unroll
            for (int e = 0; e < PER; ++e) z[e] = f[j + e];
            store_pack<T, PER>(reinterpret_cast<T*>(tile + at(row, (col + j) / PER)), pack<T, PER>(z));
        }
    }
};
// What a moving thread has under way of one tile; `id` of kMovers.
template <typename T, int NV, bool WIDE>
struct Mover {
    using L = Tile<T, NV>;
    static constexpr int TAKES = WIDE ? L::EACH : (kPiece * NV + kMovers - 1) / kMovers;       // single elements, or units
    Pack<T, WIDE ? L::PER : 1> p[TAKES];
    // from a tensor: zeros behind the last row and column
    __device__ __forceinline__ void fetch(const T* from, long long ld, int rows, int cols, int id)
    {
        constexpr int PER = WIDE ? L::PER : 1, ACROSS = NV / PER;
#pragma unroll
        for (int j = 0; j < TAKES; ++j) {
            const int u = id + j * kMovers, row = u / ACROSS, col = u % ACROSS * PER;
            p[j] = load_masked<T, PER>(from + row * ld + col, row < rows && col < cols);
        }
    }
    __device__ __forceinline__ void put(unsigned char* tile, int id) const
    {
        constexpr int PER = WIDE ? L::PER : 1, ACROSS = NV / PER;
#pragma unroll
        for (int j = 0; j < TAKES; ++j) {
            const int u = id + j * kMovers, row = u / ACROSS, col = u % ACROSS * PER;
            if (row < kPiece) store_pack<T, PER>(reinterpret_cast<T*>(tile + L::at(row, col / L::PER) + col % L::PER * sizeof(T)), p[j]);
        }
    }
    static __device__ __forceinline__ void store(T* to, long long ld, const unsigned char* tile, int rows, int cols, int id)
    {
        if (WIDE) {
#pragma unroll
            for (int j = 0; j < L::EACH; ++j) {
                const int u = id + j * kMovers, row = u / L::UNITS, col = u % L::UNITS * L::PER;
                if (row < rows && col < cols) store_pack<T, L::PER>(to + row * ld + col, load_pack<T, L::PER>(reinterpret_cast<const T*>(tile + L::at(row, col / L::PER))));
            }
        } else {
            for (int i = id; i < kPiece * NV; i += kMovers) {
                const int row = i / NV, col = i % NV;
                if (row < rows && col < cols) to[row * ld + col] = *reinterpret_cast<const T*>(tile + L::at(row, col / L::PER) + col % L::PER * sizeof(T));
            }
        }
    }
};
// The moving warps' part of a walk over `pieces` pieces, from the first on or from the last back, with the same three barriers a piece: values are fetched a piece
// ahead and put when they have been read, outputs are stored a piece later.
template <typename T, int NV, bool WIDE, bool BACK>
__device__ __forceinline__ void move_values(const T* from, long long ldfrom, T* to, long long ldto, unsigned char* values, const unsigned char* outputs, int len, int pieces,
                                            int cols, int id)
{
    Mover<T, NV, WIDE> m;
    auto piece = [&](int s) { return BACK ? pieces - 1 - s : s; };
    auto row = [&](int s) { return (long long)piece(s) * kPiece; };
    auto rows = [&](int s) { return min(len - piece(s) * kPiece, kPiece); };
    if (pieces > 0) {
        m.fetch(from + row(0) * ldfrom, ldfrom, rows(0), cols, id);
        m.put(values, id);
    }
    for (int s = 0; s < pieces; ++s) {
        __syncthreads();
        if (s + 1 < pieces) m.fetch(from + row(s + 1) * ldfrom, ldfrom, rows(s + 1), cols, id);
        if (s > 0) m.store(to + row(s - 1) * ldto, ldto, outputs, rows(s - 1), cols, id);
        __syncthreads();
        if (s + 1 < pieces) m.put(values, id);
        __syncthreads();
    }
    __syncthreads();                                           // (all have done their part)
    if (pieces > 0) m.store(to + row(pieces - 1) * ldto, ldto, outputs, rows(pieces - 1), cols, id);
}

// Products of parts with B's three side by side along N: part p of A, of `a_parts`, with the first 3 - p of B onto the digits from p on.  A is read once for
// each of its parts so (it is A's 4 KB that an MMA waits for while N is below 128: with every pair of parts an MMA of its own the three
// products of a piece took 2.4 times as long), and small terms are not added to large ones before the end.
template <int NV, bool A_BY_M, bool B_BY_N, typename DescA, typename DescB>
__device__ __forceinline__ void multiply_digits(uint32_t d, int a_parts, int ks, uint32_t elected, DescA desc_a, DescB desc_b)
{
#pragma unroll
    for (int p = 0; p < a_parts; ++p) {
        const uint32_t idesc = ptx::idesc_b16(128, (kSum - p) * NV, false) | (A_BY_M ? kIdescAMajorM : 0) | (B_BY_N ? ptx::kIdescBMajorMN : 0);
#pragma unroll
        for (int k = 0; k < ks; ++k) ptx::mma_b16(d + p * NV, desc_a(p, k), desc_b(k), idesc, p + k > 0, elected);
    }
}
// The same one after the other onto one place, those of the last digits first; B has `b_parts` parts.  `more`: onto what is there.
template <typename DescA, typename DescB>
__device__ __forceinline__ void multiply(uint32_t d, int a_parts, int b_parts, int ks, uint32_t idesc, uint32_t elected, bool more, DescA desc_a, DescB desc_b)
{
#pragma unroll
    for (int digits = kSum - 1; digits >= 0; --digits) {
#pragma unroll
        for (int p = 0; p <= digits; ++p) {
            if (p >= a_parts || digits - p >= b_parts) continue;
#pragma unroll
            for (int k = 0; k < ks; ++k) {
                ptx::mma_b16(d, desc_a(p, k), desc_b(digits - p, k), idesc, more, elected);
                more = true;
            }
        }
    }
}

// Of numbers in three parts, the products of first parts, and all others that count, small ones first.
template <typename DescA, typename DescB>
__device__ __forceinline__ void multiply_first(uint32_t d, int ks, uint32_t idesc, uint32_t elected, bool more, DescA desc_a, DescB desc_b)
{
#pragma unroll
    for (int k = 0; k < ks; ++k) ptx::mma_b16(d, desc_a(0, k), desc_b(0, k), idesc, more || k > 0, elected);
}
template <typename DescA, typename DescB>
__device__ __forceinline__ void multiply_small(uint32_t d, int ks, uint32_t idesc, uint32_t elected, bool more, DescA desc_a, DescB desc_b)
{
#pragma unroll
    for (int digits = kSum - 1; digits >= 1; --digits)
#pragma unroll
        for (int p = 0; p <= digits; ++p)
#pragma unroll
            for (int k = 0; k < ks; ++k) {
                ptx::mma_b16(d, desc_a(p, k), desc_b(digits - p, k), idesc, more, elected);
                more = true;
            }
}

// Columns a block walks with: 32, or 64 where those are fewer rounds of the machine's SMs.  A piece takes 2.3 us with 32 columns and 3.4 with 64; where the keys of two
// pieces do not fit beside 64 (fp16, in two parts) and are waited for, 4.5, so that two rounds of 32 are no slower.  Keys of 128 fp32 numbers, in three parts,
// leave room for 32, and rows that rule out accesses of 16 bytes are walked with 32.
template <typename T, int KD, int ROWS>
int delta_columns(const DeltaArgs& a, bool wide)
{
    if (!wide || a.V <= 32 || (sizeof(T) == 4 && a.K > 64)) return 32;
    const long long heads = (long long)a.B * a.H, sms = sm_count();
    const long long by32 = (heads * ceil_div_u(a.V, 32) + sms - 1) / sms, by64 = (heads * ceil_div_u(a.V, 64) + sms - 1) / sms;
    bool two = false;
    if constexpr (sizeof(T) == 2 || KD == 64) two = Walk<T, KD, 64, ROWS>::stages == 2;
    return env_int("CONV2D_B200_DELTA_COLUMNS", (two ? 3 * by64 <= 2 * by32 : 2 * by64 < by32) ? 64 : 32) == 64 ? 64 : 32;
}

}  // namespace conv2d_b200
