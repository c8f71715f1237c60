// What the two kernels that walk a sequence's pieces share: warps that compute, warps that load, the stages of shared memory between them.
#pragma once

#include "delta_common.cuh"

namespace conv2d_b200 {

// Up to four warps of 16 columns compute, four others copy what the next piece needs into the other stage: one barrier of the block for a piece, no
// waiting in loops.  One stage where two do not fit.
constexpr int kLoaders = 4, kComputing = 4;

template <typename T, int KD>
struct Walk {
    static constexpr int IN = Parts<T>::in, SUM = Parts<T>::sum;
    static constexpr size_t keys = (size_t)IN * kPiece * KD * 2, square = (size_t)SUM * kPiece * kPiece * 2;
    static constexpr int kPad = 16 / (int)sizeof(T);                              // elements between rows of values, against bank conflicts
    // K, Q, t, P, values of `warps` * 16 columns, factors
    __host__ __device__ static constexpr size_t values(int warps) { return (size_t)kPiece * (warps * 16 + kPad) * sizeof(T); }
    __host__ __device__ static constexpr size_t stage(int warps) { return 2 * keys + 2 * square + values(warps) + kFactors * kPiece * 4; }
    __host__ __device__ static constexpr size_t staging(int warps) { return (size_t)warps * kPiece * (16 + kPad) * sizeof(T); }      // a warp's output rows
    static constexpr int stages = 2 * stage(kComputing) + staging(kComputing) <= 232448 ? 2 : 1;
    static size_t smem(int warps) { return stages * stage(warps) + staging(warps); }
};

// Addresses of a stage.
template <typename T, int KD>
struct Stage {
    unsigned char* at;
    int warps;
    __device__ uint32_t k() const { return ptx::smem_u32(at); }
    __device__ uint32_t q() const { return k() + (uint32_t)Walk<T, KD>::keys; }
    __device__ uint32_t t() const { return q() + (uint32_t)Walk<T, KD>::keys; }
    __device__ uint32_t p() const { return t() + (uint32_t)Walk<T, KD>::square; }
    __device__ T* values() const { return reinterpret_cast<T*>(at + 2 * Walk<T, KD>::keys + 2 * Walk<T, KD>::square); }
    __device__ float* factors() const { return reinterpret_cast<float*>(at + Walk<T, KD>::stage(warps) - kFactors * kPiece * 4); }
    __device__ int pitch() const { return warps * 16 + Walk<T, KD>::kPad; }
};

// Everything of a piece into a stage; by the loading warps, or by all.
template <typename T, int KD>
__device__ __forceinline__ void load_piece(const DeltaArgs& a, const Stage<T, KD>& s, const T* values, long long ldvalues, bool wide, int b, int h, int piece, int live,
                                           int v0, int id, int threads)
{
    constexpr int SUM = Parts<T>::sum;
    const size_t unit = ((size_t)b * a.H + h) * a.pieces + piece;
    const int hk = h / a.share;
    copy_keys<KD, Parts<T>::in>(a, s.k(), 0, b, hk, piece, live, id, threads);
    copy_keys<KD, Parts<T>::in>(a, s.q(), 1, b, hk, piece, live, id, threads);
    copy_rows<kPiece>(a.t + unit * (SUM * kPiece * kPiece), s.t(), SUM * kPiece, SUM * kPiece, id, threads);
    copy_rows<kPiece>(a.p + unit * (SUM * kPiece * kPiece), s.p(), SUM * kPiece, SUM * kPiece, id, threads);
    const float* f = a.factors + unit * (kFactors * kPiece);
    for (int i = id; i < 3 * kPiece / 4; i += threads) copy_async<16>(s.factors() + 4 * i, f + 4 * i);
    copy_values(values + ((long long)b * a.L + (long long)piece * kPiece) * ldvalues + (long long)h * a.V + v0, ldvalues, s.values(), s.pitch(), s.warps * 16, live,
                a.V - v0, wide, id, threads);
}

// A warp's 16 columns of 64 tokens, transposed in accumulators, out as rows; rows from `live` on are left alone.
template <typename T>
__device__ __forceinline__ void store_columns(const float (&x)[8][4], T* mine, T* to, long long ld, int live, int cols, bool wide, int lane)
{
    constexpr int PITCH = 16 + 16 / (int)sizeof(T), PER = 16 / (int)sizeof(T);
    const int g = lane >> 2, c = 2 * (lane & 3);
#pragma unroll
    for (int n = 0; n < 8; ++n) {
#pragma unroll
        for (int e = 0; e < 4; ++e) mine[(n * 8 + c + (e & 1)) * PITCH + g + 8 * (e >> 1)] = from_float<T>(x[n][e]);
    }
    __syncwarp();
    if (wide) {
        constexpr int UNITS = 16 / PER;
#pragma unroll
        for (int i = lane; i < kPiece * UNITS; i += 32) {
            const int row = i / UNITS, u = i % UNITS * PER;
            if (row < live && u < cols) *reinterpret_cast<uint4*>(to + row * ld + u) = *reinterpret_cast<const uint4*>(mine + row * PITCH + u);
        }
    } else {
        for (int i = lane; i < kPiece * 16; i += 32) {
            const int row = i / 16, u = i % 16;
            if (row < live && u < cols) to[row * ld + u] = mine[row * PITCH + u];
        }
    }
    __syncwarp();
}

// Rows of zeros behind a sequence: columns 0 .. cols - 1 of rows first .. L - 1.
template <typename T>
__device__ __forceinline__ void zero_rows(T* to, long long ld, int first, int L, int cols, int id, int threads)
{
    for (long long i = id; i < (long long)(L - first) * cols; i += threads) to[(first + i / cols) * ld + i % cols] = from_float<T>(0.f);
}

// How many warps a block computes with: as many as leave a block for every SM, since a warp's time for a piece is its own and only loading is shared.
inline int delta_warps(const DeltaArgs& a)
{
    int warps = kComputing;
    while (warps > 1 && (a.VP / 16 < warps || (long long)a.B * a.H * ceil_div_u(a.VP / 16, warps) < sm_count())) warps /= 2;
    return warps;
}

}  // namespace conv2d_b200
