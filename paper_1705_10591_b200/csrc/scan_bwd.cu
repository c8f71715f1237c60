// Launchers of the backward scan.
#include "scan_bwd.cuh"

namespace conv2d_b200 {
namespace {

// Columns of the partial sums by channel: dA, then dDskip, then ddelta_bias.
struct ChannelStore {
    float *dA, *dD, *dbias;
    int D, N, NQ;
    __device__ void operator()(long long col, float s) const
    {
        const long long quads = (long long)D * NQ;
        if (col < quads) {
            if (col % NQ < N) dA[col / NQ * N + col % NQ] = s;
        } else if (col < quads + D) {
            if (dD) dD[col - quads] = s;
        } else if (dbias) {
            dbias[col - quads - D] = s;
        }
    }
};

// dB, dC from the blocks' partial sums; a thread per row, group, tensor and state.
template <typename T>
__global__ void __launch_bounds__(256) scan_bwd_rows_kernel(const float* __restrict__ in, const int* lengths, T* dB, T* dC, int parts, long long rows, int L,
                                                            int G, int N, int NP, long long lddB, long long lddC)
{
    ptx::grid_dep_wait();
    const long long id = (long long)blockIdx.x * 256 + threadIdx.x;
    const int i = (int)(id % (2 * NP)), n = i % NP;
    const long long rg = id / (2 * NP), row = rg / G;
    const int g = (int)(rg % G);
    if (row >= rows || n >= N) return;
    float s = 0.f;
    if (row % L < sequence_length(lengths, (int)(row / L), L)) {
        const float* p = in + (((size_t)g * parts) * rows + row) * (2 * NP) + i;
        for (int k = 0; k < parts; ++k) s += p[(size_t)k * rows * (2 * NP)];
    }
    if (i < NP) dB[row * lddB + (long long)g * N + n] = from_float<T>(s);
    else dC[row * lddC + (long long)g * N + n] = from_float<T>(s);
}

// How the backward pass is cut: channel sets a block takes in turn, segments of time.
struct BwdCut { int nl, cb, sets, blocks_group, segs, rows; };
BwdCut bwd_cut(int B, int L, int D, int N, int G)
{
    BwdCut c;
    c.nl = lanes_for(N, kSpt);
    c.cb = c.nl == 1 ? 64 : 128 / c.nl;
    const int E = D / G;
    // A block's partial sums of dB and dC are for 32 channels (64 with up to eight states, 16 with more than 64: more sets do not fit into shared memory), to
    // keep the workspace down: they take 2 NP / 32 floats for each row and channel, 4 bytes with 16 states, 16 with 64 and 64 with 128.
    int sets = c.cb >= 32 ? 1 : 32 / c.cb;
    if (sets > 4) sets = 4;
    // fewer where half the machine would have no block, cut into segments as below (1 x 246 x 128 in two groups, 64 states, with the forward pass: 100 us with four sets, 61 with one)
    while (sets > 1 && (long long)B * G * ceil_div_u(E, (long long)c.cb * sets) * (L < 128 ? 1 : L / 64) * 2 <= 148) sets /= 2;
    c.sets = env_int("CONV2D_B200_SCAN_SETS", sets);
    if (c.sets < 1) c.sets = 1;
    c.blocks_group = (int)ceil_div_u(E, (long long)c.cb * c.sets);
    // segments of time, where the blocks leave two thirds of the machine idle: two blocks for every SM then, of 64 rows at least
    const long long blocks = (long long)B * G * c.blocks_group;
    long long segs = blocks * 3 <= 148 ? 2 * 148 / blocks : 1;
    if (segs > L / 64) segs = L / 64;
    segs = env_int("CONV2D_B200_SCAN_BWD_SEGS", (int)segs);
    if (segs < 1) segs = 1;
    c.rows = (int)(ceil_div_u(ceil_div_u(L, segs), kCheckpointRows) * kCheckpointRows);
    c.segs = (int)ceil_div_u(L, c.rows);
    return c;
}

struct BwdLayout { size_t local, steps, per_channel, per_row, total; };   // offsets in floats, each a multiple of four
BwdLayout bwd_layout(const BwdCut& c, int B, int L, int D, int N, int G)
{
    auto up4 = [](size_t n) { return (n + 3) / 4 * 4; };
    const size_t NQ = round4(N), bs = (size_t)B * c.segs;
    BwdLayout o;
    o.local = 0;
    o.steps = o.local + (c.segs > 1 ? bs * D * NQ : 0);
    o.per_channel = o.steps + (c.segs > 1 ? up4(bs * D) : 0);
    o.per_row = o.per_channel + bs * channel_floats(D, (int)NQ);
    o.total = o.per_row + (size_t)G * c.blocks_group * B * L * 2 * c.nl * kSpt;
    return o;
}

template <typename T, int NL, int V>
conv2d_status_t bwd(const ScanSeq& s, cudaStream_t stream)
{
    using Tile = ScanBwdTile<NL>;
    constexpr int e = sizeof(T);
    ScanBwdArgs<T> a;
    a.u = static_cast<const T*>(s.u), a.delta = static_cast<const T*>(s.delta), a.z = static_cast<const T*>(s.z), a.dy = static_cast<const T*>(s.dy);
    a.Bm = static_cast<const T*>(s.Bm), a.Cm = static_cast<const T*>(s.Cm);
    a.A = s.A, a.Dskip = s.Dskip, a.delta_bias = s.delta_bias, a.states = s.states_in, a.dstate_out = s.dstate_out, a.lengths = s.lengths;
    a.du = static_cast<T*>(s.du), a.ddelta = static_cast<T*>(s.ddelta), a.dz = static_cast<T*>(s.dz), a.dstate_in = s.dstate_in;
    a.B = s.B, a.L = s.L, a.D = s.D, a.N = s.N, a.G = s.G, a.E = s.D / s.G;
    a.ldu = (int)s.ldu, a.lddelta = (int)s.lddelta, a.ldB = (int)s.ldB, a.ldC = (int)s.ldC, a.ldz = s.z ? (int)s.ldz : 0, a.lddy = (int)s.lddy;
    a.lddu = (int)s.lddu, a.ldddelta = (int)s.ldddelta, a.lddz = s.dz ? (int)s.lddz : 0, a.softplus = s.softplus;
    const BwdCut c = bwd_cut(s.B, s.L, s.D, s.N, s.G);
    const BwdLayout o = bwd_layout(c, s.B, s.L, s.D, s.N, s.G);
    a.segs = c.segs, a.seg_rows = c.rows, a.blocks_group = c.blocks_group, a.sets = c.sets;
    a.local = s.ws + o.local, a.steps = s.ws + o.steps, a.per_channel = s.ws + o.per_channel, a.per_row = s.ws + o.per_row;
    const long long jobs = (long long)s.B * a.segs * s.G, blocks = (long long)a.segs * s.G * c.blocks_group, rows = (long long)s.B * s.L;     // blocks: of a sequence
    const int carry_group = (int)ceil_div_u(a.E, Tile::CB);
    const long long join = (long long)s.B * s.D * round4(s.N), per_row = rows * s.G * 2 * Tile::NP;
    // (segments are cut where there are few blocks; 2^39 elements of dB and dC are more than there is memory)
    if ((a.segs > 1 && jobs * carry_group > 0x7fffffffLL) || per_row / 256 > 0x7ffffff0LL) return CONV2D_ERR_SHAPE;
    if (a.segs > 1) {
        if (launch_pdl(scan_bwd_carry_kernel<T, NL, V>, dim3((unsigned)(jobs * carry_group)), dim3(Tile::SCAN), 0, stream, a, carry_group) != cudaSuccess)
            return CONV2D_ERR_CUDA;
        count_launch();
        if (launch_pdl(scan_join_kernel<true>, dim3(ceil_div_u(join, 256)), dim3(256), 0, stream, a.local, a.steps, s.A, s.dstate_out, s.dstate_in,
                       s.B, a.segs, s.D, s.N) != cudaSuccess) return CONV2D_ERR_CUDA;
        count_launch();
    }
    a.u_unit = copy_unit(s.u, s.ldu, a.E, e), a.delta_unit = copy_unit(s.delta, s.lddelta, a.E, e), a.z_unit = copy_unit(s.z, s.ldz, a.E, e);
    a.dy_unit = copy_unit(s.dy, s.lddy, a.E, e), a.B_unit = copy_unit(s.Bm, s.ldB, a.N, e), a.C_unit = copy_unit(s.Cm, s.ldC, a.N, e);
    a.out_quads = a.E % 4 == 0 && rows_aligned(s.du, s.lddu, e, 4 * e) && rows_aligned(s.ddelta, s.ldddelta, e, 4 * e) && rows_aligned(s.dz, s.lddz, e, 4 * e);
    static_assert(Tile::fixed(e) + (Tile::CB >= 32 ? 1 : 4) * Tile::set_bytes <= 227 * 1024, "the sets that bwd_cut allows");
    const size_t smem = Tile::fixed(e) + a.sets * Tile::set_bytes;
    static SmemLimit limit;
    if (raise_smem_limit(reinterpret_cast<const void*>(scan_bwd_kernel<T, NL>), smem, limit) != cudaSuccess) return CONV2D_ERR_CUDA;
    const int most = sequences_of_launch(blocks, 0x7fffffffLL, s.B);
    for (int b0 = 0; b0 < s.B; b0 += most) {
        ScanBwdArgs<T> r = a;           // (B stays: the partial sums of dB and dC are laid out by it)
        const size_t first = (size_t)b0 * s.L, state = (size_t)b0 * s.D * s.N, seg = (size_t)b0 * a.segs, NQ = round4(s.N);
        r.u += first * a.ldu, r.delta += first * a.lddelta, r.Bm += first * a.ldB, r.Cm += first * a.ldC, r.dy += first * a.lddy;
        r.du += first * a.lddu, r.ddelta += first * a.ldddelta;
        if (r.z) r.z += first * a.ldz, r.dz += first * a.lddz;
        if (r.dstate_out) r.dstate_out += state;
        if (r.dstate_in) r.dstate_in += state;
        if (r.lengths) r.lengths += b0;
        r.states += (size_t)b0 * ceil_div_u(s.L, kCheckpointRows) * s.D * NQ;
        if (a.segs > 1) r.local += seg * s.D * NQ, r.steps += seg * s.D;
        r.per_channel += seg * channel_floats(s.D, (int)NQ), r.per_row += first * 2 * Tile::NP;
        const int count = s.B - b0 < most ? s.B - b0 : most;
        if (launch_pdl(scan_bwd_kernel<T, NL>, dim3((unsigned)(blocks * count)), dim3(Tile::TH), smem, stream, r) != cudaSuccess) return CONV2D_ERR_CUDA;
        count_launch();
    }
    const conv2d_status_t st = launch_column_sums(a.per_channel, (long long)s.B * a.segs, (long long)s.D * (round4(s.N) + 2), channel_floats(s.D, round4(s.N)),
                                                  ChannelStore{s.dA, s.dD, s.ddelta_bias, s.D, s.N, round4(s.N)}, stream);
    if (st != CONV2D_OK) return st;
    if (launch_pdl(scan_bwd_rows_kernel<T>, dim3(ceil_div_u(per_row, 256)), dim3(256), 0, stream, a.per_row, s.lengths, static_cast<T*>(s.dB),
                   static_cast<T*>(s.dC), c.blocks_group, rows, s.L, s.G, s.N, Tile::NP, s.lddB, s.lddC) != cudaSuccess) return CONV2D_ERR_CUDA;
    count_launch();
    return CONV2D_OK;
}

template <typename T, int V>
conv2d_status_t bwd_lanes(const ScanSeq& s, cudaStream_t stream)
{
    switch (lanes_for(s.N, kSpt)) {
        case 1: return bwd<T, 1, V>(s, stream);
        case 2: return bwd<T, 2, V>(s, stream);
        case 4: return bwd<T, 4, V>(s, stream);
        case 8: return bwd<T, 8, V>(s, stream);
        case 16: return bwd<T, 16, V>(s, stream);
        case 32: return bwd<T, 32, V>(s, stream);
    }
    return CONV2D_ERR_UNSUPPORTED;
}

template <typename T>
conv2d_status_t bwd_typed(const ScanSeq& s, cudaStream_t stream)
{
    constexpr int e = sizeof(T), n = 4 * e;
    const bool wide = (s.D / s.G) % 4 == 0 && rows_aligned(s.u, s.ldu, e, n) && rows_aligned(s.delta, s.lddelta, e, n)
                   && rows_aligned(s.z, s.ldz, e, n) && rows_aligned(s.dy, s.lddy, e, n) && rows_aligned(s.du, s.lddu, e, n)
                   && rows_aligned(s.ddelta, s.ldddelta, e, n) && rows_aligned(s.dz, s.lddz, e, n);
    return wide ? bwd_lanes<T, 4>(s, stream) : bwd_lanes<T, 1>(s, stream);
}

}  // namespace

size_t scan_bwd_workspace_bytes(int B, int L, int D, int N, int G)
{
    return sizeof(float) * bwd_layout(bwd_cut(B, L, D, N, G), B, L, D, N, G).total;
}

conv2d_status_t launch_scan_bwd(const ScanSeq& s, conv2d_operand_t type, cudaStream_t stream)
{
    if (type == CONV2D_OPERAND_BF16) return bwd_typed<bf16>(s, stream);
    if (type == CONV2D_OPERAND_FP16) return bwd_typed<fp16>(s, stream);
    return bwd_typed<float>(s, stream);
}

}  // namespace conv2d_b200
