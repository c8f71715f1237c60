// Launchers of the forward scan.
#include "scan_fwd.cuh"

namespace conv2d_b200 {
namespace {

// States of a lane: four, so that a channel's states make several lanes' work; eight where four would take more lanes than a warp has.
int states_of_lane(int N) { return N > 64 ? 8 : 4; }

// Segments of time.  A segmented walk takes every exponential twice, so sequences stay whole unless their blocks leave two thirds of the machine
// idle; then there are two blocks for every SM, of 64 rows at least.
struct FwdCut { int segs, rows; };
FwdCut fwd_cut(int B, int L, int D, int N, int G)
{
    const int nl = lanes_for(N, states_of_lane(N)), cb = (nl >= 16 ? 8 : 4) * 32 / nl;
    const long long blocks = (long long)B * G * ceil_div_u(D / G, cb);
    long long segs = blocks * 3 <= 148 ? 2 * 148 / blocks : 1;
    if (segs > L / 64) segs = L / 64;
    segs = env_int("CONV2D_B200_SCAN_SEGS", (int)segs);
    if (segs < 1) segs = 1;
    FwdCut c;
    c.rows = (int)(ceil_div_u(ceil_div_u(L, segs), 32) * 32);
    c.segs = (int)ceil_div_u(L, c.rows);
    return c;
}

template <typename T, int NL, int SPT, bool STATE_ONLY>
conv2d_status_t walk(ScanFwdArgs<T> a, cudaStream_t stream)
{
    using Tile = ScanFwdTile<NL, SPT>;
    constexpr size_t smem = Tile::smem(sizeof(T));
    static_assert(smem <= 227 * 1024, "shared memory of a block");
    a.blocks_group = (int)ceil_div_u(a.E, Tile::CB);
    const long long blocks = (long long)a.segs * a.G * a.blocks_group;      // of a sequence
    const int most = sequences_of_launch(blocks, 0x7fffffffLL, a.B);
    static SmemLimit limit;
    if (raise_smem_limit(reinterpret_cast<const void*>(scan_fwd_kernel<T, NL, SPT, STATE_ONLY>), smem, limit) != cudaSuccess) return CONV2D_ERR_CUDA;
    for (int b0 = 0; b0 < a.B; b0 += most) {
        ScanFwdArgs<T> r = a;
        const size_t rows = (size_t)b0 * a.L, state = (size_t)b0 * a.D * a.N, NQ = round4(a.N);
        r.u += rows * a.ldu, r.delta += rows * a.lddelta, r.Bm += rows * a.ldB, r.Cm += rows * a.ldC, r.y += rows * a.ldy;
        if (r.z) r.z += rows * a.ldz;
        if (r.state_in) r.state_in += state;
        if (r.state_out) r.state_out += state;
        if (r.lengths) r.lengths += b0;
        if (r.states) r.states += (size_t)b0 * ceil_div_u(a.L, kCheckpointRows) * a.D * NQ;
        if (a.segs > 1) r.local += (size_t)b0 * a.segs * a.D * NQ, r.steps += (size_t)b0 * a.segs * a.D;
        r.B = a.B - b0 < most ? a.B - b0 : most;
        if (launch_pdl(scan_fwd_kernel<T, NL, SPT, STATE_ONLY>, dim3((unsigned)(blocks * r.B)), dim3(Tile::TH), smem, stream, r) != cudaSuccess)
            return CONV2D_ERR_CUDA;
        count_launch();
    }
    return CONV2D_OK;
}

template <typename T, int NL, int SPT>
conv2d_status_t fwd(const ScanSeq& s, cudaStream_t stream)
{
    constexpr int e = sizeof(T);
    ScanFwdArgs<T> a;
    a.u = static_cast<const T*>(s.u), a.delta = static_cast<const T*>(s.delta), a.z = static_cast<const T*>(s.z);
    a.Bm = static_cast<const T*>(s.Bm), a.Cm = static_cast<const T*>(s.Cm);
    a.A = s.A, a.Dskip = s.Dskip, a.delta_bias = s.delta_bias, a.state_in = s.state_in, a.lengths = s.lengths;
    a.y = static_cast<T*>(s.y), a.state_out = s.state_out, a.states = s.states;
    a.B = s.B, a.L = s.L, a.D = s.D, a.N = s.N, a.G = s.G, a.E = s.D / s.G;
    a.ldu = (int)s.ldu, a.lddelta = (int)s.lddelta, a.ldB = (int)s.ldB, a.ldC = (int)s.ldC, a.ldz = s.z ? (int)s.ldz : 0, a.ldy = (int)s.ldy, a.softplus = s.softplus;
    const FwdCut cut = fwd_cut(s.B, s.L, s.D, s.N, s.G);
    a.segs = cut.segs, a.seg_rows = cut.rows, a.blocks_group = 0;
    a.u_unit = copy_unit(s.u, s.ldu, a.E, e), a.delta_unit = copy_unit(s.delta, s.lddelta, a.E, e), a.z_unit = copy_unit(s.z, s.ldz, a.E, e);
    a.B_unit = copy_unit(s.Bm, s.ldB, a.N, e), a.C_unit = copy_unit(s.Cm, s.ldC, a.N, e);
    a.wide = a.u_unit == 16 && a.delta_unit == 16 && (!s.z || a.z_unit == 16) && a.B_unit == 16 && a.C_unit == 16;
    a.y_quads = a.E % 4 == 0 && rows_aligned(s.y, s.ldy, e, 4 * e);
    a.local = s.ws;
    a.steps = s.ws ? s.ws + (size_t)s.B * a.segs * s.D * round4(s.N) : nullptr;
    if (a.segs > 1) {
        const conv2d_status_t st = walk<T, NL, SPT, true>(a, stream);
        if (st != CONV2D_OK) return st;
        if (launch_pdl(scan_join_kernel<false>, dim3(ceil_div_u((long long)s.B * s.D * round4(s.N), 256)), dim3(256), 0, stream, a.local, a.steps, s.A,
                       s.state_in, (float*)nullptr, s.B, a.segs, s.D, s.N) != cudaSuccess) return CONV2D_ERR_CUDA;
        count_launch();
    }
    return walk<T, NL, SPT, false>(a, stream);
}

template <typename T>
conv2d_status_t fwd_typed(const ScanSeq& s, cudaStream_t stream)
{
    if (states_of_lane(s.N) == 8) return fwd<T, 16, 8>(s, stream);
    switch (lanes_for(s.N, 4)) {
        case 1: return fwd<T, 1, 4>(s, stream);
        case 2: return fwd<T, 2, 4>(s, stream);
        case 4: return fwd<T, 4, 4>(s, stream);
        case 8: return fwd<T, 8, 4>(s, stream);
        case 16: return fwd<T, 16, 4>(s, stream);
    }
    return CONV2D_ERR_UNSUPPORTED;
}

}  // namespace

size_t scan_states_bytes(int B, int L, int D, int N)
{
    return sizeof(float) * (size_t)B * ceil_div_u(L, kCheckpointRows) * D * round4(N);
}
size_t scan_fwd_workspace_bytes(int B, int L, int D, int N, int G)
{
    const FwdCut s = fwd_cut(B, L, D, N, G);
    return s.segs > 1 ? sizeof(float) * (size_t)B * s.segs * D * (round4(N) + 1) : 0;
}

conv2d_status_t launch_scan_fwd(const ScanSeq& s, conv2d_operand_t type, cudaStream_t stream)
{
    if (type == CONV2D_OPERAND_BF16) return fwd_typed<bf16>(s, stream);
    if (type == CONV2D_OPERAND_FP16) return fwd_typed<fp16>(s, stream);
    return fwd_typed<float>(s, stream);
}
}  // namespace conv2d_b200
