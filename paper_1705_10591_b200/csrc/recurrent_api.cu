// C-ABI boundary of the gated delta rule and of RMS norm: checks of arguments and dispatch.
#include <math.h>

#include "delta_common.cuh"
#include "rms_common.cuh"

namespace conv2d_b200 {
namespace {

bool known(conv2d_operand_t t) { return t == CONV2D_OPERAND_BF16 || t == CONV2D_OPERAND_FP16 || t == CONV2D_OPERAND_FP32; }
bool element_aligned(const void* p, size_t size) { return reinterpret_cast<uintptr_t>(p) % size == 0; }
template <typename... P>
bool all_aligned(size_t size, P... p) { return (element_aligned(p, size) && ...); }
// A tensor of rows: distance at least the row's length (a tensor that is not given has none), in 32 bits.
bool rows_ok(const void* p, long long ld, long long width) { return !p || (ld >= width && ld <= 0x7fffffffLL); }

conv2d_status_t check_workspace(const void* workspace, size_t given, size_t need)
{
    if (need == 0) return CONV2D_OK;
    if (!workspace) return CONV2D_ERR_NULL;
    if (!element_aligned(workspace, 16)) return CONV2D_ERR_ALIGN;
    return given < need ? CONV2D_ERR_WORKSPACE : CONV2D_OK;
}

constexpr int kMaxValues = 65536;

conv2d_status_t delta_extents(int B, int L, int Hk, int H, int K, int V)
{
    if (B <= 0 || L <= 0 || Hk <= 0 || H <= 0 || K <= 0 || V <= 0 || H % Hk != 0) return CONV2D_ERR_SHAPE;
    if ((long long)B * L > (1LL << 30) || (long long)H * V > (1 << 22) || (long long)Hk * K > (1 << 22)) return CONV2D_ERR_SHAPE;
    if (K > kMost || V > kMaxValues) return CONV2D_ERR_UNSUPPORTED;
    return delta_extents_ok(B, L, H, V) ? CONV2D_OK : CONV2D_ERR_SHAPE;
}

conv2d_status_t rms_extents(int M, int C, int G)
{
    if (M <= 0 || M > (1 << 30) || C <= 0 || G <= 0 || C % G != 0) return CONV2D_ERR_SHAPE;
    return C <= kMaxRmsChannels ? CONV2D_OK : CONV2D_ERR_UNSUPPORTED;
}

template <typename Bytes>
conv2d_status_t delta_size(int B, int L, int Hk, int H, int K, int V, conv2d_operand_t type, size_t* bytes, Bytes of)
{
    if (!bytes) return CONV2D_ERR_NULL;
    *bytes = 0;
    const conv2d_status_t st = delta_extents(B, L, Hk, H, K, V);
    if (st != CONV2D_OK) return st;
    if (!known(type)) return CONV2D_ERR_UNSUPPORTED;
    *bytes = of(DeltaLayout(B, L, Hk, H, K, V, type));
    return CONV2D_OK;
}

// What single tokens and whole sequences are checked for alike.
conv2d_status_t check_delta(const DeltaArgs& a, conv2d_operand_t type)
{
    if (!a.q || !a.k || !a.v || !a.g || !a.beta || !a.o) return CONV2D_ERR_NULL;
    const conv2d_status_t st = delta_extents(a.B, a.L, a.Hk, a.H, a.K, a.V);
    if (st != CONV2D_OK) return st;
    const long long qk = (long long)a.Hk * a.K, vo = (long long)a.H * a.V;
    if (!rows_ok(a.q, a.ldq, qk) || !rows_ok(a.k, a.ldk, qk) || !rows_ok(a.v, a.ldv, vo) || !rows_ok(a.o, a.ldo, vo) || !rows_ok(a.g, a.ldg, a.H) ||
        !rows_ok(a.beta, a.ldbeta, a.H))
        return CONV2D_ERR_SHAPE;
    if (!known(type)) return CONV2D_ERR_UNSUPPORTED;
    if (!all_aligned(element_size(type), a.q, a.k, a.v, a.o) || !all_aligned(4, a.g, a.beta, a.state_in, a.state_out, a.lengths)) return CONV2D_ERR_ALIGN;
    return CONV2D_OK;
}

}  // namespace
}  // namespace conv2d_b200

using namespace conv2d_b200;

extern "C" {

conv2d_status_t delta_states_size(int B, int L, int Hk, int H, int K, int V, conv2d_operand_t type, size_t* bytes)
{
    return delta_size(B, L, Hk, H, K, V, type, bytes, delta_states_bytes);
}
conv2d_status_t delta_fwd_gated_workspace_size(int B, int L, int Hk, int H, int K, int V, conv2d_operand_t type, size_t* bytes)
{
    return delta_size(B, L, Hk, H, K, V, type, bytes, delta_fwd_workspace_bytes);
}
conv2d_status_t delta_bwd_gated_workspace_size(int B, int L, int Hk, int H, int K, int V, conv2d_operand_t type, size_t* bytes)
{
    return delta_size(B, L, Hk, H, K, V, type, bytes, delta_bwd_workspace_bytes);
}

conv2d_status_t delta_fwd_gated(const void* q, const void* k, const void* v, const float* g, const float* beta,
                                const float* state_in, const int* lengths, void* o, float* state_out, void* states,
                                int B, int L, int Hk, int H, int K, int V, long long ldq, long long ldk, long long ldv,
                                long long ldg, long long ldbeta, long long ldo, float scale, conv2d_operand_t type,
                                void* workspace, size_t workspace_bytes, void* cuda_stream)
{
    DeltaArgs a{};
    a.q = q, a.k = k, a.v = v, a.g = g, a.beta = beta, a.state_in = state_in, a.lengths = lengths, a.o = o, a.state_out = state_out;
    a.B = B, a.L = L, a.Hk = Hk, a.H = H, a.K = K, a.V = V;
    a.ldq = ldq, a.ldk = ldk, a.ldv = ldv, a.ldg = ldg, a.ldbeta = ldbeta, a.ldo = ldo, a.scale = scale;
    conv2d_status_t st = check_delta(a, type);
    if (st != CONV2D_OK) return st;
    if (!element_aligned(states, 16)) return CONV2D_ERR_ALIGN;
    st = check_workspace(workspace, workspace_bytes, delta_fwd_workspace_bytes(DeltaLayout(B, L, Hk, H, K, V, type)));
    if (st != CONV2D_OK) return st;
    st = check_device();
    if (st != CONV2D_OK) return st;
    return launch_delta_fwd(a, type, states, workspace, static_cast<cudaStream_t>(cuda_stream));
}

conv2d_status_t delta_step_gated(const void* q, const void* k, const void* v, const float* g, const float* beta,
                                 const float* state_in, void* o, float* state_out,
                                 int B, int Hk, int H, int K, int V, long long ldq, long long ldk, long long ldv,
                                 long long ldg, long long ldbeta, long long ldo, float scale, conv2d_operand_t type, void* cuda_stream)
{
    if (!state_in || !state_out) return CONV2D_ERR_NULL;
    DeltaArgs a{};
    a.q = q, a.k = k, a.v = v, a.g = g, a.beta = beta, a.state_in = state_in, a.o = o, a.state_out = state_out;
    a.B = B, a.L = 1, a.Hk = Hk, a.H = H, a.K = K, a.V = V;
    a.ldq = ldq, a.ldk = ldk, a.ldv = ldv, a.ldg = ldg, a.ldbeta = ldbeta, a.ldo = ldo, a.scale = scale;
    conv2d_status_t st = check_delta(a, type);
    if (st != CONV2D_OK) return st;
    st = check_device();
    if (st != CONV2D_OK) return st;
    a.share = H / Hk;
    return launch_delta_step(a, type, static_cast<cudaStream_t>(cuda_stream));
}

conv2d_status_t delta_bwd_gated(const void* q, const void* k, const int* lengths, const void* states, const void* dout, const float* dstate_out,
                                void* dq, void* dk, void* dv, float* dg, float* dbeta, float* dstate_in,
                                int B, int L, int Hk, int H, int K, int V, long long ldq, long long ldk, long long lddo,
                                long long lddq, long long lddk, long long lddv, long long lddg, long long lddbeta,
                                float scale, conv2d_operand_t type, void* workspace, size_t workspace_bytes, void* cuda_stream)
{
    if (!q || !k || !states || !dout || !dq || !dk || !dv || !dg || !dbeta) return CONV2D_ERR_NULL;
    conv2d_status_t st = delta_extents(B, L, Hk, H, K, V);
    if (st != CONV2D_OK) return st;
    const long long qk = (long long)Hk * K, vo = (long long)H * V;
    if (!rows_ok(q, ldq, qk) || !rows_ok(k, ldk, qk) || !rows_ok(dout, lddo, vo) || !rows_ok(dq, lddq, qk) || !rows_ok(dk, lddk, qk) || !rows_ok(dv, lddv, vo) ||
        !rows_ok(dg, lddg, H) || !rows_ok(dbeta, lddbeta, H))
        return CONV2D_ERR_SHAPE;
    if (!known(type)) return CONV2D_ERR_UNSUPPORTED;
    if (!all_aligned(element_size(type), q, k, dout, dq, dk, dv) || !all_aligned(4, dg, dbeta, dstate_out, dstate_in, lengths) || !element_aligned(states, 16))
        return CONV2D_ERR_ALIGN;
    st = check_workspace(workspace, workspace_bytes, delta_bwd_workspace_bytes(DeltaLayout(B, L, Hk, H, K, V, type)));
    if (st != CONV2D_OK) return st;
    st = check_device();
    if (st != CONV2D_OK) return st;
    DeltaArgs a{};
    a.q = q, a.k = k, a.lengths = lengths, a.dout = dout, a.dstate_out = dstate_out;
    a.dq = dq, a.dk = dk, a.dv = dv, a.dg = dg, a.dbeta = dbeta, a.dstate_in = dstate_in;
    a.B = B, a.L = L, a.Hk = Hk, a.H = H, a.K = K, a.V = V;
    a.ldq = ldq, a.ldk = ldk, a.lddo = lddo, a.lddq = lddq, a.lddk = lddk, a.lddv = lddv, a.lddg = lddg, a.lddbeta = lddbeta, a.scale = scale;
    return launch_delta_bwd(a, type, states, workspace, static_cast<cudaStream_t>(cuda_stream));
}

conv2d_status_t norm_fwd_rms(const void* x, const void* residual, const void* z, const float* gamma, void* y, void* h,
                             void* y8, float* scales, float* rstd, int M, int C, int G, int block,
                             long long ldx, long long ldr, long long ldz, long long ldy, long long ldh, long long ld8,
                             float eps, conv2d_operand_t type, void* cuda_stream)
{
    if (!x || (!y && !y8) || !residual != !h || !y8 != !scales) return CONV2D_ERR_NULL;
    conv2d_status_t st = rms_extents(M, C, G);
    if (st != CONV2D_OK) return st;
    if (!rows_ok(x, ldx, C) || !rows_ok(residual, ldr, C) || !rows_ok(z, ldz, C) || !rows_ok(y, ldy, C) || !rows_ok(h, ldh, C) || !rows_ok(y8, ld8, C))
        return CONV2D_ERR_SHAPE;
    if ((y8 && block <= 0) || !(eps >= 0.f) || isinf(eps)) return CONV2D_ERR_SHAPE;
    if (!known(type)) return CONV2D_ERR_UNSUPPORTED;
    if (!all_aligned(element_size(type), x, residual, z, y, h) || !all_aligned(4, gamma, scales, rstd)) return CONV2D_ERR_ALIGN;
    st = check_device();
    if (st != CONV2D_OK) return st;
    RmsArgs a{};
    a.x = x, a.residual = residual, a.z = z, a.gamma = gamma, a.y = y, a.h = h, a.y8 = y8, a.scales = scales, a.rstd = rstd;
    a.M = M, a.C = C, a.G = G, a.block = block < C ? block : C, a.ldx = ldx, a.ldr = ldr, a.ldz = ldz, a.ldy = ldy, a.ldh = ldh, a.ld8 = ld8, a.eps = eps;
    return launch_rms_fwd(a, type, static_cast<cudaStream_t>(cuda_stream));
}

conv2d_status_t norm_bwd_rms_workspace_size(int M, int C, int G, size_t* bytes)
{
    if (!bytes) return CONV2D_ERR_NULL;
    *bytes = 0;
    const conv2d_status_t st = rms_extents(M, C, G);
    if (st == CONV2D_OK) *bytes = rms_bwd_workspace_bytes(M, C, G);
    return st;
}

conv2d_status_t norm_bwd_rms(const void* h, const void* z, const float* gamma, const float* rstd, const void* dy, const void* dh,
                             void* dx, void* dz, float* dgamma, int M, int C, int G,
                             long long ldh, long long ldz, long long lddy, long long lddh, long long lddx, long long lddz,
                             conv2d_operand_t type, void* workspace, size_t workspace_bytes, void* cuda_stream)
{
    if (!h || !rstd || !dy || !dx || !z != !dz) return CONV2D_ERR_NULL;
    conv2d_status_t st = rms_extents(M, C, G);
    if (st != CONV2D_OK) return st;
    if (!rows_ok(h, ldh, C) || !rows_ok(z, ldz, C) || !rows_ok(dy, lddy, C) || !rows_ok(dh, lddh, C) || !rows_ok(dx, lddx, C) || !rows_ok(dz, lddz, C))
        return CONV2D_ERR_SHAPE;
    if (!known(type)) return CONV2D_ERR_UNSUPPORTED;
    if (!all_aligned(element_size(type), h, z, dy, dh, dx, dz) || !all_aligned(4, gamma, rstd, dgamma)) return CONV2D_ERR_ALIGN;
    st = check_workspace(workspace, workspace_bytes, dgamma ? rms_bwd_workspace_bytes(M, C, G) : 0);
    if (st != CONV2D_OK) return st;
    st = check_device();
    if (st != CONV2D_OK) return st;
    RmsArgs a{};
    a.x = h, a.z = z, a.gamma = gamma, a.rstd_in = rstd, a.dy = dy, a.dh = dh, a.dx = dx, a.dz = dz, a.dgamma = dgamma;
    a.M = M, a.C = C, a.G = G, a.ldx = ldh, a.ldz = ldz, a.lddy = lddy, a.lddh = lddh, a.lddx = lddx, a.lddz = lddz;
    a.ws = static_cast<float*>(workspace);
    return launch_rms_bwd(a, type, static_cast<cudaStream_t>(cuda_stream));
}

}  // extern "C"
