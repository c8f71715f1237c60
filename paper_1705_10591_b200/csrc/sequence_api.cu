// C-ABI boundary of the operators along a sequence: checks of arguments and dispatch.
#include "seq_common.cuh"

#include <math.h>

namespace conv2d_b200 {
namespace {

constexpr int kMaxTaps = 8, kMaxStates = 128;

bool known(conv2d_operand_t t) { return t == CONV2D_OPERAND_BF16 || t == CONV2D_OPERAND_FP16 || t == CONV2D_OPERAND_FP32; }
bool known(conv2d_activation_t a) { return a >= CONV2D_ACT_NONE && a <= CONV2D_ACT_GELU; }

// Extents of B sequences of L rows of D channels: rows are counted in 32 bits (and by blocks, one of which may lie behind the last row), elements in 64;
// workspaces stay below 2^63 bytes.
bool extents_ok(long long B, long long L, long long D)
{
    return B > 0 && L > 0 && D > 0 && B * L <= (1LL << 30) && D <= (1 << 22);
}
bool element_aligned(const void* p, size_t size) { return reinterpret_cast<uintptr_t>(p) % size == 0; }

// A tensor of rows: distance at least the row's length (a tensor that is not given has none), in 32 bits.
bool rows_ok(const void* p, long long ld, long long width) { return !p || (ld >= width && ld <= 0x7fffffffLL); }

template <typename... P>
bool all_aligned(size_t size, P... p) { return (element_aligned(p, size) && ...); }

conv2d_status_t check_workspace(const void* workspace, size_t given, size_t need)
{
    if (need == 0) return CONV2D_OK;
    if (!workspace) return CONV2D_ERR_NULL;
    if (!element_aligned(workspace, 16)) return CONV2D_ERR_ALIGN;
    return given < need ? CONV2D_ERR_WORKSPACE : CONV2D_OK;
}

conv2d_status_t conv_extents(int B, int L, int D, int K)
{
    if (!extents_ok(B, L, D) || K <= 0) return CONV2D_ERR_SHAPE;
    return K > kMaxTaps ? CONV2D_ERR_UNSUPPORTED : CONV2D_OK;
}
conv2d_status_t scan_extents(int B, int L, int D, int N, int G)
{
    if (!extents_ok(B, L, D) || N <= 0 || G <= 0 || D % G != 0) return CONV2D_ERR_SHAPE;
    return N > kMaxStates ? CONV2D_ERR_UNSUPPORTED : CONV2D_OK;
}
conv2d_status_t norm_extents(int N, int S, int C, int G)
{
    if (!extents_ok(N, S, C) || G <= 0 || C % G != 0) return CONV2D_ERR_SHAPE;
    return CONV2D_OK;
}

}  // namespace
}  // namespace conv2d_b200

using namespace conv2d_b200;

extern "C" {

conv2d_status_t conv1d_fwd_causal(const void* x, const void* w, const void* bias, const void* state_in, const int* lengths,
                                  void* y, void* state_out, int B, int L, int D, int K, long long ldx, long long ldy,
                                  conv2d_operand_t type, conv2d_activation_t act, void* cuda_stream)
{
    if (!x || !w || !y) return CONV2D_ERR_NULL;
    conv2d_status_t st = conv_extents(B, L, D, K);
    if (st != CONV2D_OK) return st;
    if (!rows_ok(x, ldx, D) || !rows_ok(y, ldy, D)) return CONV2D_ERR_SHAPE;
    if (!known(type) || !known(act)) return CONV2D_ERR_UNSUPPORTED;
    if (!all_aligned(element_size(type), x, w, bias, state_in, y, state_out) || !element_aligned(lengths, 4)) return CONV2D_ERR_ALIGN;
    st = check_device();
    if (st != CONV2D_OK) return st;
    ConvSeq a{};
    a.x = x, a.w = w, a.bias = bias, a.state_in = state_in, a.lengths = lengths, a.y = y, a.state_out = state_out;
    a.B = B, a.L = L, a.D = D, a.K = K, a.ldx = ldx, a.ldy = ldy, a.act = act;
    return launch_conv1d_fwd(a, type, static_cast<cudaStream_t>(cuda_stream));
}

conv2d_status_t conv1d_step_causal(const void* x, const void* w, const void* bias, const void* state_in, void* y, void* state_out,
                                   int B, int D, int K, long long ldx, long long ldy,
                                   conv2d_operand_t type, conv2d_activation_t act, void* cuda_stream)
{
    if (K > 1 && (!state_in || !state_out)) return CONV2D_ERR_NULL;
    return conv1d_fwd_causal(x, w, bias, state_in, nullptr, y, state_out, B, 1, D, K, ldx, ldy, type, act, cuda_stream);
}

conv2d_status_t conv1d_bwd_causal_workspace_size(int B, int L, int D, int K, size_t* bytes)
{
    if (!bytes) return CONV2D_ERR_NULL;
    *bytes = 0;
    const conv2d_status_t st = conv_extents(B, L, D, K);
    if (st == CONV2D_OK) *bytes = conv1d_bwd_workspace_bytes(B, L, D, K);
    return st;
}

conv2d_status_t conv1d_bwd_causal(const void* x, const void* w, const void* bias, const void* state_in, const int* lengths,
                                  const void* dy, const void* dstate_out, void* dx, float* dw, float* dbias, void* dstate_in,
                                  int B, int L, int D, int K, long long ldx, long long lddy, long long lddx,
                                  conv2d_operand_t type, conv2d_activation_t act,
                                  void* workspace, size_t workspace_bytes, void* cuda_stream)
{
    if (!x || !w || !dy || !dx) return CONV2D_ERR_NULL;
    conv2d_status_t st = conv_extents(B, L, D, K);
    if (st != CONV2D_OK) return st;
    if (!rows_ok(x, ldx, D) || !rows_ok(dy, lddy, D) || !rows_ok(dx, lddx, D)) return CONV2D_ERR_SHAPE;
    if (!known(type) || !known(act)) return CONV2D_ERR_UNSUPPORTED;
    if (!all_aligned(element_size(type), x, w, bias, state_in, dy, dstate_out, dx, dstate_in) || !all_aligned(4, dw, dbias, lengths))
        return CONV2D_ERR_ALIGN;
    st = check_workspace(workspace, workspace_bytes, dw || dbias ? conv1d_bwd_workspace_bytes(B, L, D, K) : 0);
    if (st != CONV2D_OK) return st;
    st = check_device();
    if (st != CONV2D_OK) return st;
    ConvSeq a{};
    a.x = x, a.w = w, a.bias = bias, a.state_in = state_in, a.lengths = lengths, a.dy = dy, a.dstate_out = dstate_out;
    a.dx = dx, a.dw = dw, a.dbias = dbias, a.dstate_in = dstate_in;
    a.B = B, a.L = L, a.D = D, a.K = K, a.ldx = ldx, a.lddy = lddy, a.lddx = lddx, a.act = act;
    a.partials = static_cast<float*>(workspace);
    return launch_conv1d_bwd(a, type, static_cast<cudaStream_t>(cuda_stream));
}

conv2d_status_t scan_states_size(int B, int L, int D, int N, size_t* bytes)
{
    if (!bytes) return CONV2D_ERR_NULL;
    *bytes = 0;
    const conv2d_status_t st = scan_extents(B, L, D, N, 1);
    if (st == CONV2D_OK) *bytes = scan_states_bytes(B, L, D, N);
    return st;
}

conv2d_status_t scan_fwd_selective_workspace_size(int B, int L, int D, int N, int G, size_t* bytes)
{
    if (!bytes) return CONV2D_ERR_NULL;
    *bytes = 0;
    const conv2d_status_t st = scan_extents(B, L, D, N, G);
    if (st == CONV2D_OK) *bytes = scan_fwd_workspace_bytes(B, L, D, N, G);
    return st;
}

conv2d_status_t scan_fwd_selective(const void* u, const void* delta, const float* A, const void* Bm, const void* Cm,
                                   const float* Dskip, const void* z, const float* delta_bias,
                                   const float* state_in, const int* lengths, void* y, float* state_out, void* states,
                                   int B, int L, int D, int N, int G, long long ldu, long long lddelta,
                                   long long ldB, long long ldC, long long ldz, long long ldy,
                                   conv2d_operand_t type, unsigned flags,
                                   void* workspace, size_t workspace_bytes, void* cuda_stream)
{
    if (!u || !delta || !A || !Bm || !Cm || !y) return CONV2D_ERR_NULL;
    conv2d_status_t st = scan_extents(B, L, D, N, G);
    if (st != CONV2D_OK) return st;
    const long long gn = (long long)G * N;
    if (!rows_ok(u, ldu, D) || !rows_ok(delta, lddelta, D) || !rows_ok(z, ldz, D) || !rows_ok(y, ldy, D) || !rows_ok(Bm, ldB, gn)
        || !rows_ok(Cm, ldC, gn)) return CONV2D_ERR_SHAPE;
    if (!known(type) || (flags & ~(unsigned)CONV2D_FLAG_SCAN_SOFTPLUS)) return CONV2D_ERR_UNSUPPORTED;
    if (!all_aligned(element_size(type), u, delta, Bm, Cm, z, y) || !all_aligned(4, A, Dskip, delta_bias, state_in, lengths, state_out)
        || !element_aligned(states, 16)) return CONV2D_ERR_ALIGN;
    st = check_workspace(workspace, workspace_bytes, scan_fwd_workspace_bytes(B, L, D, N, G));
    if (st != CONV2D_OK) return st;
    st = check_device();
    if (st != CONV2D_OK) return st;
    ScanSeq a{};
    a.u = u, a.delta = delta, a.A = A, a.Bm = Bm, a.Cm = Cm, a.Dskip = Dskip, a.z = z, a.delta_bias = delta_bias, a.state_in = state_in;
    a.lengths = lengths, a.y = y, a.state_out = state_out, a.states = static_cast<float*>(states);
    a.B = B, a.L = L, a.D = D, a.N = N, a.G = G;
    a.ldu = ldu, a.lddelta = lddelta, a.ldB = ldB, a.ldC = ldC, a.ldz = ldz, a.ldy = ldy;
    a.softplus = flags & CONV2D_FLAG_SCAN_SOFTPLUS, a.ws = static_cast<float*>(workspace);
    return launch_scan_fwd(a, type, static_cast<cudaStream_t>(cuda_stream));
}

conv2d_status_t scan_step_selective(const void* u, const void* delta, const float* A, const void* Bm, const void* Cm,
                                    const float* Dskip, const void* z, const float* delta_bias,
                                    const float* state_in, void* y, float* state_out,
                                    int B, int D, int N, int G, long long ldu, long long lddelta,
                                    long long ldB, long long ldC, long long ldz, long long ldy,
                                    conv2d_operand_t type, unsigned flags, void* cuda_stream)
{
    if (!u || !delta || !A || !Bm || !Cm || !y || !state_in || !state_out) return CONV2D_ERR_NULL;
    conv2d_status_t st = scan_extents(B, 1, D, N, G);
    if (st != CONV2D_OK) return st;
    const long long gn = (long long)G * N;
    if (!rows_ok(u, ldu, D) || !rows_ok(delta, lddelta, D) || !rows_ok(z, ldz, D) || !rows_ok(y, ldy, D) || !rows_ok(Bm, ldB, gn)
        || !rows_ok(Cm, ldC, gn)) return CONV2D_ERR_SHAPE;
    if (!known(type) || (flags & ~(unsigned)CONV2D_FLAG_SCAN_SOFTPLUS)) return CONV2D_ERR_UNSUPPORTED;
    if (!all_aligned(element_size(type), u, delta, Bm, Cm, z, y) || !all_aligned(4, A, Dskip, delta_bias, state_in, state_out))
        return CONV2D_ERR_ALIGN;
    st = check_device();
    if (st != CONV2D_OK) return st;
    ScanSeq a{};
    a.u = u, a.delta = delta, a.A = A, a.Bm = Bm, a.Cm = Cm, a.Dskip = Dskip, a.z = z, a.delta_bias = delta_bias, a.state_in = state_in;
    a.y = y, a.state_out = state_out, a.B = B, a.L = 1, a.D = D, a.N = N, a.G = G;
    a.ldu = ldu, a.lddelta = lddelta, a.ldB = ldB, a.ldC = ldC, a.ldz = ldz, a.ldy = ldy;
    a.softplus = flags & CONV2D_FLAG_SCAN_SOFTPLUS;
    return launch_scan_step(a, type, static_cast<cudaStream_t>(cuda_stream));
}

conv2d_status_t scan_bwd_selective_workspace_size(int B, int L, int D, int N, int G, size_t* bytes)
{
    if (!bytes) return CONV2D_ERR_NULL;
    *bytes = 0;
    const conv2d_status_t st = scan_extents(B, L, D, N, G);
    if (st == CONV2D_OK) *bytes = scan_bwd_workspace_bytes(B, L, D, N, G);
    return st;
}

conv2d_status_t scan_bwd_selective(const void* u, const void* delta, const float* A, const void* Bm, const void* Cm,
                                   const float* Dskip, const void* z, const float* delta_bias, const int* lengths,
                                   const void* states, const void* dy, const float* dstate_out,
                                   void* du, void* ddelta, float* dA, void* dB, void* dC, float* dDskip, void* dz,
                                   float* ddelta_bias, float* dstate_in,
                                   int B, int L, int D, int N, int G, long long ldu, long long lddelta,
                                   long long ldB, long long ldC, long long ldz, long long lddy,
                                   long long lddu, long long ldddelta, long long lddB, long long lddC, long long lddz,
                                   conv2d_operand_t type, unsigned flags,
                                   void* workspace, size_t workspace_bytes, void* cuda_stream)
{
    if (!u || !delta || !A || !Bm || !Cm || !states || !dy || !du || !ddelta || !dA || !dB || !dC || !workspace) return CONV2D_ERR_NULL;
    if ((z != nullptr) != (dz != nullptr) || (dDskip && !Dskip)) return CONV2D_ERR_NULL;
    conv2d_status_t st = scan_extents(B, L, D, N, G);
    if (st != CONV2D_OK) return st;
    const long long gn = (long long)G * N;
    if (!rows_ok(u, ldu, D) || !rows_ok(delta, lddelta, D) || !rows_ok(z, ldz, D) || !rows_ok(dy, lddy, D) || !rows_ok(Bm, ldB, gn)
        || !rows_ok(Cm, ldC, gn) || !rows_ok(du, lddu, D) || !rows_ok(ddelta, ldddelta, D) || !rows_ok(dz, lddz, D)
        || !rows_ok(dB, lddB, gn) || !rows_ok(dC, lddC, gn)) return CONV2D_ERR_SHAPE;
    if (!known(type) || (flags & ~(unsigned)CONV2D_FLAG_SCAN_SOFTPLUS)) return CONV2D_ERR_UNSUPPORTED;
    if (!all_aligned(element_size(type), u, delta, Bm, Cm, z, dy, du, ddelta, dB, dC, dz)
        || !all_aligned(4, A, Dskip, delta_bias, lengths, dstate_out, dA, dDskip, ddelta_bias, dstate_in)
        || !element_aligned(states, 16)) return CONV2D_ERR_ALIGN;
    st = check_workspace(workspace, workspace_bytes, scan_bwd_workspace_bytes(B, L, D, N, G));
    if (st != CONV2D_OK) return st;
    st = check_device();
    if (st != CONV2D_OK) return st;
    ScanSeq a{};
    a.u = u, a.delta = delta, a.A = A, a.Bm = Bm, a.Cm = Cm, a.Dskip = Dskip, a.z = z, a.delta_bias = delta_bias;
    a.lengths = lengths, a.states_in = static_cast<const float*>(states), a.dy = dy, a.dstate_out = dstate_out;
    a.du = du, a.ddelta = ddelta, a.dA = dA, a.dB = dB, a.dC = dC, a.dD = dDskip, a.dz = dz, a.ddelta_bias = ddelta_bias, a.dstate_in = dstate_in;
    a.B = B, a.L = L, a.D = D, a.N = N, a.G = G;
    a.ldu = ldu, a.lddelta = lddelta, a.ldB = ldB, a.ldC = ldC, a.ldz = ldz, a.lddy = lddy;
    a.lddu = lddu, a.ldddelta = ldddelta, a.lddB = lddB, a.lddC = lddC, a.lddz = lddz;
    a.softplus = flags & CONV2D_FLAG_SCAN_SOFTPLUS, a.ws = static_cast<float*>(workspace);
    return launch_scan_bwd(a, type, static_cast<cudaStream_t>(cuda_stream));
}

conv2d_status_t norm_fwd_groups_workspace_size(int N, int S, int C, int G, size_t* bytes)
{
    if (!bytes) return CONV2D_ERR_NULL;
    *bytes = 0;
    const conv2d_status_t st = norm_extents(N, S, C, G);
    if (st == CONV2D_OK) *bytes = norm_fwd_workspace_bytes(N, S, C, G);
    return st;
}

conv2d_status_t norm_fwd_groups(const void* x, const float* gamma, const float* beta, void* y, float* mean, float* rstd,
                                int N, int S, int C, int G, long long ldx, long long ldy, float eps,
                                conv2d_operand_t type, conv2d_activation_t act,
                                void* workspace, size_t workspace_bytes, void* cuda_stream)
{
    if (!x || !y) return CONV2D_ERR_NULL;
    conv2d_status_t st = norm_extents(N, S, C, G);
    if (st != CONV2D_OK) return st;
    if (!rows_ok(x, ldx, C) || !rows_ok(y, ldy, C) || !(eps >= 0.f) || isinf(eps)) return CONV2D_ERR_SHAPE;
    if (!known(type) || !known(act)) return CONV2D_ERR_UNSUPPORTED;
    if (!all_aligned(element_size(type), x, y) || !all_aligned(4, gamma, beta, mean, rstd)) return CONV2D_ERR_ALIGN;
    st = check_workspace(workspace, workspace_bytes, norm_fwd_workspace_bytes(N, S, C, G));
    if (st != CONV2D_OK) return st;
    st = check_device();
    if (st != CONV2D_OK) return st;
    NormSeq a{};
    a.x = x, a.gamma = gamma, a.beta = beta, a.y = y, a.mean = mean, a.rstd = rstd;
    a.N = N, a.S = S, a.C = C, a.G = G, a.ldx = ldx, a.ldy = ldy, a.eps = eps, a.act = act, a.ws = static_cast<float*>(workspace);
    return launch_norm_fwd(a, type, static_cast<cudaStream_t>(cuda_stream));
}

conv2d_status_t norm_bwd_groups_workspace_size(int N, int S, int C, int G, size_t* bytes)
{
    if (!bytes) return CONV2D_ERR_NULL;
    *bytes = 0;
    const conv2d_status_t st = norm_extents(N, S, C, G);
    if (st == CONV2D_OK) *bytes = norm_bwd_workspace_bytes(N, S, C, G);
    return st;
}

conv2d_status_t norm_bwd_groups(const void* x, const float* gamma, const float* beta, const float* mean, const float* rstd,
                                const void* dy, void* dx, float* dgamma, float* dbeta,
                                int N, int S, int C, int G, long long ldx, long long lddy, long long lddx,
                                conv2d_operand_t type, conv2d_activation_t act,
                                void* workspace, size_t workspace_bytes, void* cuda_stream)
{
    if (!x || !mean || !rstd || !dy || !dx) return CONV2D_ERR_NULL;
    conv2d_status_t st = norm_extents(N, S, C, G);
    if (st != CONV2D_OK) return st;
    if (!rows_ok(x, ldx, C) || !rows_ok(dy, lddy, C) || !rows_ok(dx, lddx, C)) return CONV2D_ERR_SHAPE;
    if (!known(type) || !known(act)) return CONV2D_ERR_UNSUPPORTED;
    if (!all_aligned(element_size(type), x, dy, dx) || !all_aligned(4, gamma, beta, mean, rstd, dgamma, dbeta)) return CONV2D_ERR_ALIGN;
    st = check_workspace(workspace, workspace_bytes, norm_bwd_workspace_bytes(N, S, C, G));
    if (st != CONV2D_OK) return st;
    st = check_device();
    if (st != CONV2D_OK) return st;
    NormSeq a{};
    a.x = x, a.gamma = gamma, a.beta = beta, a.mean = const_cast<float*>(mean), a.rstd = const_cast<float*>(rstd);
    a.dy = dy, a.dx = dx, a.dgamma = dgamma, a.dbeta = dbeta;
    a.N = N, a.S = S, a.C = C, a.G = G, a.ldx = ldx, a.lddy = lddy, a.lddx = lddx, a.act = act, a.ws = static_cast<float*>(workspace);
    return launch_norm_bwd(a, type, static_cast<cudaStream_t>(cuda_stream));
}

}  // extern "C"
