"""ctypes binding of libconv2d_b200.so: same names and argument order as the C headers.

Pointers are passed as integers (``tensor.data_ptr()`` / ``ndarray.ctypes.data``),
streams as the integer ``torch.cuda.current_stream().cuda_stream``.  Nothing here
computes anything and nothing falls back to another implementation: if the
library is missing or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes
from pathlib import Path

ALGO_AUTO, ALGO_FFMA, ALGO_TF32, ALGO_16BIT = 0, 1, 2, 3
OPERAND_BF16, OPERAND_FP16, OPERAND_FP32 = 0, 1, 2
ACT_NONE, ACT_RELU, ACT_SILU, ACT_GELU = 0, 1, 2, 3
FLAG_WEIGHTS_PACKED = 1
FLAG_SCAN_SOFTPLUS = 1

_LIB_PATH = Path(__file__).resolve().parent / "libconv2d_b200.so"
_lib = None


class Conv2dError(RuntimeError):
    """A library call returned a status other than CONV2D_OK."""

    def __init__(self, status: int, where: str):
        self.status = int(status)
        super().__init__(f"{where}: status {self.status} ({conv2d_status_string(self.status)})")


def library_path() -> Path:
    return _LIB_PATH


def load_library() -> ctypes.CDLL:
    """Loads the shared library (built in-tree by ``python -m paper_1705_10591_b200.build``)."""
    global _lib
    if _lib is not None:
        return _lib
    if not _LIB_PATH.exists():
        raise FileNotFoundError(
            f"{_LIB_PATH} is missing: build it with `python -m paper_1705_10591_b200.build` "
            "(there is no fallback implementation)")
    lib = ctypes.CDLL(str(_LIB_PATH))
    vp, i, sz, u = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t, ctypes.c_uint
    lib.conv2d_fwd_workspace_size.argtypes = [i] * 7 + [i, ctypes.POINTER(sz)]
    lib.conv2d_fwd_workspace_size.restype = i
    lib.conv2d_fwd_plan_describe.argtypes = [i] * 7 + [i, ctypes.c_char_p, sz]
    lib.conv2d_fwd_plan_describe.restype = i
    lib.conv2d_fwd_single_channel.argtypes = [vp, vp, vp] + [i] * 6 + [vp, sz, u, vp]
    lib.conv2d_fwd_single_channel.restype = i
    lib.conv2d_fwd_general.argtypes = [vp, vp, vp] + [i] * 7 + [i, vp, sz, u, vp]
    lib.conv2d_fwd_general.restype = i
    lib.conv2d_fwd_general_16bit.argtypes = [vp, vp, vp] + [i] * 7 + [i, vp, sz, u, vp]
    lib.conv2d_fwd_general_16bit.restype = i
    lib.conv2d_fwd_padded_workspace_size.argtypes = [i] * 9 + [i, ctypes.POINTER(sz)]
    lib.conv2d_fwd_padded_workspace_size.restype = i
    lib.conv2d_fwd_general_padded.argtypes = [vp, vp, vp] + [i] * 9 + [i, vp, sz, u, vp]
    lib.conv2d_fwd_general_padded.restype = i
    lib.conv2d_fwd_strided_workspace_size.argtypes = [i] * 10 + [i, ctypes.POINTER(sz)]
    lib.conv2d_fwd_strided_workspace_size.restype = i
    lib.conv2d_fwd_general_strided.argtypes = [vp, vp, vp] + [i] * 10 + [i, vp, sz, u, vp]
    lib.conv2d_fwd_general_strided.restype = i
    lib.conv2d_fwd_general_noalloc.argtypes = [vp, vp, vp] + [i] * 7 + [i, vp]
    lib.conv2d_fwd_general_noalloc.restype = i
    lib.conv2d_fwd_host.argtypes = [vp] * 6 + [i] * 7 + [i, vp, sz, vp]
    lib.conv2d_fwd_host.restype = i
    lib.conv2d_get_status.argtypes = [vp, vp]
    lib.conv2d_get_status.restype = i
    lib.conv2d_status_string.argtypes = [i]
    lib.conv2d_status_string.restype = ctypes.c_char_p
    lib.conv2d_launch_count.argtypes = []
    lib.conv2d_launch_count.restype = ctypes.c_ulonglong
    ll, f = ctypes.c_longlong, ctypes.c_float
    for name, args in {
        "conv1d_fwd_causal": [vp] * 7 + [i] * 4 + [ll] * 2 + [i, i, vp],
        "conv1d_step_causal": [vp] * 6 + [i] * 3 + [ll] * 2 + [i, i, vp],
        "conv1d_bwd_causal_workspace_size": [i] * 4 + [ctypes.POINTER(sz)],
        "conv1d_bwd_causal": [vp] * 11 + [i] * 4 + [ll] * 3 + [i, i, vp, sz, vp],
        "scan_states_size": [i] * 4 + [ctypes.POINTER(sz)],
        "scan_fwd_selective_workspace_size": [i] * 5 + [ctypes.POINTER(sz)],
        "scan_fwd_selective": [vp] * 13 + [i] * 5 + [ll] * 6 + [i, u, vp, sz, vp],
        "scan_step_selective": [vp] * 11 + [i] * 4 + [ll] * 6 + [i, u, vp],
        "scan_bwd_selective_workspace_size": [i] * 5 + [ctypes.POINTER(sz)],
        "scan_bwd_selective": [vp] * 21 + [i] * 5 + [ll] * 11 + [i, u, vp, sz, vp],
        "norm_fwd_groups_workspace_size": [i] * 4 + [ctypes.POINTER(sz)],
        "norm_fwd_groups": [vp] * 6 + [i] * 4 + [ll] * 2 + [f, i, i, vp, sz, vp],
        "norm_bwd_groups_workspace_size": [i] * 4 + [ctypes.POINTER(sz)],
        "norm_bwd_groups": [vp] * 9 + [i] * 4 + [ll] * 3 + [i, i, vp, sz, vp],
        "delta_states_size": [i] * 7 + [ctypes.POINTER(sz)],
        "delta_fwd_gated_workspace_size": [i] * 7 + [ctypes.POINTER(sz)],
        "delta_fwd_gated": [vp] * 10 + [i] * 6 + [ll] * 6 + [f, i, vp, sz, vp],
        "delta_step_gated": [vp] * 8 + [i] * 5 + [ll] * 6 + [f, i, vp],
        "delta_bwd_gated_workspace_size": [i] * 7 + [ctypes.POINTER(sz)],
        "delta_bwd_gated": [vp] * 12 + [i] * 6 + [ll] * 8 + [f, i, vp, sz, vp],
        "norm_fwd_rms": [vp] * 9 + [i] * 4 + [ll] * 6 + [f, i, vp],
        "norm_bwd_rms_workspace_size": [i] * 3 + [ctypes.POINTER(sz)],
        "norm_bwd_rms": [vp] * 9 + [i] * 3 + [ll] * 6 + [i, vp, sz, vp],
    }.items():
        getattr(lib, name).argtypes = args
        getattr(lib, name).restype = i
    _lib = lib
    return lib


def _check(status: int, where: str) -> None:
    if status != 0:
        raise Conv2dError(status, where)


def conv2d_status_string(status: int) -> str:
    return load_library().conv2d_status_string(int(status)).decode()


def conv2d_launch_count() -> int:
    return int(load_library().conv2d_launch_count())


def conv2d_fwd_workspace_size(N, C, H, W, K, R, S, algo=ALGO_AUTO) -> int:
    out = ctypes.c_size_t(0)
    _check(load_library().conv2d_fwd_workspace_size(N, C, H, W, K, R, S, algo, ctypes.byref(out)),
           "conv2d_fwd_workspace_size")
    return int(out.value)


def conv2d_fwd_plan_describe(N, C, H, W, K, R, S, algo=ALGO_AUTO) -> dict:
    """The library's description of its tensor-core plan for a shape, as a dict of its key=value pairs."""
    buf = ctypes.create_string_buffer(1024)
    _check(load_library().conv2d_fwd_plan_describe(N, C, H, W, K, R, S, algo, buf, len(buf)), "conv2d_fwd_plan_describe")
    out = {}
    for pair in buf.value.decode().split():
        key, _, val = pair.partition("=")
        try:
            out[key] = int(val)
        except ValueError:
            try:
                out[key] = float(val)
            except ValueError:
                out[key] = val
    return out


def conv2d_fwd_single_channel(x_ptr, w_ptr, y_ptr, N, H, W, K, R, S,
                              workspace_ptr=0, workspace_bytes=0, flags=0, stream=0) -> None:
    _check(load_library().conv2d_fwd_single_channel(x_ptr, w_ptr, y_ptr, N, H, W, K, R, S,
                                                    workspace_ptr or None, workspace_bytes, flags, stream or None),
           "conv2d_fwd_single_channel")


def conv2d_fwd_general(x_ptr, w_ptr, y_ptr, N, C, H, W, K, R, S, algo=ALGO_AUTO,
                       workspace_ptr=0, workspace_bytes=0, flags=0, stream=0) -> None:
    _check(load_library().conv2d_fwd_general(x_ptr, w_ptr, y_ptr, N, C, H, W, K, R, S, algo,
                                             workspace_ptr or None, workspace_bytes, flags, stream or None),
           "conv2d_fwd_general")


def conv2d_fwd_general_16bit(x_ptr, w_ptr, y_ptr, N, C, H, W, K, R, S, operand=OPERAND_BF16,
                             workspace_ptr=0, workspace_bytes=0, flags=0, stream=0) -> None:
    """x, w: device tensors of bf16 or fp16 elements (as `operand` says); y: device fp32 tensor."""
    _check(load_library().conv2d_fwd_general_16bit(x_ptr, w_ptr, y_ptr, N, C, H, W, K, R, S, operand,
                                                   workspace_ptr or None, workspace_bytes, flags, stream or None),
           "conv2d_fwd_general_16bit")


def conv2d_fwd_padded_workspace_size(N, C, H, W, K, R, S, pad_h, pad_w, algo=ALGO_AUTO) -> int:
    out = ctypes.c_size_t(0)
    _check(load_library().conv2d_fwd_padded_workspace_size(N, C, H, W, K, R, S, pad_h, pad_w, algo, ctypes.byref(out)),
           "conv2d_fwd_padded_workspace_size")
    return int(out.value)


def conv2d_fwd_general_padded(x_ptr, w_ptr, y_ptr, N, C, H, W, K, R, S, pad_h, pad_w, algo=ALGO_AUTO,
                              workspace_ptr=0, workspace_bytes=0, flags=0, stream=0) -> None:
    """Zero padding of pad_h rows / pad_w columns on every side; y is [N, K, H+2*pad_h-R+1, W+2*pad_w-S+1]."""
    _check(load_library().conv2d_fwd_general_padded(x_ptr, w_ptr, y_ptr, N, C, H, W, K, R, S, pad_h, pad_w, algo,
                                                    workspace_ptr or None, workspace_bytes, flags, stream or None),
           "conv2d_fwd_general_padded")


def conv2d_fwd_strided_workspace_size(N, C, H, W, K, R, S, pad_h, pad_w, stride, algo=ALGO_AUTO) -> int:
    out = ctypes.c_size_t(0)
    _check(load_library().conv2d_fwd_strided_workspace_size(N, C, H, W, K, R, S, pad_h, pad_w, stride, algo,
                                                            ctypes.byref(out)), "conv2d_fwd_strided_workspace_size")
    return int(out.value)


def conv2d_fwd_general_strided(x_ptr, w_ptr, y_ptr, N, C, H, W, K, R, S, pad_h, pad_w, stride, algo=ALGO_AUTO,
                               workspace_ptr=0, workspace_bytes=0, flags=0, stream=0) -> None:
    """Zero padding and stride; y is [N, K, (H+2*pad_h-R)//stride+1, (W+2*pad_w-S)//stride+1]."""
    _check(load_library().conv2d_fwd_general_strided(x_ptr, w_ptr, y_ptr, N, C, H, W, K, R, S, pad_h, pad_w, stride, algo,
                                                     workspace_ptr or None, workspace_bytes, flags, stream or None),
           "conv2d_fwd_general_strided")


def conv2d_fwd_general_noalloc(x_ptr, w_ptr, y_ptr, N, C, H, W, K, R, S, wait=0, stream=0) -> None:
    """Tensor-core convolution whose scratch is the library's own fixed device array (see the header)."""
    _check(load_library().conv2d_fwd_general_noalloc(x_ptr, w_ptr, y_ptr, N, C, H, W, K, R, S,
                                                     int(wait), stream or None),
           "conv2d_fwd_general_noalloc")


def conv2d_fwd_host(x_host_ptr, w_host_ptr, y_host_ptr, x_ptr, w_ptr, y_ptr, N, C, H, W, K, R, S,
                    algo=ALGO_AUTO, workspace_ptr=0, workspace_bytes=0, stream=0) -> None:
    _check(load_library().conv2d_fwd_host(x_host_ptr, w_host_ptr, y_host_ptr, x_ptr, w_ptr, y_ptr,
                                          N, C, H, W, K, R, S, algo,
                                          workspace_ptr or None, workspace_bytes, stream or None),
           "conv2d_fwd_host")


def conv2d_get_status(workspace_ptr=0, stream=0) -> None:
    """Waits for the stream; raises if a kernel reported a device-side timeout."""
    _check(load_library().conv2d_get_status(workspace_ptr or None, stream or None), "conv2d_get_status")


# ---- operators along a sequence (sequence_b200.h).  Pointers that are optional there may be 0.

def _size(name, *args) -> int:
    out = ctypes.c_size_t(0)
    _check(getattr(load_library(), name)(*args, ctypes.byref(out)), name)
    return int(out.value)


def conv1d_fwd_causal(x_ptr, w_ptr, bias_ptr, state_in_ptr, lengths_ptr, y_ptr, state_out_ptr, B, L, D, K, ldx, ldy,
                      operand=OPERAND_BF16, act=ACT_NONE, stream=0) -> None:
    """Causal convolution of every channel with its own K taps; x, y [B*L, D] with rows ldx, ldy elements apart."""
    _check(load_library().conv1d_fwd_causal(x_ptr or None, w_ptr or None, bias_ptr or None, state_in_ptr or None, lengths_ptr or None,
                                            y_ptr or None, state_out_ptr or None, B, L, D, K, ldx, ldy, operand, act, stream or None),
           "conv1d_fwd_causal")


def conv1d_step_causal(x_ptr, w_ptr, bias_ptr, state_in_ptr, y_ptr, state_out_ptr, B, D, K, ldx, ldy,
                       operand=OPERAND_BF16, act=ACT_NONE, stream=0) -> None:
    """One token of every sequence; the two states [B, K-1, D] may be one buffer."""
    _check(load_library().conv1d_step_causal(x_ptr or None, w_ptr or None, bias_ptr or None, state_in_ptr or None, y_ptr or None,
                                             state_out_ptr or None, B, D, K, ldx, ldy, operand, act, stream or None),
           "conv1d_step_causal")


def conv1d_bwd_causal_workspace_size(B, L, D, K) -> int:
    return _size("conv1d_bwd_causal_workspace_size", B, L, D, K)


def conv1d_bwd_causal(x_ptr, w_ptr, bias_ptr, state_in_ptr, lengths_ptr, dy_ptr, dstate_out_ptr, dx_ptr, dw_ptr, dbias_ptr,
                      dstate_in_ptr, B, L, D, K, ldx, lddy, lddx, operand=OPERAND_BF16, act=ACT_NONE,
                      workspace_ptr=0, workspace_bytes=0, stream=0) -> None:
    """dw [D, K] and dbias [D] are fp32, whatever the operand type."""
    _check(load_library().conv1d_bwd_causal(x_ptr or None, w_ptr or None, bias_ptr or None, state_in_ptr or None, lengths_ptr or None,
                                            dy_ptr or None, dstate_out_ptr or None, dx_ptr or None, dw_ptr or None, dbias_ptr or None,
                                            dstate_in_ptr or None, B, L, D, K, ldx, lddy, lddx, operand, act,
                                            workspace_ptr or None, workspace_bytes, stream or None),
           "conv1d_bwd_causal")


def scan_states_size(B, L, D, N) -> int:
    """Bytes of the states that scan_fwd_selective leaves for scan_bwd_selective."""
    return _size("scan_states_size", B, L, D, N)


def scan_fwd_selective_workspace_size(B, L, D, N, G=1) -> int:
    return _size("scan_fwd_selective_workspace_size", B, L, D, N, G)


def scan_fwd_selective(u_ptr, delta_ptr, A_ptr, Bm_ptr, Cm_ptr, Dskip_ptr, z_ptr, delta_bias_ptr, state_in_ptr, lengths_ptr,
                       y_ptr, state_out_ptr, states_ptr, B, L, D, N, G, ldu, lddelta, ldB, ldC, ldz, ldy,
                       operand=OPERAND_BF16, flags=0, workspace_ptr=0, workspace_bytes=0, stream=0) -> None:
    """Selective state space scan of [B*L, D]; A, Dskip, delta_bias and the states are fp32."""
    _check(load_library().scan_fwd_selective(u_ptr or None, delta_ptr or None, A_ptr or None, Bm_ptr or None, Cm_ptr or None,
                                             Dskip_ptr or None, z_ptr or None, delta_bias_ptr or None, state_in_ptr or None,
                                             lengths_ptr or None, y_ptr or None, state_out_ptr or None, states_ptr or None,
                                             B, L, D, N, G, ldu, lddelta, ldB, ldC, ldz, ldy, operand, flags,
                                             workspace_ptr or None, workspace_bytes, stream or None),
           "scan_fwd_selective")


def scan_step_selective(u_ptr, delta_ptr, A_ptr, Bm_ptr, Cm_ptr, Dskip_ptr, z_ptr, delta_bias_ptr, state_in_ptr, y_ptr,
                        state_out_ptr, B, D, N, G, ldu, lddelta, ldB, ldC, ldz, ldy, operand=OPERAND_BF16, flags=0, stream=0) -> None:
    """One token of every sequence; the two states [B, D, N] may be one buffer."""
    _check(load_library().scan_step_selective(u_ptr or None, delta_ptr or None, A_ptr or None, Bm_ptr or None, Cm_ptr or None,
                                              Dskip_ptr or None, z_ptr or None, delta_bias_ptr or None, state_in_ptr or None,
                                              y_ptr or None, state_out_ptr or None, B, D, N, G, ldu, lddelta, ldB, ldC, ldz, ldy,
                                              operand, flags, stream or None),
           "scan_step_selective")


def scan_bwd_selective_workspace_size(B, L, D, N, G=1) -> int:
    return _size("scan_bwd_selective_workspace_size", B, L, D, N, G)


def scan_bwd_selective(u_ptr, delta_ptr, A_ptr, Bm_ptr, Cm_ptr, Dskip_ptr, z_ptr, delta_bias_ptr, lengths_ptr, states_ptr,
                       dy_ptr, dstate_out_ptr, du_ptr, ddelta_ptr, dA_ptr, dB_ptr, dC_ptr, dDskip_ptr, dz_ptr, ddelta_bias_ptr,
                       dstate_in_ptr, B, L, D, N, G, ldu, lddelta, ldB, ldC, ldz, lddy, lddu, ldddelta, lddB, lddC, lddz,
                       operand=OPERAND_BF16, flags=0, workspace_ptr=0, workspace_bytes=0, stream=0) -> None:
    """states: as scan_fwd_selective of the same inputs left them; dA, dDskip, ddelta_bias and dstate_in are fp32."""
    _check(load_library().scan_bwd_selective(u_ptr or None, delta_ptr or None, A_ptr or None, Bm_ptr or None, Cm_ptr or None,
                                             Dskip_ptr or None, z_ptr or None, delta_bias_ptr or None, lengths_ptr or None,
                                             states_ptr or None, dy_ptr or None, dstate_out_ptr or None, du_ptr or None,
                                             ddelta_ptr or None, dA_ptr or None, dB_ptr or None, dC_ptr or None, dDskip_ptr or None,
                                             dz_ptr or None, ddelta_bias_ptr or None, dstate_in_ptr or None, B, L, D, N, G,
                                             ldu, lddelta, ldB, ldC, ldz, lddy, lddu, ldddelta, lddB, lddC, lddz, operand, flags,
                                             workspace_ptr or None, workspace_bytes, stream or None),
           "scan_bwd_selective")


def norm_fwd_groups_workspace_size(N, S, C, G) -> int:
    return _size("norm_fwd_groups_workspace_size", N, S, C, G)


def norm_fwd_groups(x_ptr, gamma_ptr, beta_ptr, y_ptr, mean_ptr, rstd_ptr, N, S, C, G, ldx, ldy, eps,
                    operand=OPERAND_BF16, act=ACT_NONE, workspace_ptr=0, workspace_bytes=0, stream=0) -> None:
    """Group norm over S positions and C / G channels of [N*S, C], then the activation; gamma, beta [C] are fp32."""
    _check(load_library().norm_fwd_groups(x_ptr or None, gamma_ptr or None, beta_ptr or None, y_ptr or None, mean_ptr or None,
                                          rstd_ptr or None, N, S, C, G, ldx, ldy, eps, operand, act,
                                          workspace_ptr or None, workspace_bytes, stream or None),
           "norm_fwd_groups")


def norm_bwd_groups_workspace_size(N, S, C, G) -> int:
    return _size("norm_bwd_groups_workspace_size", N, S, C, G)


def norm_bwd_groups(x_ptr, gamma_ptr, beta_ptr, mean_ptr, rstd_ptr, dy_ptr, dx_ptr, dgamma_ptr, dbeta_ptr, N, S, C, G,
                    ldx, lddy, lddx, operand=OPERAND_BF16, act=ACT_NONE, workspace_ptr=0, workspace_bytes=0, stream=0) -> None:
    """mean, rstd [N, G] as norm_fwd_groups left them; dgamma, dbeta [C] are fp32."""
    _check(load_library().norm_bwd_groups(x_ptr or None, gamma_ptr or None, beta_ptr or None, mean_ptr or None, rstd_ptr or None,
                                          dy_ptr or None, dx_ptr or None, dgamma_ptr or None, dbeta_ptr or None, N, S, C, G,
                                          ldx, lddy, lddx, operand, act, workspace_ptr or None, workspace_bytes, stream or None),
           "norm_bwd_groups")


# ---- gated delta rule and RMS norm (recurrent_b200.h).  Pointers that are optional there may be 0.

def delta_states_size(B, L, Hk, H, K, V, operand=OPERAND_BF16) -> int:
    """Bytes of the states that delta_fwd_gated leaves for delta_bwd_gated."""
    return _size("delta_states_size", B, L, Hk, H, K, V, operand)


def delta_fwd_gated_workspace_size(B, L, Hk, H, K, V, operand=OPERAND_BF16) -> int:
    return _size("delta_fwd_gated_workspace_size", B, L, Hk, H, K, V, operand)


def delta_fwd_gated(q_ptr, k_ptr, v_ptr, g_ptr, beta_ptr, state_in_ptr, lengths_ptr, o_ptr, state_out_ptr, states_ptr, B, L, Hk, H, K, V,
                    ldq, ldk, ldv, ldg, ldbeta, ldo, scale, operand=OPERAND_BF16, workspace_ptr=0, workspace_bytes=0, stream=0) -> None:
    """Gated delta rule over sequences; q, k [B*L, Hk*K], v, o [B*L, H*V]; g, beta [B*L, H] and the states [B, H, K, V] are fp32."""
    _check(load_library().delta_fwd_gated(q_ptr or None, k_ptr or None, v_ptr or None, g_ptr or None, beta_ptr or None, state_in_ptr or None,
                                          lengths_ptr or None, o_ptr or None, state_out_ptr or None, states_ptr or None, B, L, Hk, H, K, V,
                                          ldq, ldk, ldv, ldg, ldbeta, ldo, scale, operand, workspace_ptr or None, workspace_bytes, stream or None),
           "delta_fwd_gated")


def delta_step_gated(q_ptr, k_ptr, v_ptr, g_ptr, beta_ptr, state_in_ptr, o_ptr, state_out_ptr, B, Hk, H, K, V, ldq, ldk, ldv, ldg, ldbeta, ldo,
                     scale, operand=OPERAND_BF16, stream=0) -> None:
    """One token of every sequence; the two states [B, H, K, V] may be one buffer."""
    _check(load_library().delta_step_gated(q_ptr or None, k_ptr or None, v_ptr or None, g_ptr or None, beta_ptr or None, state_in_ptr or None,
                                           o_ptr or None, state_out_ptr or None, B, Hk, H, K, V, ldq, ldk, ldv, ldg, ldbeta, ldo, scale, operand,
                                           stream or None),
           "delta_step_gated")


def delta_bwd_gated_workspace_size(B, L, Hk, H, K, V, operand=OPERAND_BF16) -> int:
    return _size("delta_bwd_gated_workspace_size", B, L, Hk, H, K, V, operand)


def delta_bwd_gated(q_ptr, k_ptr, lengths_ptr, states_ptr, dout_ptr, dstate_out_ptr, dq_ptr, dk_ptr, dv_ptr, dg_ptr, dbeta_ptr, dstate_in_ptr,
                    B, L, Hk, H, K, V, ldq, ldk, lddo, lddq, lddk, lddv, lddg, lddbeta, scale, operand=OPERAND_BF16,
                    workspace_ptr=0, workspace_bytes=0, stream=0) -> None:
    """states: as delta_fwd_gated of the same inputs left them; dg, dbeta and dstate_in are fp32."""
    _check(load_library().delta_bwd_gated(q_ptr or None, k_ptr or None, lengths_ptr or None, states_ptr or None, dout_ptr or None,
                                          dstate_out_ptr or None, dq_ptr or None, dk_ptr or None, dv_ptr or None, dg_ptr or None,
                                          dbeta_ptr or None, dstate_in_ptr or None, B, L, Hk, H, K, V, ldq, ldk, lddo, lddq, lddk, lddv, lddg, lddbeta,
                                          scale, operand, workspace_ptr or None, workspace_bytes, stream or None),
           "delta_bwd_gated")


def norm_fwd_rms(x_ptr, residual_ptr, z_ptr, gamma_ptr, y_ptr, h_ptr, y8_ptr, scales_ptr, rstd_ptr, M, C, G, block, ldx, ldr, ldz, ldy, ldh, ld8,
                 eps, operand=OPERAND_BF16, stream=0) -> None:
    """RMS norm of [M, C] in G groups, with the residual's addition, a gate and an output in 8 bits; gamma [C / G], scales and rstd are fp32."""
    _check(load_library().norm_fwd_rms(x_ptr or None, residual_ptr or None, z_ptr or None, gamma_ptr or None, y_ptr or None, h_ptr or None,
                                       y8_ptr or None, scales_ptr or None, rstd_ptr or None, M, C, G, block, ldx, ldr, ldz, ldy, ldh, ld8, eps,
                                       operand, stream or None),
           "norm_fwd_rms")


def norm_bwd_rms_workspace_size(M, C, G=1) -> int:
    return _size("norm_bwd_rms_workspace_size", M, C, G)


def norm_bwd_rms(h_ptr, z_ptr, gamma_ptr, rstd_ptr, dy_ptr, dh_ptr, dx_ptr, dz_ptr, dgamma_ptr, M, C, G, ldh, ldz, lddy, lddh, lddx, lddz,
                 operand=OPERAND_BF16, workspace_ptr=0, workspace_bytes=0, stream=0) -> None:
    """h, rstd as norm_fwd_rms left them; dgamma [C / G] is fp32."""
    _check(load_library().norm_bwd_rms(h_ptr or None, z_ptr or None, gamma_ptr or None, rstd_ptr or None, dy_ptr or None, dh_ptr or None,
                                       dx_ptr or None, dz_ptr or None, dgamma_ptr or None, M, C, G, ldh, ldz, lddy, lddh, lddx, lddz, operand,
                                       workspace_ptr or None, workspace_bytes, stream or None),
           "norm_bwd_rms")
