"""CPU-side checks of the operators along a sequence: they are exported and bound, and refuse what they do not take before any device work."""
import ctypes
import re
from pathlib import Path

import pytest

ROOT = Path(__file__).resolve().parent.parent
OK = 4096          # any aligned non-NULL address: checks come before it is used
NULL, SHAPE, ALIGN, WORKSPACE, UNSUPPORTED = 1, 2, 3, 4, 5


@pytest.fixture(scope="module")
def lib():
    from paper_1705_10591_b200 import build, binding
    build.build()
    return binding


def refused(lib, fn, base, cases):
    before = lib.conv2d_launch_count()
    for override, status in cases:
        with pytest.raises(lib.Conv2dError) as e:
            fn(**{**base, **override})
        assert e.value.status == status, (fn.__name__, override, e.value.status)
    assert lib.conv2d_launch_count() == before


def test_every_declared_symbol_is_exported_and_bound(lib):
    import paper_1705_10591_b200 as package
    text = re.sub(r"/\*.*?\*/", "", (ROOT / "include" / "sequence_b200.h").read_text(), flags=re.S)
    names = set(re.findall(r"\b((?:conv1d|scan|norm)_[a-z0-9_]+)\s*\(", text))
    assert len(names) == 14
    for name in names:
        assert hasattr(lib.load_library(), name) and hasattr(lib, name) and hasattr(package, name), name


CONV = dict(x_ptr=OK, w_ptr=OK, bias_ptr=OK, state_in_ptr=OK, lengths_ptr=OK, y_ptr=OK, state_out_ptr=OK, B=2, L=5, D=8, K=4, ldx=8, ldy=8,
            operand=0, act=2)


def test_convolution_refusals(lib):
    shapes = [(dict(B=0), SHAPE), (dict(L=0), SHAPE), (dict(D=-1), SHAPE), (dict(K=0), SHAPE), (dict(K=9), UNSUPPORTED), (dict(ldx=7), SHAPE),
              (dict(B=1 << 16, L=1 << 15), SHAPE), (dict(D=1 << 25, ldx=1 << 25), SHAPE), (dict(B=1, L=(1 << 30) + 1), SHAPE),
              (dict(D=(1 << 22) + 1, ldx=1 << 23), SHAPE), (dict(ldx=1 << 31), SHAPE), (dict(operand=3), UNSUPPORTED),
              (dict(operand=-1), UNSUPPORTED), (dict(act=4), UNSUPPORTED), (dict(act=-1), UNSUPPORTED)]
    refused(lib, lib.conv1d_fwd_causal, CONV, shapes + [
        (dict(x_ptr=0), NULL), (dict(w_ptr=0), NULL), (dict(y_ptr=0), NULL), (dict(ldy=7), SHAPE), (dict(x_ptr=OK + 1), ALIGN),
        (dict(state_out_ptr=OK + 1), ALIGN), (dict(lengths_ptr=OK + 2), ALIGN), (dict(operand=2, y_ptr=OK + 2), ALIGN)])
    step = {k: v for k, v in CONV.items() if k not in ("L", "lengths_ptr")}
    refused(lib, lib.conv1d_step_causal, step, [(dict(state_in_ptr=0), NULL), (dict(state_out_ptr=0), NULL), (dict(K=9), UNSUPPORTED),
                                                (dict(B=0), SHAPE), (dict(w_ptr=0), NULL)])
    need = lib.conv1d_bwd_causal_workspace_size(2, 5, 8, 4)
    assert need > 0
    bwd = dict(x_ptr=OK, w_ptr=OK, bias_ptr=OK, state_in_ptr=0, lengths_ptr=0, dy_ptr=OK, dstate_out_ptr=0, dx_ptr=OK, dw_ptr=OK, dbias_ptr=OK,
               dstate_in_ptr=0, B=2, L=5, D=8, K=4, ldx=8, lddy=8, lddx=8, operand=0, act=2, workspace_ptr=OK, workspace_bytes=need)
    refused(lib, lib.conv1d_bwd_causal, bwd, shapes + [
        (dict(dy_ptr=0), NULL), (dict(dx_ptr=0), NULL), (dict(workspace_ptr=0), NULL), (dict(workspace_bytes=need - 1), WORKSPACE),
        (dict(workspace_ptr=OK + 8), ALIGN), (dict(lddy=7), SHAPE), (dict(lddx=7), SHAPE), (dict(dw_ptr=OK + 2), ALIGN)])
    with pytest.raises(lib.Conv2dError) as e:
        lib.conv1d_bwd_causal_workspace_size(2, 5, 8, 9)
    assert e.value.status == UNSUPPORTED
    assert lib.load_library().conv1d_bwd_causal_workspace_size(2, 5, 8, 4, ctypes.POINTER(ctypes.c_size_t)()) == NULL


def test_scan_refusals(lib):
    base = dict(u_ptr=OK, delta_ptr=OK, A_ptr=OK, Bm_ptr=OK, Cm_ptr=OK, Dskip_ptr=OK, z_ptr=OK, delta_bias_ptr=OK, state_in_ptr=OK, y_ptr=OK,
                state_out_ptr=OK, B=2, D=8, N=16, G=2, ldu=8, lddelta=8, ldB=32, ldC=32, ldz=8, ldy=8, operand=0, flags=1)
    shapes = [(dict(B=0), SHAPE), (dict(N=0), SHAPE), (dict(N=129, ldB=258, ldC=258), UNSUPPORTED), (dict(G=3), SHAPE), (dict(G=0), SHAPE),
              (dict(D=0), SHAPE), (dict(ldu=7), SHAPE), (dict(lddelta=7), SHAPE), (dict(ldB=31), SHAPE), (dict(ldC=31), SHAPE), (dict(ldz=7), SHAPE),
              (dict(operand=3), UNSUPPORTED), (dict(flags=2), UNSUPPORTED), (dict(u_ptr=0), NULL), (dict(delta_ptr=0), NULL), (dict(A_ptr=0), NULL),
              (dict(Bm_ptr=0), NULL), (dict(Cm_ptr=0), NULL), (dict(A_ptr=OK + 2), ALIGN), (dict(Bm_ptr=OK + 1), ALIGN)]
    refused(lib, lib.scan_step_selective, base, shapes + [(dict(state_in_ptr=0), NULL), (dict(state_out_ptr=0), NULL), (dict(ldy=7), SHAPE),
                                                          (dict(y_ptr=0), NULL)])
    need = max(lib.scan_fwd_selective_workspace_size(2, 5, 8, 16, 2), 16)
    fwd = dict(base, L=5, lengths_ptr=0, states_ptr=OK, workspace_ptr=OK, workspace_bytes=need)
    refused(lib, lib.scan_fwd_selective, fwd, shapes + [(dict(L=0), SHAPE), (dict(y_ptr=0), NULL), (dict(ldy=7), SHAPE), (dict(states_ptr=OK + 4), ALIGN),
                                                        (dict(lengths_ptr=OK + 1), ALIGN), (dict(B=1 << 16, L=1 << 15), SHAPE)])
    need = lib.scan_bwd_selective_workspace_size(2, 5, 8, 16, 2)
    assert need > 0 and lib.scan_states_size(2, 5, 8, 16) == 2 * 8 * 16 * 4
    bwd = {k: v for k, v in fwd.items() if k not in ("state_in_ptr", "y_ptr", "state_out_ptr", "ldy")}
    bwd.update(dy_ptr=OK, dstate_out_ptr=0, du_ptr=OK, ddelta_ptr=OK, dA_ptr=OK, dB_ptr=OK, dC_ptr=OK, dDskip_ptr=OK, dz_ptr=OK, ddelta_bias_ptr=OK,
               dstate_in_ptr=0, lddy=8, lddu=8, ldddelta=8, lddB=32, lddC=32, lddz=8, workspace_bytes=need)
    refused(lib, lib.scan_bwd_selective, bwd, shapes + [
        (dict(states_ptr=0), NULL), (dict(dy_ptr=0), NULL), (dict(du_ptr=0), NULL), (dict(ddelta_ptr=0), NULL), (dict(dA_ptr=0), NULL),
        (dict(dB_ptr=0), NULL), (dict(dC_ptr=0), NULL), (dict(dz_ptr=0), NULL), (dict(z_ptr=0), NULL), (dict(Dskip_ptr=0), NULL),
        (dict(workspace_ptr=0), NULL), (dict(workspace_bytes=need - 1), WORKSPACE), (dict(lddy=7), SHAPE), (dict(lddu=7), SHAPE),
        (dict(ldddelta=7), SHAPE), (dict(lddB=31), SHAPE), (dict(lddC=31), SHAPE), (dict(lddz=7), SHAPE)])
    for query, args in ((lib.scan_states_size, (2, 0, 8, 16)), (lib.scan_fwd_selective_workspace_size, (2, 5, 8, 16, 3)),
                        (lib.scan_bwd_selective_workspace_size, (0, 5, 8, 16, 1))):
        with pytest.raises(lib.Conv2dError) as e:
            query(*args)
        assert e.value.status == SHAPE


def test_norm_refusals(lib):
    need = max(lib.norm_fwd_groups_workspace_size(2, 5, 8, 4), 16)
    fwd = dict(x_ptr=OK, gamma_ptr=OK, beta_ptr=OK, y_ptr=OK, mean_ptr=OK, rstd_ptr=OK, N=2, S=5, C=8, G=4, ldx=8, ldy=8, eps=1e-5, operand=0, act=2,
               workspace_ptr=OK, workspace_bytes=need)
    shapes = [(dict(N=0), SHAPE), (dict(S=0), SHAPE), (dict(C=0), SHAPE), (dict(G=0), SHAPE), (dict(G=3), SHAPE), (dict(ldx=7), SHAPE),
              (dict(operand=3), UNSUPPORTED), (dict(act=4), UNSUPPORTED), (dict(x_ptr=0), NULL), (dict(x_ptr=OK + 1), ALIGN),
              (dict(gamma_ptr=OK + 2), ALIGN), (dict(N=1 << 16, S=1 << 15), SHAPE)]
    refused(lib, lib.norm_fwd_groups, fwd, shapes + [(dict(y_ptr=0), NULL), (dict(ldy=7), SHAPE), (dict(eps=-1e-9), SHAPE),
                                                     (dict(eps=float("nan")), SHAPE), (dict(eps=float("inf")), SHAPE)])
    need = lib.norm_bwd_groups_workspace_size(2, 5, 8, 4)
    assert need > 0
    bwd = {k: v for k, v in fwd.items() if k not in ("y_ptr", "ldy", "eps")}
    bwd.update(dy_ptr=OK, dx_ptr=OK, dgamma_ptr=OK, dbeta_ptr=OK, lddy=8, lddx=8, workspace_bytes=need)
    refused(lib, lib.norm_bwd_groups, bwd, shapes + [
        (dict(mean_ptr=0), NULL), (dict(rstd_ptr=0), NULL), (dict(dy_ptr=0), NULL), (dict(dx_ptr=0), NULL), (dict(workspace_ptr=0), NULL),
        (dict(workspace_bytes=need - 1), WORKSPACE), (dict(lddy=7), SHAPE), (dict(lddx=7), SHAPE)])


def test_without_a_gpu_nothing_falls_back(lib):
    import torch
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    with pytest.raises(lib.Conv2dError) as e:
        lib.conv1d_fwd_causal(**CONV)
    assert e.value.status in (6, 7)


def test_workspace_sizes_do_not_wrap(lib):
    """Sizes beyond 32 bits: long sequences of many channels."""
    assert lib.scan_states_size(8, 1 << 20, 4096, 16) == 8 * (1 << 16) * 4096 * 16 * 4
    assert lib.scan_bwd_selective_workspace_size(8, 1 << 20, 4096, 16, 1) > 1 << 32
    assert lib.conv1d_bwd_causal_workspace_size(8, 1 << 20, 8192, 4) < 1 << 28
    # the largest extents there are: 2^62 bytes for the partial sums alone
    assert lib.scan_bwd_selective_workspace_size(1, 1 << 30, 1 << 22, 128, 1 << 22) > 1 << 62
    assert lib.scan_states_size(1, 1 << 30, 1 << 22, 128) == (1 << 26) * (1 << 22) * 128 * 4
    assert lib.norm_bwd_groups_workspace_size(1 << 20, 4, 4096, 32) >= (1 << 20) * 2 * 4096 * 4


def test_the_backward_scan_wants_what_its_header_says(lib):
    """Bytes of workspace and of kept states for each row and channel, of many channels: 4 with 16 states, 16 with 64, 64 with 128, and N / 4."""
    for B, L, D in ((4, 2048, 2048), (8, 1000, 4096)):
        for N, per in ((4, 4), (16, 4), (64, 16), (128, 64)):
            assert lib.scan_bwd_selective_workspace_size(B, L, D, N, 1) <= 1.03 * per * B * L * D
            assert N / 4 <= lib.scan_states_size(B, L, D, N) / (B * L * D) <= 1.01 * N / 4
