"""CPU-side checks of the gated delta rule and RMS norm: they are exported and bound, and refuse what they do not take before any device work."""
import ctypes
import re
from pathlib import Path

import pytest

from test_sequence_abi import ALIGN, NULL, OK, SHAPE, UNSUPPORTED, WORKSPACE, lib, refused  # noqa: F401

ROOT = Path(__file__).resolve().parent.parent


def test_every_declared_symbol_is_exported_and_bound(lib):  # noqa: F811
    import paper_1705_10591_b200 as package
    text = re.sub(r"/\*.*?\*/", "", (ROOT / "include" / "recurrent_b200.h").read_text(), flags=re.S)
    names = set(re.findall(r"\b((?:delta|norm)_[a-z0-9_]+)\s*\(", text))
    assert len(names) == 9
    for name in names:
        assert hasattr(lib.load_library(), name) and hasattr(lib, name) and hasattr(package, name), name


STEP = dict(q_ptr=OK, k_ptr=OK, v_ptr=OK, g_ptr=OK, beta_ptr=OK, state_in_ptr=OK, o_ptr=OK, state_out_ptr=OK, B=2, Hk=2, H=4, K=8, V=6, ldq=16, ldk=16, ldv=24,
            ldg=4, ldbeta=4, ldo=24, scale=0.5, operand=0)
SHAPES = [(dict(B=0), SHAPE), (dict(Hk=0), SHAPE), (dict(H=0), SHAPE), (dict(H=3, Hk=2), SHAPE), (dict(K=0), SHAPE), (dict(V=0), SHAPE),
          (dict(K=129, ldq=258, ldk=258), UNSUPPORTED), (dict(H=1, Hk=1, V=65537, ldv=65537, ldo=65537), UNSUPPORTED), (dict(ldq=15), SHAPE), (dict(ldk=15), SHAPE),
          (dict(ldq=1 << 31), SHAPE), (dict(operand=3), UNSUPPORTED), (dict(operand=-1), UNSUPPORTED), (dict(q_ptr=0), NULL), (dict(k_ptr=0), NULL),
          (dict(q_ptr=OK + 1), ALIGN), (dict(k_ptr=OK + 1), ALIGN), (dict(H=1 << 21, Hk=1 << 21, K=8, ldq=1 << 24, ldk=1 << 24), SHAPE)]


def test_delta_refusals(lib):  # noqa: F811
    forward = SHAPES + [(dict(v_ptr=0), NULL), (dict(g_ptr=0), NULL), (dict(beta_ptr=0), NULL), (dict(o_ptr=0), NULL), (dict(ldv=23), SHAPE), (dict(ldo=23), SHAPE),
                        (dict(ldg=3), SHAPE), (dict(ldbeta=3), SHAPE), (dict(v_ptr=OK + 1), ALIGN), (dict(g_ptr=OK + 2), ALIGN), (dict(state_in_ptr=OK + 2), ALIGN),
                        (dict(operand=2, o_ptr=OK + 2), ALIGN)]
    refused(lib, lib.delta_step_gated, STEP, forward + [(dict(state_in_ptr=0), NULL), (dict(state_out_ptr=0), NULL)])
    need = lib.delta_fwd_gated_workspace_size(2, 5, 2, 4, 8, 6)
    fwd = dict(STEP, L=5, lengths_ptr=0, states_ptr=OK, workspace_ptr=OK, workspace_bytes=need)
    refused(lib, lib.delta_fwd_gated, fwd, forward + [
        (dict(L=0), SHAPE), (dict(B=1 << 16, L=1 << 15), SHAPE), (dict(lengths_ptr=OK + 2), ALIGN), (dict(states_ptr=OK + 8), ALIGN), (dict(workspace_ptr=0), NULL),
        (dict(workspace_ptr=OK + 8), ALIGN), (dict(workspace_bytes=need - 1), WORKSPACE),
        (dict(B=1 << 20, L=1 << 10, H=1 << 7, V=1 << 8, ldv=1 << 15, ldo=1 << 15, ldg=128, ldbeta=128), SHAPE)])      # more pieces than are counted
    need = lib.delta_bwd_gated_workspace_size(2, 5, 2, 4, 8, 6)
    bwd = dict(q_ptr=OK, k_ptr=OK, lengths_ptr=0, states_ptr=OK, dout_ptr=OK, dstate_out_ptr=0, dq_ptr=OK, dk_ptr=OK, dv_ptr=OK, dg_ptr=OK, dbeta_ptr=OK,
               dstate_in_ptr=0, B=2, L=5, Hk=2, H=4, K=8, V=6, ldq=16, ldk=16, lddo=24, lddq=16, lddk=16, lddv=24, lddg=4, lddbeta=4, scale=0.5, operand=0,
               workspace_ptr=OK, workspace_bytes=need)
    shapes = [(d if "ldv" not in d else {k: v for k, v in d.items() if k not in ("ldv", "ldo")}, s) for d, s in SHAPES]
    refused(lib, lib.delta_bwd_gated, bwd, shapes + [
        (dict(L=0), SHAPE), (dict(states_ptr=0), NULL), (dict(dout_ptr=0), NULL), (dict(dq_ptr=0), NULL), (dict(dk_ptr=0), NULL), (dict(dv_ptr=0), NULL),
        (dict(dg_ptr=0), NULL), (dict(dbeta_ptr=0), NULL), (dict(lddo=23), SHAPE), (dict(lddq=15), SHAPE), (dict(lddk=15), SHAPE), (dict(lddv=23), SHAPE),
        (dict(lddg=3), SHAPE), (dict(lddbeta=3), SHAPE), (dict(states_ptr=OK + 8), ALIGN), (dict(dg_ptr=OK + 2), ALIGN), (dict(dstate_out_ptr=OK + 2), ALIGN),
        (dict(workspace_ptr=0), NULL), (dict(workspace_bytes=need - 1), WORKSPACE), (dict(workspace_ptr=OK + 4), ALIGN)])
    for query in (lib.delta_states_size, lib.delta_fwd_gated_workspace_size, lib.delta_bwd_gated_workspace_size):
        for args, status in (((0, 5, 2, 4, 8, 6, 0), SHAPE), ((2, 5, 3, 4, 8, 6, 0), SHAPE), ((2, 5, 2, 4, 129, 6, 0), UNSUPPORTED), ((2, 5, 2, 4, 8, 6, 7), UNSUPPORTED)):
            with pytest.raises(lib.Conv2dError) as e:
                query(*args)
            assert e.value.status == status
    assert lib.load_library().delta_states_size(2, 5, 2, 4, 8, 6, 0, ctypes.POINTER(ctypes.c_size_t)()) == NULL


def test_rms_refusals(lib):  # noqa: F811
    fwd = dict(x_ptr=OK, residual_ptr=OK, z_ptr=OK, gamma_ptr=OK, y_ptr=OK, h_ptr=OK, y8_ptr=OK, scales_ptr=OK, rstd_ptr=OK, M=3, C=8, G=2, block=4,
               ldx=8, ldr=8, ldz=8, ldy=8, ldh=8, ld8=8, eps=1e-6, operand=0)
    shapes = [(dict(M=0), SHAPE), (dict(C=0), SHAPE), (dict(G=0), SHAPE), (dict(G=3), SHAPE), (dict(M=(1 << 30) + 1), SHAPE),
              (dict(C=16385, G=1, ldx=20000, ldr=20000, ldz=20000, ldy=20000, ldh=20000, ld8=20000, lddy=20000, lddh=20000, lddx=20000, lddz=20000), UNSUPPORTED),
              (dict(ldz=7), SHAPE), (dict(ldh=7), SHAPE), (dict(operand=3), UNSUPPORTED), (dict(gamma_ptr=OK + 2), ALIGN), (dict(z_ptr=OK + 1), ALIGN),
              (dict(rstd_ptr=OK + 2), ALIGN)]
    own = lambda cases, base: [({k: v for k, v in d.items() if k in base}, s) for d, s in cases]  # noqa: E731
    refused(lib, lib.norm_fwd_rms, fwd, own(shapes, fwd) + [
        (dict(x_ptr=0), NULL), (dict(y_ptr=0, y8_ptr=0, scales_ptr=0), NULL), (dict(y8_ptr=0), NULL), (dict(scales_ptr=0), NULL), (dict(h_ptr=0), NULL),
        (dict(residual_ptr=0), NULL), (dict(ldx=7), SHAPE), (dict(ldr=7), SHAPE), (dict(ldy=7), SHAPE), (dict(ld8=7), SHAPE), (dict(block=0), SHAPE),
        (dict(block=-1), SHAPE), (dict(eps=-1e-9), SHAPE), (dict(eps=float("nan")), SHAPE), (dict(eps=float("inf")), SHAPE), (dict(scales_ptr=OK + 2), ALIGN)])
    need = lib.norm_bwd_rms_workspace_size(3, 8, 2)
    assert need > 0
    bwd = dict(h_ptr=OK, z_ptr=OK, gamma_ptr=OK, rstd_ptr=OK, dy_ptr=OK, dh_ptr=OK, dx_ptr=OK, dz_ptr=OK, dgamma_ptr=OK, M=3, C=8, G=2, ldh=8, ldz=8, lddy=8,
               lddh=8, lddx=8, lddz=8, operand=0, workspace_ptr=OK, workspace_bytes=need)
    refused(lib, lib.norm_bwd_rms, bwd, own(shapes, bwd) + [
        (dict(h_ptr=0), NULL), (dict(rstd_ptr=0), NULL), (dict(dy_ptr=0), NULL), (dict(dx_ptr=0), NULL), (dict(z_ptr=0), NULL), (dict(dz_ptr=0), NULL),
        (dict(workspace_ptr=0), NULL), (dict(workspace_bytes=need - 1), WORKSPACE), (dict(workspace_ptr=OK + 8), ALIGN), (dict(lddy=7), SHAPE), (dict(lddh=7), SHAPE),
        (dict(lddx=7), SHAPE), (dict(lddz=7), SHAPE), (dict(dgamma_ptr=OK + 1), ALIGN)])
    for args, status in (((0, 8, 2), SHAPE), ((3, 8, 3), SHAPE), ((3, 16385, 1), UNSUPPORTED)):
        with pytest.raises(lib.Conv2dError) as e:
            lib.norm_bwd_rms_workspace_size(*args)
        assert e.value.status == status


def test_without_a_gpu_nothing_falls_back(lib):  # noqa: F811
    import torch
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    with pytest.raises(lib.Conv2dError) as e:
        lib.delta_step_gated(**STEP)
    assert e.value.status in (6, 7)


def test_sizes_do_not_wrap(lib):  # noqa: F811
    pieces = 1 << 14
    squares, factors, state, update = 3 * 2 * 64 * 64 * 2, 5 * 64 * 4, 128 * 128 * 4, 64 * 128 * 4
    assert lib.delta_states_size(8, 1 << 20, 16, 32, 128, 128) == 8 * 32 * pieces * (squares + factors + state + update)
    assert lib.delta_fwd_gated_workspace_size(8, 1 << 20, 16, 32, 128, 128) == 8 * pieces * (32 * (squares + factors) + 16 * 2 * 64 * 128 * 2)
    assert lib.delta_bwd_gated_workspace_size(8, 1 << 20, 16, 32, 128, 128, 2) > 8 * 32 * pieces * (state + update)
    assert lib.norm_bwd_rms_workspace_size(1 << 30, 16384, 1) < 1 << 28
