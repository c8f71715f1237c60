"""The operators along a sequence against 64-bit forms by whole tensors: sums over thousands of rows, and every number of channel sets of a block."""
import pytest
import torch

import sequence_sums as sums
from test_gpu_sequence import Rows, activation, cuda, ints, lib, operand, stream, workspace  # noqa: F401

pytestmark = pytest.mark.gpu


def name(c):
    return f"{c[0]}-{'x'.join(map(str, c[1:6]))}"


def compare(c, got, scales=None):
    want = c.reference()
    scales = scales(want) if scales else {}
    for k, units in c.units.items():
        sums.close(got[k].reshape(want[k].shape), want[k], units, k, scales.get(k))


@pytest.mark.parametrize("case", sums.CONV, ids=name)
def test_convolution(lib, case):  # noqa: F811
    c = sums.Conv(case)
    B, L, D, K, t = c.B, c.L, c.D, c.K, c.t
    x, w, bias, state, dy, dends, n = (*(cuda(v, t) for v in (c.x, c.w, c.bias, c.state, c.dy, c.dends)), ints(c.n))
    y, dx, ds, dw, db = Rows((B, L, D), t), Rows((B, L, D), t), Rows((B, K - 1, D), t), Rows((D, K), torch.float32), Rows((D,), torch.float32)
    need = lib.conv1d_bwd_causal_workspace_size(B, L, D, K)
    ws, args = workspace(need), (operand(lib, c.type), activation(lib, c.act))
    lib.conv1d_fwd_causal(x.data_ptr(), w.data_ptr(), bias.data_ptr(), state.data_ptr(), n.data_ptr(), y.ptr, 0, B, L, D, K, D, D, *args, stream())
    lib.conv1d_bwd_causal(x.data_ptr(), w.data_ptr(), bias.data_ptr(), state.data_ptr(), n.data_ptr(), dy.data_ptr(), dends.data_ptr(), dx.ptr, dw.ptr, db.ptr, ds.ptr,
                          B, L, D, K, D, D, D, *args, ws.data_ptr(), need, stream())
    compare(c, {"y": y.result(), "dx": dx.result(), "dw": dw.result(), "dbias": db.result(), "dstate": ds.result()})


def scan(lib, c):  # noqa: F811
    B, L, D, N, G, t = c.B, c.L, c.D, c.N, c.G, c.t
    u, z, delta, Bm, Cm, dy = (cuda(v, t) for v in (c.u, c.z, c.delta, c.Bm, c.Cm, c.dy))
    bias, A, skip, state, dlast = (cuda(v) for v in (c.bias, c.A, c.skip, c.state, c.dlast))
    n, f32 = ints(c.n), torch.float32
    out = {"y": Rows((B, L, D), t), "state": Rows((B, D, N), f32), "du": Rows((B, L, D), t), "ddelta": Rows((B, L, D), t), "dz": Rows((B, L, D), t),
           "dB": Rows((B, L, G * N), t), "dC": Rows((B, L, G * N), t), "dA": Rows((D, N), f32), "dskip": Rows((D,), f32), "dbias": Rows((D,), f32),
           "dstate": Rows((B, D, N), f32)}
    o = {k: v.ptr for k, v in out.items()}
    states = workspace(lib.scan_states_size(B, L, D, N))
    inputs = [v.data_ptr() for v in (u, delta, A, Bm, Cm, skip, z, bias)]
    need, need_b = lib.scan_fwd_selective_workspace_size(B, L, D, N, G), lib.scan_bwd_selective_workspace_size(B, L, D, N, G)
    ws = workspace(max(need, need_b))
    lib.scan_fwd_selective(*inputs, state.data_ptr(), n.data_ptr(), o["y"], o["state"], states.data_ptr(), B, L, D, N, G, D, D, G * N, G * N, D, D,
                           operand(lib, c.type), 1, ws.data_ptr(), need, stream())
    lib.scan_bwd_selective(*inputs, n.data_ptr(), states.data_ptr(), dy.data_ptr(), dlast.data_ptr(), *(o[k] for k in (
        "du", "ddelta", "dA", "dB", "dC", "dskip", "dz", "dbias", "dstate")), B, L, D, N, G, D, D, G * N, G * N, D, D, D, D, G * N, G * N, D,
        operand(lib, c.type), 1, ws.data_ptr(), need_b, stream())
    return {k: v.result() for k, v in out.items()}


@pytest.mark.parametrize("case", sums.SCAN, ids=name)
def test_scan(lib, case):  # noqa: F811
    c = sums.Scan(case)
    compare(c, scan(lib, c))


@pytest.mark.parametrize("segs", ["1", "2"])
@pytest.mark.parametrize("case", sums.SETS, ids=name)
def test_scan_of_four_sets_a_block(lib, monkeypatch, case, segs):  # noqa: F811
    """32 channels a block, or 16 with more than 64 states, of which the last block has 1, 2 or 3 sets and one of them partly filled."""
    monkeypatch.setenv("CONV2D_B200_SCAN_BWD_SEGS", segs)
    monkeypatch.setenv("CONV2D_B200_SCAN_SETS", "4")
    c = sums.Scan(case)
    compare(c, scan(lib, c))


@pytest.mark.parametrize("B, L, D, N", [(2, 2000, 64, 64), (20, 40, 128, 64), (20, 40, 100, 128), (4, 2048, 2048, 64)])
def test_sizes_that_take_four_sets_by_themselves(lib, monkeypatch, B, L, D, N):  # noqa: F811
    """The workspace holds a partial sum of dB and dC for every block: as many as with four sets, fewer than with two."""
    sizes = [lib.scan_bwd_selective_workspace_size(B, L, D, N)]
    for n in "42":
        monkeypatch.setenv("CONV2D_B200_SCAN_SETS", n)
        sizes.append(lib.scan_bwd_selective_workspace_size(B, L, D, N))
    assert sizes[0] == sizes[1] < sizes[2]


@pytest.mark.parametrize("variant", ["0", "1", "-1"])
@pytest.mark.parametrize("case", sums.NORM, ids=name)
def test_norm(lib, monkeypatch, case, variant):  # noqa: F811
    monkeypatch.setenv("CONV2D_B200_NORM_STREAM", variant)
    c = sums.Norm(case)
    N, S, C, G, t = c.N, c.S, c.C, c.G, c.t
    x, dy, gamma, beta = cuda(c.x, t), cuda(c.dy, t), cuda(c.gamma), cuda(c.beta)
    y, dx, mean, rstd, dg, db = Rows((N, S, C), t), Rows((N, S, C), t), *(Rows(s, torch.float32) for s in ((N, G), (N, G), (C,), (C,)))
    ws = workspace(max(lib.norm_fwd_groups_workspace_size(N, S, C, G), lib.norm_bwd_groups_workspace_size(N, S, C, G)))
    args = operand(lib, c.type), activation(lib, c.act), ws.data_ptr(), ws.numel(), stream()
    lib.norm_fwd_groups(x.data_ptr(), gamma.data_ptr(), beta.data_ptr(), y.ptr, mean.ptr, rstd.ptr, N, S, C, G, C, C, c.eps, *args)
    lib.norm_bwd_groups(x.data_ptr(), gamma.data_ptr(), beta.data_ptr(), mean.ptr, rstd.ptr, dy.data_ptr(), dx.ptr, dg.ptr, db.ptr, N, S, C, G, C, C, C, *args)
    compare(c, {"y": y.result(), "mean": mean.result(), "rstd": rstd.result(), "dx": dx.result(), "dgamma": dg.result(), "dbeta": db.result()}, c.scales)
