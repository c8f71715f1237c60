"""RMS norm's sums: rows of large numbers, whose squares are near the end of fp32, and the gradient of gamma, of integers so that a row that is left out or counted twice shows."""
import pytest
import torch

import recurrent_reference as ref
from sequence_reference import TYPES, check
from test_gpu_sequence import Rows, cuda, draw, lib, operand, stream, workspace  # noqa: F401

pytestmark = pytest.mark.gpu
F = torch.float64

# packs of eight, four, two and one element, of one thread and of several places of it; groups over lanes, over rows, through shared memory
SPREADS = [("bf16", 3, 4096, 1, 0, 0), ("bf16", 5, 512, 1, 0, 0), ("bf16", 4, 2048, 16, 8, 8), ("bf16", 2, 16384, 2, 0, 0), ("bf16", 3, 1084, 1, 0, 0), ("bf16", 3, 1162, 7, 0, 0),
           ("bf16", 3, 661, 1, 0, 0), ("bf16", 2, 16383, 1, 0, 1), ("fp32", 3, 4096, 1, 0, 0), ("fp32", 3, 520, 5, 0, 0), ("fp32", 2, 16384, 1, 0, 0), ("fp32", 3, 16383, 129, 1, 1),
           ("fp32", 9, 90, 5, 0, 2), ("fp32", 1, 1, 1, 0, 0), ("bf16", 21, 1792, 32, 0, 0)]
name = lambda c: "-".join(map(str, c))  # noqa: E731


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("case", SPREADS, ids=name)
def test_rows_of_large_numbers(lib, case, residual):  # noqa: F811
    """Numbers between 2^62 and 2^63: their squares, and the mean of those, are finite."""
    type, M, C, G, pad, offset = case
    t, n = TYPES[type], C // G
    x = (torch.sign(draw(1100, M, C)) * 2.0 ** 62 * (1 + torch.rand(M, C, generator=torch.Generator().manual_seed(1101), dtype=F))).to(t).to(F)
    x[0] = 2.0 ** 63
    res, gamma = torch.zeros(M, C, dtype=F), draw(1102, n, shift=1.0, scale=0.3).float().to(F)
    R = lambda v=None: Rows((M, C), t, pad, offset, v)  # noqa: E731
    xr, rr, yr, hr, gr, rstd = R(x), R(res), R(), R(), cuda(gamma), Rows((M, G), torch.float32)
    lib.norm_fwd_rms(xr.ptr, rr.ptr if residual else 0, 0, gr.data_ptr(), yr.ptr, hr.ptr if residual else 0, 0, 0, rstd.ptr, M, C, G, 0, xr.ld, rr.ld, 0, yr.ld, hr.ld, 0,
                     1e-5, operand(lib, type), stream())
    (want, size), r = ref.rms_fwd(x, None, gamma, G, 1e-5)
    adds = min(n, 16) + 12
    check(rstd.result(), r, r, adds + 4, "rstd")
    check(yr.result(), want, size, adds + 16, "y")
    if residual:
        assert torch.equal(hr.result().double().cpu(), x)


@pytest.mark.parametrize("type", ["bf16", "fp32"])
def test_rows_beyond_the_range(lib, type):  # noqa: F811
    """Numbers whose squares are infinite: their row becomes zeros, forward and backward; the others are as ever."""
    t, M, C = TYPES[type], 4, 512
    x, dy = draw(1105, M, C, dtype=t), draw(1106, M, C, dtype=t)
    x[1] = 2.0 ** 64
    R = lambda v=None: Rows((M, C), t, 0, 0, v)  # noqa: E731
    xr, dyr, yr, dxr, rstd = R(x), R(dy), R(), R(), Rows((M, 1), torch.float32)
    lib.norm_fwd_rms(xr.ptr, 0, 0, 0, yr.ptr, 0, 0, 0, rstd.ptr, M, C, 1, 0, C, 0, 0, C, 0, 0, 1e-5, operand(lib, type), stream())
    lib.norm_bwd_rms(xr.ptr, 0, 0, rstd.ptr, dyr.ptr, 0, dxr.ptr, 0, 0, M, C, 1, C, 0, C, 0, C, 0, operand(lib, type), 0, 0, stream())
    y, dx = yr.result(), dxr.result()
    assert (y[1] == 0).all() and (dx[1] == 0).all() and (rstd.result()[1] == 0).all()
    one = torch.ones(C, dtype=F)
    for i in (0, 2, 3):
        (want, size), _ = ref.rms_fwd(x[i:i + 1], None, one, 1, 1e-5)
        check(y[i:i + 1], want, size, 44, "y")
        check(dx[i:i + 1], *ref.rms_bwd(x[i:i + 1], None, one, 1, 1e-5, dy[i:i + 1], None)[0], 3 * 28 + 40, "dx")


@pytest.mark.parametrize("gate", [False, True])
@pytest.mark.parametrize("case", SPREADS, ids=name)
def test_large_gradients(lib, case, gate):  # noqa: F811
    """Gradients of 2^122 of either sign, all of one in the first row: the mean of their products with the row is finite, a sum of some hundred is not."""
    type, M, C, G, pad, offset = case
    t, n = TYPES[type], C // G
    x, z = draw(1110, M, C, dtype=t), draw(1111, M, C, dtype=t)
    dy = (draw(1112, M, C, scale=2.0 ** 121)).to(t).to(F)
    x[0], dy[0], z[0] = 1.0, 2.0 ** 122, 1.0
    gamma = (1 + draw(1113, n).abs() / 8).float().to(F)
    R = lambda v=None: Rows((M, C), t, pad, offset, v)  # noqa: E731
    r = (x.reshape(M, G, n).square().mean(-1) + 1e-5).rsqrt().float()
    xr, zr, dyr, dxr, dzr, gr, rd = R(x), R(z), R(dy), R(), R(), cuda(gamma), r.cuda()
    lib.norm_bwd_rms(xr.ptr, zr.ptr if gate else 0, gr.data_ptr(), rd.data_ptr(), dyr.ptr, 0, dxr.ptr, dzr.ptr if gate else 0, 0, M, C, G, xr.ld, zr.ld, dyr.ld, 0, dxr.ld,
                     dzr.ld, operand(lib, type), 0, 0, stream())
    dx, dz, _ = ref.rms_bwd(x, z if gate else None, gamma, G, 1e-5, dy, None)
    adds = min(n, 16) + 12
    check(dxr.result(), *dx, 3 * adds + 40, "dx")
    if gate:
        check(dzr.result(), *dz, adds + 40, "dz")


GAMMA = SPREADS + [("fp16", 2, 11000, 1, 0, 0), ("bf16", 3001, 1280, 1, 0, 0), ("fp16", 6001, 520, 5, 0, 0), ("fp32", 4003, 300, 3, 1, 1), ("bf16", 5003, 264, 1, 0, 0),
                   ("fp32", 1300, 4096, 32, 0, 0), ("bf16", 1501, 8200, 1, 0, 0), ("bf16", 700, 40, 5, 0, 0), ("fp16", 16411, 24, 3, 0, 0), ("bf16", 2377, 661, 1, 0, 0),
                   ("bf16", 593, 256, 1, 0, 0), ("fp32", 2049, 7, 7, 0, 0)]


@pytest.mark.parametrize("gate", [False, True])
@pytest.mark.parametrize("case", GAMMA, ids=name)
def test_every_row_counts_once_for_gamma(lib, case, gate):  # noqa: F811
    """h of -1 and 1, rstd of one and small whole dy: every sum of the M * G terms is a whole number below 2^24, exact in any order.  With a gate, z of 64, whose silu is 64 but
    for 4 roundings: terms of 64 each; a sum of them is off by 2^-24 for each of at most 160 additions one after the other and those 4, below half a term here."""
    type, M, C, G, pad, offset = case
    t, n = TYPES[type], C // G
    assert 3 * M * G < 1 << 24
    whole = lambda seed, most: torch.randint(-most, most + 1, (M, C), generator=torch.Generator().manual_seed(seed)).to(F)  # noqa: E731
    h = 2.0 * (whole(1120, 1) > 0) - 1
    dy = whole(1121, 3) if not gate else 2.0 * (whole(1122, 1) > 0) - 1
    dh, z = whole(1123, 3), torch.full((M, C), 64.0, dtype=F)
    R = lambda v=None: Rows((M, C), t, pad, offset, v)  # noqa: E731
    hr, zr, dyr, dhr, dxr, dzr, rstd, dg = R(h), R(z), R(dy), R(dh), R(), R(), torch.ones(M, G, device="cuda"), Rows((n,), torch.float32)
    need = lib.norm_bwd_rms_workspace_size(M, C, G)
    ws = workspace(need)
    want = (dy * h).reshape(M, G, n).sum((0, 1)) * (64 if gate else 1)
    for with_dh in (False, True):
        lib.norm_bwd_rms(hr.ptr, zr.ptr if gate else 0, 0, rstd.data_ptr(), dyr.ptr, dhr.ptr if with_dh else 0, dxr.ptr, dzr.ptr if gate else 0, dg.ptr, M, C, G, hr.ld, zr.ld,
                         dyr.ld, dhr.ld, dxr.ld, dzr.ld, operand(lib, type), ws.data_ptr(), need, stream())
        got = dg.result().double().cpu()
        if gate:
            assert 164 * 2.0 ** -24 * M * G < 0.5
            assert ((got - want).abs() <= 64 * 164 * 2.0 ** -24 * M * G).all()
        else:
            assert torch.equal(got, want)
