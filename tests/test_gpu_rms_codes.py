"""RMS norm's output in 8 bits: blocks of columns with infinities and NaN, and the sum with a residual, as a layer's entry calls it."""
import pytest
import torch

import recurrent_reference as ref
from sequence_reference import TYPES, check
from test_gpu_sequence import Rows, cuda, draw, lib, operand, stream  # noqa: F401

pytestmark = pytest.mark.gpu
F = torch.float64
INF, NAN = float("inf"), float("nan")


def check_codes(y8, scales, want, size, block):
    """Codes and scales of y8 = y / s against y in 64 bits, which may hold infinities and NaN.  size: of y's terms."""
    M, C = want.shape
    n, wide = -(-C // block), min(block, C)
    blocks = lambda v: torch.nn.functional.pad(v, (0, n * wide - C)).reshape(M, n, wide)  # noqa: E731
    columns = lambda v: v.repeat_interleave(wide, 1)[:, :C]  # noqa: E731
    want = want.float().to(F)                                   # (what is beyond fp32 is infinite)
    most = blocks(want.abs()).nan_to_num(nan=0.0, posinf=INF).amax(-1)
    s = (most / 448).clamp(min=2.0 ** -126)
    scales, codes = scales.double().cpu(), y8.view(torch.float8_e4m3fn).double().cpu()
    endless = torch.isinf(s)
    assert (scales[endless] == INF).all()
    grow = blocks(torch.where(want.isfinite(), size, 0)).amax(-1) / 448
    # 50 roundings on the way to y, two of the quotient by 448
    assert ((scales - s).abs()[~endless] <= 52 * 2.0 ** -24 * torch.maximum(grow, s)[~endless]).all()
    nan = want.isnan() | want.isinf()                           # infinity over infinity has no value
    assert torch.equal(codes.isnan(), nan)
    within = columns(endless) & ~nan
    assert (codes[within] == 0).all()
    rest = ~columns(endless) & ~nan
    values, spread = (codes * columns(scales))[rest], columns(s)[rest]
    # half a step: 2^-4 of the value, 2^-10 of a scale below the smallest normal code; 60 roundings before
    assert ((values - want[rest]).abs() <= 2.0 ** -4 * want[rest].abs() * (1 + 2.0 ** -17) + 2.0 ** -10 * spread + 60 * 2.0 ** -24 * (size[rest] + 448 * spread)).all()
    return int(endless.sum()), int(within.sum()), int(nan.sum()), int(rest.sum())


@pytest.mark.parametrize("type, M, C, G, block, residual, gate", [
    # (a layer's entry: one scale for 128 columns, and for a row)
    ("bf16", 6, 512, 1, 128, True, False), ("bf16", 5, 4096, 1, 128, True, False), ("bf16", 6, 4096, 1, 4096, True, False), ("fp32", 5, 640, 1, 128, True, False),
    ("fp16", 7, 1000, 1, 128, True, False),
    # (the others)
    ("bf16", 6, 512, 1, 128, False, True), ("bf16", 7, 1024, 8, 128, False, True), ("fp32", 6, 260, 1, 260, False, True), ("fp16", 8, 77, 7, 10, False, True),
    ("fp32", 6, 96, 3, 7, True, True), ("bf16", 5, 8200, 1, 100, True, True)])
def test_blocks_with_infinities_and_nan(lib, type, M, C, G, block, residual, gate):  # noqa: F811
    t = TYPES[type]
    x, res, z = draw(1010, M, C, dtype=t), draw(1011, M, C, dtype=t), draw(1012, M, C, dtype=t)
    gamma = draw(1013, C // G, shift=1.0).float().to(F)
    if gate:                                                    # of single elements: first, last and inner ones
        z[0, 3], z[1, C - 1], z[2, C // 2], z[3, 0], z[3, 1] = INF, INF, NAN, INF, NAN
        if type != "fp16":
            x[4, 5], z[4, 5] = 30.0, torch.finfo(t).max         # finite, but not their product
        x[M - 1, 2], z[M - 1, 2] = 0, INF                       # (with a residual of zero there: 0 * infinity)
        res[M - 1, 2] = 0
    else:                                                       # of columns
        gamma[3], gamma[C // G - 1] = INF, NAN
        x[1, 3], res[1, 3] = 0, 0
    h = (x + res).float().to(t).to(F) if residual else x
    R = lambda v=None: Rows((M, C), t, 0, 0, v)  # noqa: E731
    xr, rr, zr, hr, gr = R(x), R(res), R(z), R(), cuda(gamma)
    y8, scales = torch.zeros(M, C, dtype=torch.uint8, device="cuda"), Rows((M, -(-C // block)), torch.float32)
    lib.norm_fwd_rms(xr.ptr, rr.ptr if residual else 0, zr.ptr if gate else 0, gr.data_ptr(), 0, hr.ptr if residual else 0, y8.data_ptr(), scales.ptr, 0, M, C, G, block,
                     C, C, C, 0, C, C, 1e-5, operand(lib, type), stream())
    (want, size), _ = ref.rms_fwd(h, z if gate else None, gamma, G, 1e-5)
    seen = check_codes(y8, scales.result(), want, size, block)
    assert all(seen[:3]), seen                                  # blocks with an infinity, finite numbers in them, and such as have no value


@pytest.mark.parametrize("type, M, C, block, pad", [
    ("bf16", 1300, 4096, 128, 0), ("bf16", 1201, 4096, 4096, 0), ("bf16", 6001, 512, 128, 0), ("bf16", 37, 8192, 128, 0), ("bf16", 5, 16384, 16384, 0), ("fp16", 33, 1000, 128, 8),
    ("fp16", 3001, 264, 264, 0), ("fp16", 9, 4096, 32, 0), ("fp32", 1400, 2048, 128, 0), ("fp32", 40, 2048, 1 << 30, 4), ("fp32", 7, 300, 24, 1), ("bf16", 11, 77, 10, 3)])
@pytest.mark.parametrize("place", ["h", "x", "residual"])
def test_entry_of_a_layer_in_8_bits(lib, type, M, C, block, pad, place):  # noqa: F811
    """With a residual, alone and beside an output of the type; h in a tensor of its own, in place of x, of the residual."""
    t = TYPES[type]
    x, res = draw(1020, M, C, dtype=t), draw(1021, M, C, scale=2.0, dtype=t)
    x[0], res[0] = 0, 0
    gamma, h = draw(1022, C, shift=1.0, scale=0.2).float().to(F), (x + res).float().to(t).to(F)
    (want, size), r = ref.rms_fwd(h, None, gamma, 1, 1e-5)
    gr = cuda(gamma)
    codes = []
    for both in (False, True):
        R = lambda v=None: Rows((M, C), t, pad, 0, v)  # noqa: E731
        xr, rr, hr, yr = R(x), R(res), R(), R()
        into = {"h": hr, "x": xr, "residual": rr}[place]
        y8, scales, rstd = torch.full((M, C + pad + 3), 9, dtype=torch.uint8, device="cuda"), Rows((M, -(-C // block)), torch.float32), Rows((M, 1), torch.float32)
        ld8 = C if pad == 0 else C + pad + 3
        lib.norm_fwd_rms(xr.ptr, rr.ptr, 0, gr.data_ptr(), yr.ptr if both else 0, into.ptr, y8.data_ptr(), scales.ptr, rstd.ptr if both else 0, M, C, 1, block,
                         xr.ld, rr.ld, 0, yr.ld, into.ld, ld8, 1e-5, operand(lib, type), stream())
        assert torch.equal(into.result().double().cpu(), h)
        flat = y8.reshape(-1)
        rows = flat.as_strided((M, C), (ld8, 1)).clone()
        flat.as_strided((M, C), (ld8, 1)).fill_(9)
        assert (flat == 9).all(), "written outside the codes"
        assert check_codes(rows, scales.result(), want, size, block)[:3] == (0, 0, 0)
        assert (rows[0] & 127 == 0).all() and (scales.result()[0] == 2.0 ** -126).all()
        if both:
            adds = 16 + 12
            check(yr.result(), want, size, adds + 16, "y")
            check(rstd.result(), r, r, adds + 4, "rstd")
        codes.append((rows, scales.result()))
    # two kernels: y is off by 44 roundings in each, so a code only where a border between two lies within 88 * 2^-24 of a quotient, of steps of 2^-4: in one of 10^4 at most
    a, b = (v.to(torch.int32) for v, _ in codes)
    assert ((a - b).abs() <= 1).all() and (a != b).sum() <= max(1, M * C // 10000)
