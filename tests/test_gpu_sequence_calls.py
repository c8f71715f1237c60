"""Calls of the operators along a sequence that their headers allow and that are easily missed: row distances of tensors that are not given,
parts with fewer rows than threads."""
import pytest
import torch

import sequence_reference as ref
from sequence_reference import TYPES, check
from test_gpu_sequence import SENTINEL, Rows, ScanCase, backward, cuda, draw, lib, mask_rows, operand, stream, workspace  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("type, L, D, N", [("bf16", 100, 64, 16), ("fp32", 50, 12, 16), ("fp16", 40, 30, 5)])
@pytest.mark.parametrize("ldz", [0, 7, -5, 1 << 40])
def test_the_row_distance_of_an_absent_gate_is_not_looked_at(lib, type, L, D, N, ldz, monkeypatch):  # noqa: F811
    """Without z no address is made from ldz: whole sequences, segments, single tokens and gradients have the bits that they have with ldz = D."""
    for segs in (None, "2"):
        if segs:
            monkeypatch.setenv("CONV2D_B200_SCAN_SEGS", segs)
            monkeypatch.setenv("CONV2D_B200_SCAN_BWD_SEGS", segs)
        c = ScanCase(lib, (type, 2, L, D, N, 1, True, False, True, True, [L, 21], 0, 0))
        states = workspace(lib.scan_states_size(2, L, D, N))
        want, last = c.forward(states=states).result(), torch.empty(2, D, N, device="cuda")
        need = lib.scan_fwd_selective_workspace_size(2, L, D, N, 1)
        ws, got = workspace(need), torch.empty_like(want)
        lib.scan_fwd_selective(*c.inputs(), c.sd.data_ptr(), c.lengths.data_ptr(), got.data_ptr(), last.data_ptr(), 0, 2, L, D, N, 1, c.ur.ld, c.dr.ld,
                               c.br.ld, c.cr.ld, ldz, D, operand(lib, type), c.flags(), ws.data_ptr(), need, stream())
        assert torch.equal(got, want)
    dy = draw(600, 2, L, D, dtype=c.t)
    grads = backward(c, states, dy, None)
    need = lib.scan_bwd_selective_workspace_size(2, L, D, N, 1)
    ws, dyd = workspace(need), dy.to(c.t).cuda()
    new = lambda *s, t=torch.float32: torch.empty(s, dtype=t, device="cuda")  # noqa: E731
    out = [new(2, L, D, t=c.t), new(2, L, D, t=c.t), new(D, N), new(2, L, N, t=c.t), new(2, L, N, t=c.t), new(D), None, new(D), new(2, D, N)]
    ptr = [0 if v is None else v.data_ptr() for v in out]
    lib.scan_bwd_selective(*c.inputs(), c.lengths.data_ptr(), states.data_ptr(), dyd.data_ptr(), 0, *ptr, 2, L, D, N, 1, c.ur.ld, c.dr.ld, c.br.ld, c.cr.ld, ldz,
                           D, D, D, N, N, ldz, operand(lib, type), c.flags(), ws.data_ptr(), need, stream())
    for got, want in zip(out, grads):
        assert got is None or torch.equal(got, want.reshape(got.shape))
    # one token of either sequence, the rows L tokens apart
    tokens = []
    for z in (D, ldz):
        y, st = torch.empty(2, D, dtype=c.t, device="cuda"), torch.empty(2, D, N, device="cuda")
        lib.scan_step_selective(*c.inputs(), c.sd.data_ptr(), y.data_ptr(), st.data_ptr(), 2, D, N, 1, L * D, L * D, L * N, L * N, z, D, operand(lib, type),
                                c.flags(), stream())
        tokens.append((y, st))
    assert torch.equal(tokens[0][0], tokens[1][0]) and torch.equal(tokens[0][1], tokens[1][1])


@pytest.mark.parametrize("type, N, S, C, G", [("bf16", 1, 1, 2304, 1), ("fp32", 3, 2, 16, 2), ("fp16", 1, 17, 24, 3), ("bf16", 2, 33, 8, 1), ("fp32", 5, 3, 130, 1)])
def test_streams_of_fewer_rows_than_a_block_takes(lib, type, N, S, C, G, monkeypatch):  # noqa: F811
    """Threads without a row, in parts shorter than a block's stride, at the end of a tensor: values as by the formula, nothing outside written."""
    monkeypatch.setenv("CONV2D_B200_NORM_STREAM", "1")
    t = TYPES[type]
    x, dy = draw(610, N, S, C, shift=0.4, dtype=t), draw(611, N, S, C, dtype=t)
    one, zero = torch.ones(C, dtype=torch.float64), torch.zeros(C, dtype=torch.float64)
    xr, gr, yr, dxr = Rows((N, S, C), t, 0, 0, x), Rows((N, S, C), t, 0, 0, dy), Rows((N, S, C), t), Rows((N, S, C), t)
    mean, rstd, dg, db = Rows((N, G), torch.float32), Rows((N, G), torch.float32), Rows((C,), torch.float32), Rows((C,), torch.float32)
    ws = workspace(max(lib.norm_fwd_groups_workspace_size(N, S, C, G), lib.norm_bwd_groups_workspace_size(N, S, C, G)))
    lib.norm_fwd_groups(xr.ptr, 0, 0, yr.ptr, mean.ptr, rstd.ptr, N, S, C, G, C, C, 1e-5, operand(lib, type), lib.ACT_SILU, ws.data_ptr(), ws.numel(), stream())
    lib.norm_bwd_groups(xr.ptr, 0, 0, mean.ptr, rstd.ptr, gr.ptr, dxr.ptr, dg.ptr, db.ptr, N, S, C, G, C, C, C, operand(lib, type), lib.ACT_SILU,
                        ws.data_ptr(), ws.numel(), stream())
    (y, size), *_ = ref.norm_fwd(x, one, zero, G, 1e-5, "silu")
    dx, dgamma, dbeta = ref.norm_bwd(x, one, zero, G, 1e-5, "silu", dy)
    # a thread adds at most S * C / 256 + 8 values in a row (a part has whole rows, and at most eight elements of each are one thread's unless a row is wider
    # than the block); 40 for the trees over threads and parts and the operations of an element
    chain = S * C // 256 + 48
    check(yr.result(), y, size, chain, "y")
    check(dxr.result(), *dx, 2 * chain, "dx")
    check(dg.result(), *dgamma, 2 * chain + N * S, "dgamma")
    check(db.result(), *dbeta, 2 * chain + N * S, "dbeta")


@pytest.mark.parametrize("D", [4096, 4097])
@pytest.mark.parametrize("type", ["fp32", "bf16", "fp16"])
def test_gelu_keeps_its_digits_where_it_is_small(lib, type, D):  # noqa: F811
    """v (1 + erf(v / sqrt 2)) / 2 for v down to -12, where 1 + erf cancels, and its slope: errors relative to the value.  One tap of one and a norm with
    gamma = 0 give the activation exact arguments.
    The bound is what a complementary error function good to 4 units of 2^-23 allows, in units of 2^-24 of the value: the argument v / sqrt 2 has two roundings,
    which erfc magnifies by at most v^2 + 1 (its logarithmic slope is below 2 x^2 + 1), and there is one product: 2 (v^2 + 1) + 9 <= 12 (v^2 + 1).  The slope's
    other term, v phi(v): an exponent v^2 / 2 with one rounding, a fast exponential of it, 2 + 1.173 v^2 / 2 units of 2^-23, and four products:
    2.9 v^2 + 8 of that term.  However the library takes them, it is held to that."""
    t, f = TYPES[type], torch.float64
    v = torch.cat([torch.linspace(-12, -3, D // 2, dtype=f), torch.linspace(-3, 6, D - D // 2, dtype=f)]).to(t).to(f)
    half_erfc, phi = 0.5 * torch.erfc(-v / 2 ** 0.5), torch.exp(-0.5 * v * v) / (2 * torch.pi) ** 0.5
    y, slope = v * half_erfc, half_erfc + v * phi
    y_size, slope_size = y.abs() * (1 + v * v), (half_erfc + (v * phi).abs()) * (1 + v * v)
    x, w, one = v.to(t).cuda(), torch.ones(D, 1, dtype=t, device="cuda"), torch.ones(D, dtype=t, device="cuda")
    out, dx = torch.empty_like(x), torch.empty_like(x)
    args = operand(lib, type), lib.ACT_GELU
    lib.conv1d_fwd_causal(x.data_ptr(), w.data_ptr(), 0, 0, 0, out.data_ptr(), 0, 1, 1, D, 1, D, D, *args, stream())
    lib.conv1d_bwd_causal(x.data_ptr(), w.data_ptr(), 0, 0, 0, one.data_ptr(), 0, dx.data_ptr(), 0, 0, 0, 1, 1, D, 1, D, D, D, *args, 0, 0, stream())
    check(out, y, y_size, 12, "convolution")
    check(dx, slope, slope_size, 12, "gradient of the convolution")
    for S in (1, 3):
        ones = torch.ones(S, D, dtype=t, device="cuda")
        gamma, beta, mean, rstd, dbeta = (torch.zeros(D, device="cuda"), v.float().cuda(), torch.empty(1, device="cuda"), torch.empty(1, device="cuda"),
                                          torch.empty(D, device="cuda"))
        xs, ys, dxs = draw(620, S, D, dtype=t).to(t).cuda(), torch.empty(S, D, dtype=t, device="cuda"), torch.empty(S, D, dtype=t, device="cuda")
        ws = workspace(max(lib.norm_fwd_groups_workspace_size(1, S, D, 1), lib.norm_bwd_groups_workspace_size(1, S, D, 1)))
        lib.norm_fwd_groups(xs.data_ptr(), gamma.data_ptr(), beta.data_ptr(), ys.data_ptr(), mean.data_ptr(), rstd.data_ptr(), 1, S, D, 1, D, D, 1e-5, *args,
                            ws.data_ptr(), ws.numel(), stream())
        lib.norm_bwd_groups(xs.data_ptr(), gamma.data_ptr(), beta.data_ptr(), mean.data_ptr(), rstd.data_ptr(), ones.data_ptr(), dxs.data_ptr(), 0, dbeta.data_ptr(),
                            1, S, D, 1, D, D, D, *args, ws.data_ptr(), ws.numel(), stream())
        check(ys, y.expand(S, D), y_size.expand(S, D), 12, "norm")
        check(dbeta, S * slope, S * slope_size, 12 + S, "dbeta of the norm")


@pytest.mark.parametrize("D", [2097121, (1 << 22) - 1])
def test_gradients_of_as_many_channels_as_the_header_allows(lib, D):  # noqa: F811
    """Channels one a thread, where rows are off every boundary, up to the header's 2^22: dx, dw and dbias of two rows and two taps."""
    t, L, K = torch.bfloat16, 2, 2
    x, w, dy = (torch.empty(n, dtype=t, device="cuda").normal_(generator=torch.Generator("cuda").manual_seed(i)) for i, n in enumerate((L * D, K * D, L * D)))
    dx, dw, db = torch.empty_like(x), torch.empty(D, K, device="cuda"), torch.empty(D, device="cuda")
    need = lib.conv1d_bwd_causal_workspace_size(1, L, D, K)
    ws = workspace(need)
    lib.conv1d_bwd_causal(x.data_ptr(), w.data_ptr(), 0, 0, 0, dy.data_ptr(), 0, dx.data_ptr(), dw.data_ptr(), db.data_ptr(), 0, 1, L, D, K, D, D, D,
                          lib.OPERAND_BF16, lib.ACT_NONE, ws.data_ptr(), need, stream())
    x, w, g = x.double().reshape(L, D), w.double().reshape(D, K), dy.double().reshape(L, D)
    want = torch.stack([g[0] * w[:, 1] + g[1] * w[:, 0], g[1] * w[:, 1]])
    size = torch.stack([(g[0] * w[:, 1]).abs() + (g[1] * w[:, 0]).abs(), (g[1] * w[:, 1]).abs()])
    check(dx.reshape(L, D), want, size, 3, "dx")                                  # two products and a sum
    check(dw[:, 1], (g * x).sum(0), (g * x).abs().sum(0), 8, "dw of the last tap")  # and the sums over a block's threads, of which two have rows
    check(dw[:, 0], g[1] * x[0], (g[1] * x[0]).abs(), 8, "dw of the first tap")
    check(db, g.sum(0), g.abs().sum(0), 8, "dbias")


def test_more_threads_than_32_bits_count(lib):  # noqa: F811
    """2^20 sequences of 2049 channels, one a thread: a token of each is 2.1e9 threads."""
    t, B, D = torch.bfloat16, 1 << 20, 2049
    if torch.cuda.mem_get_info()[0] < 3 * 2 * B * D:
        pytest.skip("not enough free memory")
    x = torch.empty(B, D, dtype=t, device="cuda").normal_(generator=torch.Generator("cuda").manual_seed(1))
    y, w = torch.empty_like(x), torch.full((D, 1), 0.5, dtype=t, device="cuda")
    y.fill_(SENTINEL)
    lib.conv1d_step_causal(x.data_ptr(), w.data_ptr(), 0, 0, y.data_ptr(), 0, B, D, 1, D, D, lib.OPERAND_BF16, lib.ACT_NONE, stream())
    assert all(torch.equal(a, b * 0.5) for a, b in zip(y.split(1 << 16), x.split(1 << 16)))     # (halves are exact)


@pytest.mark.parametrize("segs", ["1", "3"])
@pytest.mark.parametrize("sequences", [1, 2])
def test_sequences_of_several_launches(lib, monkeypatch, segs, sequences):  # noqa: F811
    """Calls whose grids take several launches, as more blocks than a grid holds do, have the bits of one launch."""
    case = ("bf16", 5, 100, 48, 16, 2, True, True, True, True, [100, 3, 0, 77, 41], 8, 8)
    for name in ("SEGS", "BWD_SEGS", "SETS"):
        monkeypatch.setenv("CONV2D_B200_SCAN_" + name, segs if name != "SETS" else "1")
    c = ScanCase(lib, case)
    B, L, D, N, G = c.B, c.L, c.D, c.N, c.G
    dy, dlast = mask_rows(draw(630, B, L, D, dtype=c.t), c.n, 0.0), draw(631, B, D, N)
    w, bias, ends_in = cuda(draw(632, D, 4, dtype=c.t), c.t), cuda(draw(633, D, dtype=c.t), c.t), cuda(draw(634, B, 3, D, dtype=c.t), c.t)

    def everything():
        states, last = workspace(lib.scan_states_size(B, L, D, N)), torch.empty(B, D, N, device="cuda")
        y = c.forward(state_out=last, states=states).result()
        kept = states.clone()
        conv, ends = Rows((B, L, D), c.t, 8, 8), ends_in.clone()
        lib.conv1d_fwd_causal(c.ur.ptr, w.data_ptr(), bias.data_ptr(), ends.data_ptr(), c.lengths.data_ptr(), conv.ptr, ends.data_ptr(), B, L, D, 4, c.ur.ld, conv.ld,
                              operand(lib, c.type), lib.ACT_SILU, stream())
        return [y, last, kept, conv.result(), ends] + backward(c, states, dy, dlast)

    before = lib.conv2d_launch_count()
    want = everything()
    once = lib.conv2d_launch_count() - before
    # as many blocks as `sequences` have in the scan, where a group of 24 channels is one; a sequence of the convolution has two
    monkeypatch.setenv("CONV2D_B200_SEQ_GRID", str(sequences * int(segs) * G))
    got = everything()
    assert lib.conv2d_launch_count() - before > 2 * once
    for a, b in zip(got, want):
        assert torch.equal(a, b)
