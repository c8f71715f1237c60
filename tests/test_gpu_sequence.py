"""The operators along a sequence against plain 64-bit forms: every type, sizes off every tile, row distances and offsets that rule the wide
loads out, padded batches, states handed on, calls in place, captured and on other streams, tensors beyond 32-bit offsets."""
import pytest
import torch

import sequence_reference as ref
from sequence_reference import TYPES, check

pytestmark = pytest.mark.gpu
F = torch.float64
SENTINEL = 77.0


@pytest.fixture(scope="module")
def lib():
    import paper_1705_10591_b200 as lib
    return lib


class Rows:
    """A tensor of rows inside a larger buffer: `ld` elements apart, `offset` elements into it, with rows before and behind that nobody may touch."""

    def __init__(self, shape, dtype, pad=0, offset=0, values=None):
        self.shape, width, rows = shape, shape[-1], 1
        for n in shape[:-1]:
            rows *= n
        self.ld, self.offset, self.width, self.rows = width + pad, offset, width, rows
        self.buf = torch.full((max(64, 2 * self.ld) * 2 + offset + rows * self.ld,), SENTINEL, dtype=dtype, device="cuda")
        self.lead = max(64, 2 * self.ld) // 8 * 8
        if values is not None:
            self.view().copy_(values.reshape(rows, width))

    def view(self):
        return self.buf[self.lead + self.offset:].as_strided((self.rows, self.width), (self.ld, 1))

    @property
    def ptr(self):
        return self.buf.data_ptr() + (self.lead + self.offset) * self.buf.element_size()

    def result(self):
        """The values, after a check that nothing around them was written."""
        out = self.view().clone()
        self.view().fill_(SENTINEL)
        assert (self.buf == SENTINEL).all(), "written outside the tensor"
        self.view().copy_(out)
        return out.reshape(self.shape)


def draw(seed, *shape, scale=1.0, shift=0.0, dtype=torch.float32):
    """Values of `dtype`, in 64 bits: what the kernel and the reference both see."""
    gen = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=gen) * scale + shift).to(dtype).to(F)


def cuda(v, dtype=torch.float32):
    return v.to(dtype).cuda()


def stream():
    return torch.cuda.current_stream().cuda_stream


def operand(lib, name):
    return {"bf16": lib.OPERAND_BF16, "fp16": lib.OPERAND_FP16, "fp32": lib.OPERAND_FP32}[name]


def activation(lib, name):
    return {"none": lib.ACT_NONE, "relu": lib.ACT_RELU, "silu": lib.ACT_SILU, "gelu": lib.ACT_GELU}[name]


def ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def mask_rows(v, lengths, value):
    v = v.clone()
    for b, n in enumerate(lengths):
        v[b, n:] = value
    return v


def workspace(n):
    return torch.full((max(n, 16),), 0xA5, dtype=torch.uint8, device="cuda")


# ------------------------------------------------------------------------------------------------------------ convolution

CONV = [  # type, B, L, D, K, activation, lengths, pad, offset
    ("bf16", 2, 1, 64, 4, "silu", None, 0, 0),
    ("bf16", 3, 37, 72, 4, "silu", [37, 0, 11], 8, 8),
    ("fp16", 2, 70, 33, 3, "none", [1, 70], 0, 0),
    ("fp32", 2, 19, 12, 8, "silu", [2, 19], 4, 4),
    ("fp32", 1, 129, 5, 2, "gelu", None, 3, 1),
    ("bf16", 1, 9, 1, 1, "relu", None, 0, 0),
    ("fp32", 4, 40, 260, 4, "silu", [40, 39, 33, 3], 0, 0),
    ("bf16", 2, 65, 520, 5, "gelu", None, 0, 4),
    ("fp16", 3, 33, 24, 6, "silu", [-4, 33, 99], 0, 0),
    ("fp32", 2, 64, 8, 7, "none", [5, 6], 0, 0),
]


def conv_case(seed, type, B, L, D, K, lengths):
    t = TYPES[type]
    n = [L] * B if lengths is None else [min(max(v, 0), L) for v in lengths]
    x, w, bias = draw(seed, B, L, D, dtype=t), draw(seed + 1, D, K, scale=0.6, dtype=t), draw(seed + 2, D, scale=0.3, dtype=t)
    return t, n, x, w, bias, draw(seed + 3, B, K - 1, D, dtype=t)


@pytest.mark.parametrize("with_state", [True, False])
@pytest.mark.parametrize("case", CONV, ids=lambda c: f"{c[0]}-{'x'.join(map(str, c[1:5]))}-{c[5]}")
def test_convolution(lib, case, with_state):
    type, B, L, D, K, act, lengths, pad, offset = case
    t, n, x, w, bias, state = conv_case(100, type, B, L, D, K, lengths)
    if not with_state:
        state = torch.zeros_like(state)
    xr = Rows((B, L, D), t, pad, offset, mask_rows(x, n, float("nan")))
    yr, ends = Rows((B, L, D), t, pad, offset), Rows((B, K - 1, D), t)
    lengths_dev = None if lengths is None else ints(lengths)
    wd, bd, sd = cuda(w, t), cuda(bias, t), cuda(state, t)
    lib.conv1d_fwd_causal(xr.ptr, wd.data_ptr(), bd.data_ptr(), sd.data_ptr() if with_state else 0, 0 if lengths is None else lengths_dev.data_ptr(),
                          yr.ptr, ends.ptr, B, L, D, K, xr.ld, yr.ld, operand(lib, type), activation(lib, act), stream())
    y, size, last = ref.conv_fwd(x, w, bias, state, n, act)
    got = yr.result()
    check(got, y, size, 2 * K + 20, "y")           # K products and sums, the activation's handful, its slope up to 1.13
    assert (got.double().cpu()[y == 0] == 0).all()
    assert torch.equal(ends.result().double().cpu(), last)

    # backward
    dy, dends = draw(110, B, L, D, dtype=t), draw(111, B, K - 1, D, dtype=t)
    gr, dxr, dsr = Rows((B, L, D), t, pad, offset, mask_rows(dy, n, float("nan"))), Rows((B, L, D), t, pad, offset), Rows((B, K - 1, D), t)
    dwr, dbr, de = Rows((D, K), torch.float32), Rows((D,), torch.float32), cuda(dends, t)
    nbytes = lib.conv1d_bwd_causal_workspace_size(B, L, D, K)
    ws = workspace(nbytes)
    for _ in range(2):
        lib.conv1d_bwd_causal(xr.ptr, wd.data_ptr(), bd.data_ptr(), sd.data_ptr() if with_state else 0, 0 if lengths is None else lengths_dev.data_ptr(),
                              gr.ptr, de.data_ptr() if with_state else 0, dxr.ptr, dwr.ptr, dbr.ptr, dsr.ptr if with_state else 0,
                              B, L, D, K, xr.ld, gr.ld, dxr.ld, operand(lib, type), activation(lib, act), ws.data_ptr(), nbytes, stream())
    dx, dw, db, dst = ref.conv_bwd(x, w, bias, state, n, act, dy, dends if with_state else torch.zeros_like(dends))
    check(dxr.result(), *dx, 4 * K + 40, "dx")
    rows = B * L                                    # additions on the way to a sum over all rows, in whatever order
    check(dwr.result(), *dw, 2 * K + 40 + rows, "dw")
    check(dbr.result(), *db, 2 * K + 40 + rows, "dbias")
    if with_state:
        check(dsr.result(), *dst, 4 * K + 40, "dstate")


@pytest.mark.parametrize("type, B, D, K", [("bf16", 5, 72, 4), ("fp16", 1, 7, 3), ("fp32", 3, 20, 8), ("bf16", 2, 16, 1)])
def test_convolution_token_by_token_is_the_prompt(lib, type, B, D, K):
    """Tokens one at a time, the state updated in place, give the bits of the whole sequence; so do two pieces of it."""
    L = 11
    t, n, x, w, bias, state = conv_case(120, type, B, L, D, K, None)
    xd, wd, bd, sd = cuda(x, t), cuda(w, t), cuda(bias, t), cuda(state, t)
    whole, ends = torch.empty_like(xd), torch.empty_like(sd)
    args = (operand(lib, type), lib.ACT_SILU, stream())
    lib.conv1d_fwd_causal(xd.data_ptr(), wd.data_ptr(), bd.data_ptr(), sd.data_ptr(), 0, whole.data_ptr(), ends.data_ptr(), B, L, D, K, D, D, *args)
    st, y = sd.clone(), torch.empty_like(xd)
    for i in range(L):                               # the tokens lie L * D apart
        lib.conv1d_step_causal(xd[:, i].data_ptr(), wd.data_ptr(), bd.data_ptr(), st.data_ptr(), y[:, i].data_ptr(), st.data_ptr(), B, D, K, L * D, L * D, *args)
    assert torch.equal(y, whole) and torch.equal(st, ends)
    st, cut = sd.clone(), 4
    parts = []
    for piece in (xd[:, :cut].contiguous(), xd[:, cut:].contiguous()):
        out = torch.empty_like(piece)
        lib.conv1d_fwd_causal(piece.data_ptr(), wd.data_ptr(), bd.data_ptr(), st.data_ptr(), 0, out.data_ptr(), st.data_ptr(), B, piece.shape[1], D, K, D, D, *args)
        parts.append(out)
    assert torch.equal(torch.cat(parts, 1), whole) and torch.equal(st, ends)


# ------------------------------------------------------------------------------------------------------------------- scan

SCAN = [  # type, B, L, D, N, G, softplus, z, skip, bias, lengths, pad, offset
    ("fp32", 2, 1, 8, 16, 1, True, True, True, True, None, 0, 0),
    ("fp32", 2, 45, 12, 16, 1, True, True, True, True, [45, 17], 4, 4),
    ("bf16", 3, 50, 64, 16, 2, True, True, True, True, [0, 50, 33], 8, 8),
    ("fp16", 1, 33, 36, 8, 1, True, False, True, False, None, 0, 0),
    ("fp32", 1, 40, 7, 5, 1, False, True, False, True, None, 1, 1),
    ("bf16", 2, 17, 150, 4, 3, True, True, True, True, [16, 1], 2, 2),
    ("fp32", 2, 70, 10, 20, 2, True, True, True, True, [-3, 200], 0, 0),
    ("fp32", 1, 35, 9, 64, 1, True, True, True, True, None, 0, 0),
    ("bf16", 1, 34, 12, 128, 1, True, False, False, True, None, 0, 0),
    ("fp32", 2, 48, 6, 1, 6, True, True, True, True, [48, 32], 0, 0),
    ("fp16", 1, 64, 300, 16, 1, True, True, True, True, None, 0, 4),
    ("fp32", 1, 31, 129, 3, 1, True, True, True, True, None, 0, 0),
    ("fp32", 1, 90, 4, 100, 1, True, True, True, True, [89], 0, 0),
]


class ScanCase:
    def __init__(self, lib, case, seed=200, with_state=True):
        (self.type, self.B, self.L, self.D, self.N, self.G, self.soft, gated, skipped, biased, lengths, pad, offset) = case
        B, L, D, N, G = self.B, self.L, self.D, self.N, self.G
        self.lib, t = lib, TYPES[self.type]
        self.t, self.pad, self.offset, self.with_state = t, pad, offset, with_state
        self.n = [L] * B if lengths is None else [min(max(v, 0), L) for v in lengths]
        self.lengths = None if lengths is None else ints(lengths)
        self.u, self.z = draw(seed, B, L, D, dtype=t), draw(seed + 1, B, L, D, dtype=t) if gated else None
        if self.soft:
            self.delta = draw(seed + 2, B, L, D, scale=0.7, shift=0.0 if biased else -2.0, dtype=t)
        else:
            self.delta = draw(seed + 2, B, L, D, scale=0.2, shift=0.0, dtype=t).abs()
        self.bias = draw(seed + 3, D, scale=0.3, shift=-2.0 if self.soft else 0.3).abs() * (-1 if self.soft else 1) if biased else None
        self.A = -torch.exp(draw(seed + 4, D, N, scale=0.7)).float().to(F)
        self.Bm, self.Cm = draw(seed + 5, B, L, G, N, dtype=t), draw(seed + 6, B, L, G, N, dtype=t)
        self.skip = draw(seed + 7, D) if skipped else None
        self.state = draw(seed + 8, B, D, N) if with_state else torch.zeros(B, D, N, dtype=F)
        nan = float("nan")
        rows = lambda v: Rows(tuple(v.shape[:2]) + (v[0, 0].numel(),), t, pad, offset, mask_rows(v, self.n, nan))  # noqa: E731
        self.ur, self.dr, self.br, self.cr = rows(self.u), rows(self.delta), rows(self.Bm), rows(self.Cm)
        self.zr = rows(self.z) if gated else None
        f32 = lambda v: None if v is None else cuda(v)  # noqa: E731
        self.Ad, self.kd, self.bd, self.sd = f32(self.A), f32(self.skip), f32(self.bias), f32(self.state)
        self.zero = torch.zeros(D, dtype=F)
        # roundings on the way from a state to the next: the exponential (2 ulp of 2^-23, its argument in the size), two products, a sum, the step
        # (8); over the states and channels of a sum; a dozen each for softplus, gate and outputs
        self.roundings = 16 * L + N + 120

    def p(self, v):
        return 0 if v is None else v.ptr if isinstance(v, Rows) else v.data_ptr()

    def inputs(self):
        return [self.p(v) for v in (self.ur, self.dr, self.Ad, self.br, self.cr, self.kd, self.zr, self.bd)]

    def flags(self):
        return self.lib.FLAG_SCAN_SOFTPLUS if self.soft else 0

    def forward(self, state_out=None, states=None, state_in=None, s=None):
        lib, B, L, D, N, G = self.lib, self.B, self.L, self.D, self.N, self.G
        y = Rows((B, L, D), self.t, self.pad, self.offset)
        nbytes = lib.scan_fwd_selective_workspace_size(B, L, D, N, G)
        ws = workspace(nbytes)
        state_in = state_in if state_in is not None else self.sd if self.with_state else None
        lib.scan_fwd_selective(*self.inputs(), self.p(state_in), self.p(self.lengths), y.ptr, self.p(state_out), self.p(states), B, L, D, N, G,
                               self.ur.ld, self.dr.ld, self.br.ld, self.cr.ld, self.zr.ld if self.zr else D, y.ld, operand(lib, self.type), self.flags(),
                               ws.data_ptr() if nbytes else 0, nbytes, stream() if s is None else s)
        return y

    def reference(self):
        zero = self.zero
        return (self.u, self.delta, self.A, self.Bm, self.Cm, zero if self.skip is None else self.skip, self.z, zero if self.bias is None else self.bias,
                self.state, self.n, self.soft)


@pytest.fixture(params=["whole", "segments", "default"])
def cut(request, monkeypatch):
    """Sequences walked whole, and cut into segments that are joined; one and several channel sets of a block; and as the sizes decide."""
    if request.param == "default":
        pass
    elif request.param == "segments":
        monkeypatch.setenv("CONV2D_B200_SCAN_SEGS", "3")
        monkeypatch.setenv("CONV2D_B200_SCAN_BWD_SEGS", "2")
        monkeypatch.setenv("CONV2D_B200_SCAN_SETS", "2")
    else:
        for name in ("SEGS", "BWD_SEGS", "SETS"):
            monkeypatch.setenv("CONV2D_B200_SCAN_" + name, "1")
    return request.param


@pytest.mark.parametrize("with_state", [True, False])
@pytest.mark.parametrize("case", SCAN, ids=lambda c: f"{c[0]}-{'x'.join(map(str, c[1:6]))}")
def test_scan(lib, case, cut, with_state):
    c = ScanCase(lib, case, with_state=with_state)
    B, L, D, N, G = c.B, c.L, c.D, c.N, c.G
    last = Rows((B, D, N), torch.float32)
    states = workspace(lib.scan_states_size(B, L, D, N))
    y = c.forward(last, states)
    (yr, ysize), (hr, hsize) = ref.scan_fwd(*c.reference())
    got = y.result()
    check(got, yr, ysize, c.roundings, "y")
    assert (got.double().cpu()[yr == 0] == 0).all()
    check(last.result(), hr, hsize, c.roundings, "state")

    dy, dlast = draw(230, B, L, D, dtype=c.t), draw(231, B, D, N) if with_state else torch.zeros(B, D, N, dtype=F)
    g = Rows((B, L, D), c.t, c.pad, c.offset, mask_rows(dy, c.n, float("nan")))
    like = lambda: Rows((B, L, D), c.t, c.pad, c.offset)  # noqa: E731
    du, dd, dz = like(), like(), like() if c.z is not None else None
    dB, dC = Rows((B, L, G * N), c.t, c.pad, c.offset), Rows((B, L, G * N), c.t, c.pad, c.offset)
    dA, dk, db, ds = Rows((D, N), torch.float32), Rows((D,), torch.float32), Rows((D,), torch.float32), Rows((B, D, N), torch.float32)
    dl = cuda(dlast)
    nbytes = lib.scan_bwd_selective_workspace_size(B, L, D, N, G)
    ws = workspace(nbytes)
    for _ in range(2):
        lib.scan_bwd_selective(*c.inputs(), c.p(c.lengths), states.data_ptr(), g.ptr, dl.data_ptr() if with_state else 0, du.ptr, dd.ptr, dA.ptr, dB.ptr, dC.ptr,
                               dk.ptr if c.kd is not None else 0, c.p(dz), db.ptr, ds.ptr if with_state else 0, B, L, D, N, G, c.ur.ld, c.dr.ld, c.br.ld, c.cr.ld,
                               c.zr.ld if c.zr else D, g.ld, du.ld, dd.ld, dB.ld, dC.ld, dz.ld if dz else D, operand(lib, c.type), c.flags(),
                               ws.data_ptr(), nbytes, stream())
    out = ref.scan_bwd(*c.reference(), dy, dlast)
    many = 2 * c.roundings                          # the states of the forward pass, and the walk back over them
    for name, rows, more in (("du", du, 0), ("ddelta", dd, 0), ("dz", dz, 0), ("dB", dB, D), ("dC", dC, D), ("dA", dA, B * L), ("dskip", dk, B * L),
                             ("dbias", db, B * L), ("dstate", ds, 0)):
        if rows is None or (name == "dskip" and c.kd is None) or (name == "dstate" and not with_state):
            continue
        value, size = out[name]
        check(rows.result().reshape(value.shape), value, size, many + more, name)
    for rows in (du, dd, dB, dC):
        for b, n in enumerate(c.n):
            assert (rows.result()[b, n:] == 0).all()


@pytest.mark.parametrize("whole", [True, False])
def test_padding_leaves_the_state_as_it_is(lib, monkeypatch, whole):
    """Padding does nothing to the state: walked whole, it has the bits of the shorter sequence's, and so has y.  Cut by the sizes, 200 rows are segments and 37
    rows are none: the first segment's rows have the same bits, but its share of the state, h0 exp(A sum delta) + (the segment from zero), is rounded in
    another order than a walk from h0, so the state is compared with the formula, each within the roundings of a walk."""
    if whole:
        monkeypatch.setenv("CONV2D_B200_SCAN_SEGS", "1")
    long = ScanCase(lib, ("fp32", 1, 200, 40, 16, 1, True, True, True, True, [37], 0, 0))
    st = torch.full((1, 40, 16), SENTINEL, device="cuda")
    y = long.forward(state_out=st).result()
    short = ScanCase(lib, ("fp32", 1, 200, 40, 16, 1, True, True, True, True, None, 0, 0))
    for rows in ("ur", "dr", "br", "cr", "zr"):
        getattr(short, rows).view().copy_(getattr(long, rows).view())
    short.L, st2 = 37, torch.full_like(st, SENTINEL)
    y2 = short.forward(state_out=st2).result()
    assert torch.equal(y[:, :37], y2) and (y[:, 37:] == 0).all()
    if whole:
        assert torch.equal(st, st2)
    want, size = ref.scan_fwd(*long.reference())[1]
    for got in (st, st2):
        check(got, want, size, long.roundings, "state")
    # and a sequence without a token hands the given state on
    none = ScanCase(lib, ("fp32", 2, 9, 8, 16, 1, True, True, True, True, [0, 0], 0, 0))
    st = torch.empty(2, 8, 16, device="cuda")
    none.forward(state_out=st)
    assert torch.equal(st, none.sd)


def backward(c, states, dy, dlast, optional=True):
    """du, ddelta, dA, dB, dC, dDskip, dz, ddelta_bias and dstate_in; those that a caller may leave out only where `optional`."""
    lib, B, L, D, N, G = c.lib, c.B, c.L, c.D, c.N, c.G
    new = lambda *s, t=torch.float32: Rows(s, t)  # noqa: E731
    du, dd, dz, dB, dC = new(B, L, D, t=c.t), new(B, L, D, t=c.t), new(B, L, D, t=c.t), new(B, L, G * N, t=c.t), new(B, L, G * N, t=c.t)
    dA, dk, db, ds = new(D, N), new(D), new(D), new(B, D, N)
    g, dl = cuda(dy, c.t), None if dlast is None else cuda(dlast)
    nbytes = lib.scan_bwd_selective_workspace_size(B, L, D, N, G)
    ws = workspace(nbytes)
    p = lambda v: v.ptr if optional else 0  # noqa: E731
    lib.scan_bwd_selective(*c.inputs(), c.p(c.lengths), states.data_ptr(), g.data_ptr(), c.p(dl), du.ptr, dd.ptr, dA.ptr, dB.ptr, dC.ptr,
                           p(dk) if c.kd is not None else 0, dz.ptr if c.zr else 0, p(db), p(ds), B, L, D, N, G, c.ur.ld, c.dr.ld, c.br.ld, c.cr.ld,
                           c.zr.ld if c.zr else D, D, du.ld, dd.ld, dB.ld, dC.ld, dz.ld, operand(lib, c.type), c.flags(), ws.data_ptr(), nbytes, stream())
    return [v.result() for v in (du, dd, dA, dB, dC, dk, dz, db, ds)]


def test_states_that_forget_everything(lib, cut):
    """A of -infinity is A of -1e30: a decay of zero, and of one over padding; nothing becomes NaN."""
    out = []
    for value in (float("-inf"), -1e30):
        c = ScanCase(lib, ("fp32", 2, 150, 12, 8, 1, True, True, True, True, [150, 21], 0, 0))
        c.Ad[3, 2:6] = value
        states, st = workspace(lib.scan_states_size(c.B, c.L, c.D, c.N)), torch.empty(2, 12, 8, device="cuda")
        y = c.forward(state_out=st, states=states).result()
        one = st.clone()
        yo = torch.empty(2, 12, device="cuda")
        lib.scan_step_selective(c.ur.ptr, c.dr.ptr, c.Ad.data_ptr(), c.br.ptr, c.cr.ptr, 0, 0, 0, st.data_ptr(), yo.data_ptr(), one.data_ptr(), 2, 12, 8, 1,
                                12, 12, 8, 8, 12, 12, lib.OPERAND_FP32, 1, stream())
        grads = backward(c, states, mask_rows(draw(232, 2, 150, 12), c.n, 0.0), draw(233, 2, 12, 8))
        out.append([y, st, yo, one] + grads)
    for a, b in zip(*out):
        assert torch.isfinite(a).all() and torch.equal(a, b)


def test_outputs_that_may_be_left_out(lib):
    """What is left out changes no bit of the rest; the convolution's backward pass needs no workspace without dw and dbias."""
    c = ScanCase(lib, ("bf16", 2, 50, 24, 16, 2, True, True, True, True, [50, 9], 8, 8))
    states, st = workspace(lib.scan_states_size(2, 50, 24, 16)), torch.empty(2, 24, 16, device="cuda")
    y = c.forward(state_out=st, states=states).result()
    assert torch.equal(c.forward().result(), y)
    dy, dl = mask_rows(draw(234, 2, 50, 24, dtype=c.t), c.n, 0.0), draw(235, 2, 24, 16)
    some, every = backward(c, states, dy, dl, optional=False), backward(c, states, dy, dl)
    for i, (a, b) in enumerate(zip(some, every)):
        assert (a == SENTINEL).all() if i in (5, 7, 8) else torch.equal(a, b), i
    t = torch.bfloat16
    x, w, g = cuda(draw(236, 2, 70, 24, dtype=t), t), cuda(draw(237, 24, 4, dtype=t), t), cuda(draw(238, 2, 70, 24, dtype=t), t)
    need = lib.conv1d_bwd_causal_workspace_size(2, 70, 24, 4)
    ws, out = workspace(need), []
    for dw, db in ((True, True), (True, False), (False, True), (False, False)):
        dx, wg, bg = torch.full_like(x, SENTINEL), torch.full((24, 4), SENTINEL, device="cuda"), torch.full((24,), SENTINEL, device="cuda")
        use = dw or db
        lib.conv1d_bwd_causal(x.data_ptr(), w.data_ptr(), 0, 0, 0, g.data_ptr(), 0, dx.data_ptr(), wg.data_ptr() if dw else 0, bg.data_ptr() if db else 0, 0,
                              2, 70, 24, 4, 24, 24, 24, lib.OPERAND_BF16, lib.ACT_SILU, ws.data_ptr() if use else 0, need if use else 0, stream())
        out.append((dx, wg, bg))
        for got, full, given in zip(out[-1], out[0], (True, dw, db)):
            assert torch.equal(got, full) if given else (got == SENTINEL).all()
    for S in (1, 60):
        x, g = draw(239, 3, S, 32, shift=0.3), draw(240, 3, S, 32)
        xd, gd, y, y2 = cuda(x), cuda(g), torch.empty(3, S, 32, device="cuda"), torch.empty(3, S, 32, device="cuda")
        ws = workspace(max(lib.norm_fwd_groups_workspace_size(3, S, 32, 4), lib.norm_bwd_groups_workspace_size(3, S, 32, 4)))
        m, r, dx, dx2, dg, db = (torch.full(s, SENTINEL, device="cuda") for s in ((3, 4), (3, 4), (3, S, 32), (3, S, 32), (32,), (32,)))
        f = lambda y, m, r: lib.norm_fwd_groups(xd.data_ptr(), 0, 0, y.data_ptr(), m, r, 3, S, 32, 4, 32, 32, 1e-5, lib.OPERAND_FP32, lib.ACT_GELU,  # noqa: E731
                                                ws.data_ptr(), ws.numel(), stream())
        f(y, m.data_ptr(), r.data_ptr()), f(y2, 0, 0)
        assert torch.equal(y, y2)
        b = lambda dx, dg, db: lib.norm_bwd_groups(xd.data_ptr(), 0, 0, m.data_ptr(), r.data_ptr(), gd.data_ptr(), dx.data_ptr(), dg, db, 3, S, 32, 4,  # noqa: E731
                                                   32, 32, 32, lib.OPERAND_FP32, lib.ACT_GELU, ws.data_ptr(), ws.numel(), stream())
        b(dx, dg.data_ptr(), db.data_ptr()), b(dx2, 0, 0)
        only = torch.full((32,), SENTINEL, device="cuda")
        b(dx2, 0, only.data_ptr())
        assert torch.equal(dx, dx2) and torch.equal(db, only)


@pytest.mark.parametrize("type, B, D, N, G, gated", [("bf16", 3, 24, 16, 2, True), ("fp32", 2, 7, 5, 1, True), ("fp16", 1, 12, 64, 1, False),
                                                     ("fp32", 400, 96, 32, 3, True), ("bf16", 1, 5, 128, 5, True), ("bf16", 333, 1000, 16, 1, True),
                                                     ("fp32", 1021, 160, 13, 2, False)])
def test_scan_step(lib, type, B, D, N, G, gated):
    c = ScanCase(lib, (type, B, 1, D, N, G, True, gated, True, True, None, 3, 1))
    for in_place in (False, True):
        y, st = Rows((B, 1, D), c.t, 3, 1), c.sd.clone()
        out = st if in_place else torch.full_like(st, SENTINEL)
        lib.scan_step_selective(*c.inputs(), st.data_ptr(), y.ptr, out.data_ptr(), B, D, N, G, c.ur.ld, c.dr.ld, c.br.ld, c.cr.ld, c.zr.ld if c.zr else D, y.ld,
                                operand(lib, type), c.flags(), stream())
        (yr, ysize), (hr, hsize) = ref.scan_fwd(*c.reference())
        check(y.result(), yr, ysize, c.roundings, "y")
        check(out, hr, hsize, c.roundings, "state")
        assert in_place or torch.equal(st, c.sd)


def test_scan_steps_follow_a_prompt(lib):
    """The state behind a prompt, in place, and single tokens from there: the same as the longer prompt, up to the rounding of another order."""
    c = ScanCase(lib, ("fp32", 2, 24, 20, 16, 1, True, True, True, True, None, 0, 0))
    B, L, D, N = c.B, c.L, c.D, c.N
    st = c.sd.clone()
    whole = c.forward(state_out=st, state_in=st).result()
    (yr, ysize), (hr, hsize) = ref.scan_fwd(*c.reference())
    check(st, hr, hsize, c.roundings, "state in place")
    tok, st2 = torch.empty_like(whole), c.sd.clone()
    for i in range(L):
        at = lambda r: r.view()[i:].data_ptr()  # noqa: E731
        lib.scan_step_selective(at(c.ur), at(c.dr), c.Ad.data_ptr(), at(c.br), at(c.cr), c.kd.data_ptr(), at(c.zr), c.bd.data_ptr(), st2.data_ptr(),
                                tok[:, i].data_ptr(), st2.data_ptr(), B, D, N, 1, L * D, L * D, L * N, L * N, L * D, L * D, lib.OPERAND_FP32, c.flags(), stream())
    check(tok, yr, ysize, c.roundings, "tokens")
    check(st2, hr, hsize, c.roundings, "state after tokens")


# ------------------------------------------------------------------------------------------------------------- group norm

NORM = [  # type, N, S, C, G, activation, shift of the mean, pad, offset
    ("fp32", 3, 1, 32, 4, "silu", 0.5, 0, 0),
    ("bf16", 70, 1, 96, 3, "none", 0.5, 8, 8),
    ("fp16", 5, 1, 24, 24, "none", 0.0, 0, 0),
    ("bf16", 9, 1, 4096, 1, "gelu", 0.0, 0, 0),
    ("fp32", 4, 1, 700, 2, "silu", 0.0, 1, 1),
    ("fp32", 2, 1, 20000, 1, "silu", 0.0, 0, 0),
    ("bf16", 2, 49, 64, 8, "silu", 1.0, 0, 0),
    ("fp16", 3, 200, 40, 4, "gelu", -2.0, 3, 1),
    ("fp32", 1, 1000, 36, 9, "relu", 0.5, 4, 4),
    ("fp32", 2, 333, 300, 30, "silu", 0.0, 0, 0),
    ("bf16", 1, 4000, 512, 2, "silu", 0.3, 0, 0),
    ("fp32", 1, 30000, 24, 1, "silu", 0.0, 0, 0),
    ("bf16", 2, 3, 2304, 1, "none", 0.0, 0, 0),
    ("fp32", 1, 50, 16, 2, "none", 1000.0, 0, 0),
    ("fp32", 40, 2, 8, 8, "silu", 0.0, 0, 0),
]


@pytest.fixture(params=["default", "stream", "slab"])
def variant(request, monkeypatch):
    """Slabs on chip, streams, and whichever the sizes decide for (a slab that does not fit is a stream whatever is asked for)."""
    if request.param != "default":
        monkeypatch.setenv("CONV2D_B200_NORM_STREAM", "1" if request.param == "stream" else "-1")


@pytest.mark.parametrize("params", [True, False])
@pytest.mark.parametrize("case", NORM, ids=lambda c: f"{c[0]}-{'x'.join(map(str, c[1:5]))}-{c[5]}")
def test_norm(lib, case, params, variant):
    type, N, S, C, G, act, shift, pad, offset = case
    t, eps = TYPES[type], 1e-5
    x = draw(300, N, S, C, shift=shift, dtype=t)
    gamma, beta = (draw(301, C, scale=0.3, shift=1.0), draw(302, C, scale=0.3)) if params else (torch.ones(C, dtype=F), torch.zeros(C, dtype=F))
    xr, yr = Rows((N, S, C), t, pad, offset, x), Rows((N, S, C), t, pad, offset)
    gd, bd = cuda(gamma), cuda(beta)
    mean, rstd = Rows((N, G), torch.float32), Rows((N, G), torch.float32)
    nbytes = lib.norm_fwd_groups_workspace_size(N, S, C, G)
    ws = workspace(nbytes)
    lib.norm_fwd_groups(xr.ptr, gd.data_ptr() if params else 0, bd.data_ptr() if params else 0, yr.ptr, mean.ptr, rstd.ptr, N, S, C, G, xr.ld, yr.ld, eps,
                        operand(lib, type), activation(lib, act), ws.data_ptr(), nbytes, stream())
    (y, ysize), (m, msize), (r, rsize), (_, _, v) = ref.norm_fwd(x, gamma, beta, G, eps, act)
    # a thread's sums are chains of up to this many additions, the rest are trees
    chain = 64 + min(2048, S * C // G)
    check(yr.result(), y, ysize, chain, "y")
    check(mean.result(), m, msize, chain, "mean")
    check(rstd.result(), r, rsize, chain, "rstd")

    dy = draw(303, N, S, C, dtype=t)
    gr, dxr = Rows((N, S, C), t, pad, offset, dy), Rows((N, S, C), t, pad, offset)
    dg, db = Rows((C,), torch.float32), Rows((C,), torch.float32)
    nbytes = lib.norm_bwd_groups_workspace_size(N, S, C, G)
    ws = workspace(nbytes)
    for _ in range(2):
        lib.norm_bwd_groups(xr.ptr, gd.data_ptr() if params else 0, bd.data_ptr() if params else 0, mean.ptr, rstd.ptr, gr.ptr, dxr.ptr, dg.ptr, db.ptr,
                            N, S, C, G, xr.ld, gr.ld, dxr.ld, operand(lib, type), activation(lib, act), ws.data_ptr(), nbytes, stream())
    dx, dgamma, dbeta = ref.norm_bwd(x, gamma, beta, G, eps, act, dy)
    check(dxr.result(), *dx, 2 * chain, "dx")
    check(dg.result(), *dgamma, 2 * chain + min(N * S, 4096), "dgamma")
    check(db.result(), *dbeta, 2 * chain + min(N * S, 4096), "dbeta")


def test_norm_of_many_rows_and_wide_groups(lib):
    """More samples than a chunk, groups of several packs a lane, groups wider than a block has threads: forward against torch in 64 bits."""
    for type, N, S, C, G in (("bf16", 5000, 1, 512, 2), ("fp16", 3000, 1, 96, 32), ("fp32", 700, 1, 1024, 2), ("bf16", 3, 40, 9000, 1), ("fp32", 2, 7, 3000, 3),
                             ("bf16", 6, 700, 320, 32), ("fp16", 300, 49, 80, 8)):
        t = TYPES[type]
        x = draw(310, N, S, C, shift=0.5, dtype=t)
        xd, mean, rstd = cuda(x, t), torch.empty(N, G, device="cuda"), torch.empty(N, G, device="cuda")
        y, ws = torch.empty_like(xd), workspace(lib.norm_fwd_groups_workspace_size(N, S, C, G))
        lib.norm_fwd_groups(xd.data_ptr(), 0, 0, y.data_ptr(), mean.data_ptr(), rstd.data_ptr(), N, S, C, G, C, C, 1e-5, operand(lib, type), lib.ACT_SILU,
                            ws.data_ptr(), ws.numel(), stream())
        (want, size), (m, ms), (r, rs), _ = ref.norm_fwd(x, torch.ones(C, dtype=F), torch.zeros(C, dtype=F), G, 1e-5, "silu")
        chain = 64 + min(2048, S * C // G)
        for got, ref_, sz, what in ((y, want, size, "y"), (mean, m, ms, "mean"), (rstd, r, rs, "rstd")):
            check(got, ref_, sz, chain, (what, type, N, S, C, G))
        dy = draw(311, N, S, C, dtype=t)
        gd, dx, dg, db = cuda(dy, t), torch.empty_like(xd), torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
        ws = workspace(lib.norm_bwd_groups_workspace_size(N, S, C, G))
        lib.norm_bwd_groups(xd.data_ptr(), 0, 0, mean.data_ptr(), rstd.data_ptr(), gd.data_ptr(), dx.data_ptr(), dg.data_ptr(), db.data_ptr(), N, S, C, G, C, C, C,
                            operand(lib, type), lib.ACT_SILU, ws.data_ptr(), ws.numel(), stream())
        want = ref.norm_bwd(x, torch.ones(C, dtype=F), torch.zeros(C, dtype=F), G, 1e-5, "silu", dy)
        for got, (value, sz), what in zip((dx, dg, db), want, ("dx", "dgamma", "dbeta")):
            check(got, value, sz, 2 * chain + (0 if what == "dx" else N * S), (what, type, N, S, C, G))


def test_norm_of_constant_groups(lib):
    """A group without spread: x^ is zero, y is beta, whatever the constant."""
    for S in (1, 40):
        x = torch.full((2, S, 16), 3.25, device="cuda")
        beta, y, mean = torch.arange(16.0, device="cuda"), torch.empty_like(x), torch.empty(2, 4, device="cuda")
        ws = workspace(lib.norm_fwd_groups_workspace_size(2, S, 16, 4))
        lib.norm_fwd_groups(x.data_ptr(), 0, beta.data_ptr(), y.data_ptr(), mean.data_ptr(), 0, 2, S, 16, 4, 16, 16, 1e-5, lib.OPERAND_FP32, lib.ACT_NONE,
                            ws.data_ptr(), ws.numel(), stream())
        assert torch.equal(y, beta.expand_as(y)) and (mean == 3.25).all()


# ------------------------------------------------------------------------------------------------------- together, and how calls meet

class Block:
    """Convolution, scan and group norm in a row, forward and backward, as a layer uses them."""

    def __init__(self, lib, B=2, L=40, D=24, N=16, K=4, groups=6, seed=400):
        self.lib, self.dims = lib, (B, L, D, N, K, groups)
        d = lambda i, *s, **k: draw(seed + i, *s, **k)  # noqa: E731
        self.x, self.w, self.cb = d(0, B, L, D), d(1, D, K, scale=0.5), d(2, D, scale=0.2)
        self.delta, self.bias, self.A = d(3, B, L, D, scale=0.5), d(4, D, scale=0.3, shift=-2.0), -torch.exp(d(5, D, N, scale=0.5)).float().to(F)
        self.Bm, self.Cm, self.skip, self.z = d(6, B, L, 1, N), d(7, B, L, 1, N), d(8, D), d(9, B, L, D)
        self.gamma, self.beta, self.dy = d(10, D, scale=0.3, shift=1.0), d(11, D, scale=0.3), d(12, B, L, D)
        self.names = ("x", "w", "cb", "delta", "bias", "A", "Bm", "Cm", "skip", "z", "gamma", "beta")
        self.dev = {k: cuda(getattr(self, k)) for k in self.names + ("dy",)}
        new = lambda *s: torch.full(s, SENTINEL, device="cuda")  # noqa: E731
        self.mid = [new(B, L, D) for _ in range(3)] + [new(B * L, groups), new(B * L, groups)]
        self.grad = {k: torch.full_like(self.dev[k], SENTINEL) for k in self.names}
        self.dv, self.du = new(B, L, D), new(B, L, D)
        self.states = workspace(lib.scan_states_size(B, L, D, N))
        self.ws = workspace(max(lib.scan_fwd_selective_workspace_size(B, L, D, N), lib.scan_bwd_selective_workspace_size(B, L, D, N),
                                lib.conv1d_bwd_causal_workspace_size(B, L, D, K), lib.norm_fwd_groups_workspace_size(B * L, 1, D, groups),
                                lib.norm_bwd_groups_workspace_size(B * L, 1, D, groups)))

    def run(self, s):
        lib, (B, L, D, N, K, G) = self.lib, self.dims
        p = {k: v.data_ptr() for k, v in self.dev.items()}
        g = {k: v.data_ptr() for k, v in self.grad.items()}
        c, v, y, mean, rstd = [m.data_ptr() for m in self.mid]
        w, n, f32 = self.ws.data_ptr(), self.ws.numel(), lib.OPERAND_FP32
        lib.conv1d_fwd_causal(p["x"], p["w"], p["cb"], 0, 0, c, 0, B, L, D, K, D, D, f32, lib.ACT_SILU, s)
        lib.scan_fwd_selective(c, p["delta"], p["A"], p["Bm"], p["Cm"], p["skip"], p["z"], p["bias"], 0, 0, v, 0, self.states.data_ptr(), B, L, D, N, 1,
                               D, D, N, N, D, D, f32, 1, w, n, s)
        lib.norm_fwd_groups(v, p["gamma"], p["beta"], y, mean, rstd, B * L, 1, D, G, D, D, 1e-5, f32, lib.ACT_GELU, w, n, s)
        lib.norm_bwd_groups(v, p["gamma"], p["beta"], mean, rstd, p["dy"], self.dv.data_ptr(), g["gamma"], g["beta"], B * L, 1, D, G, D, D, D, f32,
                            lib.ACT_GELU, w, n, s)
        lib.scan_bwd_selective(c, p["delta"], p["A"], p["Bm"], p["Cm"], p["skip"], p["z"], p["bias"], 0, self.states.data_ptr(), self.dv.data_ptr(), 0,
                               self.du.data_ptr(), g["delta"], g["A"], g["Bm"], g["Cm"], g["skip"], g["z"], g["bias"], 0, B, L, D, N, 1, D, D, N, N, D, D, D, D, N, N, D,
                               f32, 1, w, n, s)
        lib.conv1d_bwd_causal(p["x"], p["w"], p["cb"], 0, 0, self.du.data_ptr(), 0, g["x"], g["w"], g["cb"], 0, B, L, D, K, D, D, D, f32, lib.ACT_SILU, w, n, s)

    def outputs(self):
        return {"y": self.mid[2], **self.grad}


def test_block_of_the_three(lib):
    b = Block(lib)
    b.run(stream())
    B, L, D, N, K, G = b.dims
    leaves = [getattr(b, k).clone().requires_grad_() for k in b.names]
    v = dict(zip(b.names, leaves))
    c, _, _ = ref.conv_fwd(v["x"], v["w"], v["cb"], torch.zeros(B, K - 1, D, dtype=F), [L] * B, "silu")
    (s, _), _ = ref.scan_fwd(c, v["delta"], v["A"], v["Bm"], v["Cm"], v["skip"], v["z"], v["bias"], torch.zeros(B, D, N, dtype=F), [L] * B, True)
    (y, _), *_ = ref.norm_fwd(s.reshape(B * L, 1, D), v["gamma"], v["beta"], G, 1e-5, "gelu")
    y = y.reshape(B, L, D)
    grads = torch.autograd.grad((y * b.dy).sum(), leaves)
    # each of the six calls is off by at most 16 L + N + 120 = 776 roundings of 2^-24 of its terms' sizes, 4.6e-5; the norm divides by
    # the spread of four values, which magnifies the error before it by the ratio of a row's largest value to its smallest spread
    spread = s.detach().reshape(B * L, G, D // G)
    ratio = float((spread.abs().amax(-1) / spread.std(-1, unbiased=False)).median())
    limit = 6 * 776 * 2.0 ** -24 * max(1.0, ratio)
    for name, want in [("y", y.detach())] + list(zip(b.names, grads)):
        got = b.outputs()[name].double().cpu().reshape(want.shape)
        off = float((got - want).norm() / want.norm())
        assert off <= limit, (name, off, limit)


def test_gradients_follow_differences_of_the_kernels(lib):
    """The library's own forward, in fp32, at two points along a direction: (loss+ - loss-) / 2h against the library's gradient."""
    b = Block(lib, seed=430)
    b.run(stream())
    grads = {k: v.clone().double() for k, v in b.grad.items()}
    h = 2.0 ** -7
    for name in ("x", "w", "delta", "A", "Bm", "Cm", "z", "gamma"):
        base = b.dev[name].clone()
        along = grads[name] / grads[name].norm()
        losses = []
        for sign in (1, -1):
            b.dev[name].copy_((base.double() + sign * h * along).float())
            b.run(stream())
            losses.append(float((b.mid[2].double() * b.dev["dy"].double()).sum()))
        b.dev[name].copy_(base)
        want = float(grads[name].norm())
        got = (losses[0] - losses[1]) / (2 * h)
        # the second-order term cancels; the third, h^2 / 6 of a third derivative along the gradient that is taken to be within 100 times the
        # slope, and the rounding of 1920 terms of size about one, each known to 776 * 2^-24, in a random direction
        assert abs(got - want) <= 100 * h * h / 6 * want + 1920 ** 0.5 * 776 * 2.0 ** -24 / h, (name, got, want)


def test_captured_calls_replay_and_share_a_workspace(lib):
    """Two graphs of calls that share one workspace, replayed in turn, give the bits of the direct calls."""
    blocks = [Block(lib, seed=440), Block(lib, L=33, D=40, N=8, groups=8, seed=460)]
    shared = workspace(max(b.ws.numel() for b in blocks))
    side = torch.cuda.Stream()
    direct, graphs = [], []
    for b in blocks:
        b.ws = shared
        with torch.cuda.stream(side):
            b.run(side.cuda_stream)
        side.synchronize()
        direct.append({k: v.clone() for k, v in b.outputs().items()})
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            b.run(torch.cuda.current_stream().cuda_stream)
        graphs.append(graph)
    for _ in range(3):
        for b in blocks:
            for v in b.outputs().values():
                v.fill_(float("nan"))
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for b, want in zip(blocks, direct):
            for k, v in b.outputs().items():
                assert torch.equal(v, want[k]), k


def test_captured_single_tokens(lib):
    """Steps in place, captured: three replays are three tokens; many sequences (several fours a block) as well as few."""
    for B, D, N in ((3, 40, 16), (1500, 256, 16)):
        w, x, y = cuda(draw(480, D, 4, scale=0.5)), cuda(draw(481, B, D)), torch.empty(B, D, device="cuda")
        c = ScanCase(lib, ("fp32", B, 1, D, N, 1, True, True, True, True, None, 0, 0))
        conv, scan = cuda(draw(482, B, 3, D)), c.sd
        begin = conv.clone(), scan.clone()

        def token(s):
            lib.conv1d_step_causal(x.data_ptr(), w.data_ptr(), 0, conv.data_ptr(), y.data_ptr(), conv.data_ptr(), B, D, 4, D, D, lib.OPERAND_FP32, lib.ACT_SILU, s)
            lib.scan_step_selective(y.data_ptr(), c.dr.ptr, c.Ad.data_ptr(), c.br.ptr, c.cr.ptr, c.kd.data_ptr(), c.zr.ptr, c.bd.data_ptr(), scan.data_ptr(),
                                    out.data_ptr(), scan.data_ptr(), B, D, N, 1, D, D, N, N, D, D, lib.OPERAND_FP32, 1, s)

        out = torch.empty(B, D, device="cuda")
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        for _ in range(3):
            token(side.cuda_stream)
        side.synchronize()
        want = out.clone(), conv.clone(), scan.clone()
        conv.copy_(begin[0]), scan.copy_(begin[1])
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            token(torch.cuda.current_stream().cuda_stream)
        for _ in range(3):
            graph.replay()
        torch.cuda.synchronize()
        for got, ref_ in zip((out, conv, scan), want):
            assert torch.equal(got, ref_)


def test_calls_on_two_streams_at_once(lib):
    blocks = [Block(lib, seed=470), Block(lib, seed=490)]
    for b in blocks:
        b.run(stream())
    torch.cuda.synchronize()
    want = [{k: v.clone() for k, v in b.outputs().items()} for b in blocks]
    streams = [torch.cuda.Stream() for _ in blocks]
    for _ in range(5):
        for b, s in zip(blocks, streams):
            b.run(s.cuda_stream)
    torch.cuda.synchronize()
    for b, w in zip(blocks, want):
        for k, v in b.outputs().items():
            assert torch.equal(v, w[k]), k


def test_masked_values_reach_only_their_own_outputs(lib):
    """An infinity or NaN in one channel of one token: other sequences and channels, and earlier tokens, are what they were."""
    B, L, D, N = 2, 40, 16, 16
    c = ScanCase(lib, ("fp32", B, L, D, N, 1, True, True, True, True, None, 0, 0))
    clean = c.forward().result()
    c.ur.view()[L + 20, 5] = float("inf")
    y = c.forward().result()
    hit = torch.zeros(B, L, D, dtype=torch.bool, device="cuda")
    hit[1, 20:, 5] = True
    assert torch.equal(y[~hit], clean[~hit]) and not torch.isfinite(y[1, 20, 5])


def test_offsets_beyond_32_bits(lib):
    """Rows so far apart that element offsets pass 2^31 and 2^32: three rows of 1.5 * 2^30 elements."""
    ld, D, L = 3 << 29, 8, 3
    big = torch.zeros((L - 1) * ld + 64, dtype=torch.bfloat16, device="cuda")
    x = draw(500, 1, L, D, dtype=torch.bfloat16)
    rows = big.as_strided((L, D), (ld, 1))
    rows.copy_(x[0])
    w, y = draw(501, D, 4, dtype=torch.bfloat16), torch.empty((L, D), dtype=torch.bfloat16, device="cuda")
    wd = cuda(w, torch.bfloat16)
    lib.conv1d_fwd_causal(big.data_ptr(), wd.data_ptr(), 0, 0, 0, y.data_ptr(), 0, 1, L, D, 4, ld, D, lib.OPERAND_BF16, lib.ACT_SILU, stream())
    want, size, _ = ref.conv_fwd(x, w, torch.zeros(D, dtype=F), torch.zeros(1, 3, D, dtype=F), [L], "silu")
    check(y, want[0], size[0], 28, "y from far rows")
    # and as the target: one step back through the same rows
    src = rows.clone()
    lib.conv1d_fwd_causal(src.data_ptr(), wd.data_ptr(), 0, 0, 0, big.data_ptr(), 0, 1, L, D, 4, D, ld, lib.OPERAND_BF16, lib.ACT_SILU, stream())
    assert torch.equal(rows, y)
    rows.copy_(x[0])
    xn, ws = torch.empty_like(y), workspace(lib.norm_fwd_groups_workspace_size(1, L, D, 2))
    lib.norm_fwd_groups(big.data_ptr(), 0, 0, xn.data_ptr(), 0, 0, 1, L, D, 2, ld, D, 1e-5, lib.OPERAND_BF16, lib.ACT_NONE, ws.data_ptr(), ws.numel(), stream())
    (want, size), *_ = ref.norm_fwd(x, torch.ones(D, dtype=F), torch.zeros(D, dtype=F), 2, 1e-5, "none")
    check(xn, want[0], size[0], 100, "norm of far rows")
    c = ScanCase(lib, ("bf16", 1, L, D, 16, 1, True, False, False, False, None, 0, 0), with_state=False)
    near = c.forward().result()
    rows.copy_(c.u[0])
    far = torch.empty_like(y)
    lib.scan_fwd_selective(big.data_ptr(), c.dr.ptr, c.Ad.data_ptr(), c.br.ptr, c.cr.ptr, 0, 0, 0, 0, 0, far.data_ptr(), 0, 0, 1, L, D, 16, 1, ld, D, 16, 16, D, D,
                           lib.OPERAND_BF16, 1, ws.data_ptr(), ws.numel(), stream())
    assert torch.equal(far, near[0])
