"""The gated delta rule and RMS norm against plain 64-bit forms: every type, heads that share keys, sizes off every tile, row distances and offsets that rule the
wide loads out, padded batches, states handed on, calls in place, captured and on other streams, tensors beyond 32-bit offsets."""
import pytest
import torch

import recurrent_reference as ref
from sequence_reference import TYPES, check
from test_gpu_sequence import SENTINEL, Rows, cuda, draw, ints, lib, mask_rows, operand, stream, workspace  # noqa: F401

pytestmark = pytest.mark.gpu
F = torch.float64
NAN = float("nan")


class Delta:
    """Inputs of a case on both sides, and the calls on them."""

    def __init__(self, lib, type, B, L, Hk, H, K, V, lengths=None, pad=0, offset=0, state=True, seed=700, decay=0.0, scale=None):  # noqa: F811
        self.lib, self.type, self.t, self.dims = lib, type, TYPES[type], (B, L, Hk, H, K, V)
        self.n = [L] * B if lengths is None else [min(max(v, 0), L) for v in lengths]
        self.scale = K ** -0.5 if scale is None else scale
        unit = lambda x: (x / (x.norm(dim=-1, keepdim=True) + 1e-6)).to(self.t).to(F)  # noqa: E731
        self.q, self.k = unit(draw(seed, B, L, Hk, K)), unit(draw(seed + 1, B, L, Hk, K))
        self.v = draw(seed + 2, B, L, H, V, dtype=self.t)
        self.g = (-torch.nn.functional.softplus(draw(seed + 3, B, L, H) - decay)).float().to(F)
        self.beta = torch.sigmoid(draw(seed + 4, B, L, H)).float().to(F)
        self.state = draw(seed + 5, B, H, K, V) if state else torch.zeros(B, H, K, V, dtype=F)
        self.dout, self.dlast = draw(seed + 6, B, L, H, V, dtype=self.t), draw(seed + 7, B, H, K, V)
        self.has_state = state
        rows = lambda x, t, w: Rows((B, L, w), t, pad, offset, mask_rows(x.reshape(B, L, w), self.n, NAN))  # noqa: E731
        self.qr, self.kr = rows(self.q, self.t, Hk * K), rows(self.k, self.t, Hk * K)
        self.vr, self.gr, self.br = rows(self.v, self.t, H * V), rows(self.g, torch.float32, H), rows(self.beta, torch.float32, H)
        self.dr = rows(self.dout, self.t, H * V)
        self.pad, self.offset = pad, offset
        self.lengths = None if lengths is None else ints(lengths)
        self.sd, self.dld = cuda(self.state), cuda(self.dlast)
        self.kept = None

    def rows(self, width, t):
        B, L = self.dims[:2]
        return Rows((B, L, width), t, self.pad, self.offset)

    def forward(self, keep=False, o=None, last=None, state=None, ws=None, on=None):
        B, L, Hk, H, K, V = self.dims
        lib, op = self.lib, operand(self.lib, self.type)  # noqa: F811
        o = self.rows(H * V, self.t) if o is None else o
        last = Rows((B, H, K, V), torch.float32) if last is None else last
        if keep and self.kept is None:
            self.kept = workspace(lib.delta_states_size(*self.dims, op))
        need = lib.delta_fwd_gated_workspace_size(*self.dims, op)
        ws = workspace(need) if ws is None else ws
        given = self.sd.data_ptr() if state is None else state
        lib.delta_fwd_gated(self.qr.ptr, self.kr.ptr, self.vr.ptr, self.gr.ptr, self.br.ptr, given if self.has_state else 0,
                            0 if self.lengths is None else self.lengths.data_ptr(), o.ptr, last.ptr if isinstance(last, Rows) else last,
                            self.kept.data_ptr() if keep else 0, B, L, Hk, H, K, V, self.qr.ld, self.kr.ld, self.vr.ld, self.gr.ld, self.br.ld, o.ld,
                            self.scale, op, ws.data_ptr(), need, stream() if on is None else on)
        return o, last

    def backward(self, last=True, ws=None, on=None):
        B, L, Hk, H, K, V = self.dims
        lib, op = self.lib, operand(self.lib, self.type)  # noqa: F811
        out = {"dq": self.rows(Hk * K, self.t), "dk": self.rows(Hk * K, self.t), "dv": self.rows(H * V, self.t), "dg": self.rows(H, torch.float32),
               "dbeta": self.rows(H, torch.float32), "dstate": Rows((B, H, K, V), torch.float32)}
        need = lib.delta_bwd_gated_workspace_size(*self.dims, op)
        ws = workspace(need) if ws is None else ws
        lib.delta_bwd_gated(self.qr.ptr, self.kr.ptr, 0 if self.lengths is None else self.lengths.data_ptr(), self.kept.data_ptr(), self.dr.ptr,
                            self.dld.data_ptr() if last else 0, *(out[n].ptr for n in ("dq", "dk", "dv", "dg", "dbeta")), out["dstate"].ptr if self.has_state else 0,
                            B, L, Hk, H, K, V, self.qr.ld, self.kr.ld, self.dr.ld, out["dq"].ld, out["dk"].ld, out["dv"].ld, out["dg"].ld, out["dbeta"].ld,
                            self.scale, op, ws.data_ptr(), need, stream() if on is None else on)
        if not self.has_state:
            del out["dstate"]
        return out

    def wanted(self, grads=True, last=True):
        args = (self.q, self.k, self.v, self.g, self.beta, self.state, self.n, self.scale)
        return ref.delta_allowed(*args, **(dict(dout=self.dout, dlast=self.dlast if last else None) if grads else {}))

    def check(self, results, wanted):
        B, L, Hk, H, K, V = self.dims
        shapes = {"o": (B, L, H, V), "dq": (B, L, Hk, K), "dk": (B, L, Hk, K), "dv": (B, L, H, V), "dg": (B, L, H), "dbeta": (B, L, H)}
        for name, x in results.items():
            got = x.result().reshape(shapes.get(name, (B, H, K, V)))
            if name in shapes:
                for b, n in enumerate(self.n):
                    assert (got[b, n:] == 0).all(), f"{name}: padding"
                wanted[0][name] = mask_rows(wanted[0][name], self.n, 0.0)
                wanted = wanted[0], [{**w, name: mask_rows(w[name], self.n, 0.0)} for w in wanted[1]]
            ref.check_delta(got, name, *wanted)


CASES = [  # type, B, L, Hk, H, K, V, lengths, pad, offset
    ("bf16", 2, 1, 1, 1, 128, 128, None, 0, 0),
    ("bf16", 2, 200, 2, 4, 128, 128, [200, 65], 0, 0),
    ("bf16", 3, 130, 1, 3, 64, 64, [64, 0, 129], 8, 8),
    ("bf16", 1, 63, 2, 2, 100, 72, None, 3, 1),
    ("bf16", 1, 320, 1, 1, 16, 300, None, 0, 0),
    ("bf16", 2, 66, 1, 2, 32, 16, [1, 66], 0, 0),
    ("fp16", 2, 150, 2, 2, 128, 128, [150, 90], 0, 0),
    ("fp16", 1, 70, 1, 4, 64, 33, None, 0, 4),
    ("fp16", 2, 65, 3, 3, 5, 3, [-4, 99], 1, 0),
    ("fp32", 2, 129, 1, 2, 128, 128, [129, 2], 0, 0),
    ("fp32", 1, 200, 2, 6, 60, 90, None, 0, 0),
    ("fp32", 2, 64, 1, 1, 1, 1, None, 4, 2),
    ("fp32", 1, 100, 1, 2, 33, 40, None, 4, 4),
]


@pytest.mark.parametrize("with_state", [True, False])
@pytest.mark.parametrize("case", CASES, ids=lambda c: f"{c[0]}-{'x'.join(map(str, c[1:7]))}-{c[8]}")
def test_delta_rule(lib, case, with_state):  # noqa: F811
    type, B, L, Hk, H, K, V, lengths, pad, offset = case
    c = Delta(lib, type, B, L, Hk, H, K, V, lengths, pad, offset, with_state)
    wanted = c.wanted(last=with_state)
    o, last = c.forward(keep=True)
    c.check({"o": o, "state": last}, wanted)
    kept = c.kept.clone()
    c.check(c.backward(last=with_state), wanted)
    assert torch.equal(c.kept, kept)                           # what the forward pass left is only read
    # without kept states the same bits; again the same bits
    first, end = o.result(), last.result()
    o, last = c.forward()
    assert torch.equal(o.result(), first) and torch.equal(last.result(), end)
    one, two = c.backward(last=with_state), c.backward(last=with_state)
    for name in one:
        assert torch.equal(one[name].result(), two[name].result()), name


@pytest.mark.parametrize("type", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("decay", [-30.0, 3.0, 20.0])
def test_strong_and_weak_decays(lib, type, decay):  # noqa: F811
    """Log decays near -30 (a state that forgets within a token), near -0.05 and near zero (one that keeps all)."""
    c = Delta(lib, type, 1, 150, 1, 2, 64, 32, decay=decay)
    wanted = c.wanted()
    o, last = c.forward(keep=True)
    c.check({"o": o, "state": last}, wanted)
    c.check(c.backward(), wanted)


@pytest.mark.parametrize("type", ["bf16", "fp32"])
def test_gates_at_their_ends(lib, type):  # noqa: F811
    """beta of zero (nothing is written), of one (replaced); a decay of -infinity (all forgotten) in the middle and at the first token; scale zero."""
    c = Delta(lib, type, 1, 140, 1, 1, 32, 16)
    c.beta[0, 10:30] = 0
    c.beta[0, 30:50] = 1
    c.g[0, 0], c.g[0, 70], c.g[0, 100] = -torch.inf, -torch.inf, -torch.inf
    c.br, c.gr = Rows((1, 140, 1), torch.float32, 0, 0, c.beta), Rows((1, 140, 1), torch.float32, 0, 0, c.g)
    wanted = c.wanted()
    o, last = c.forward(keep=True)
    c.check({"o": o, "state": last}, wanted)
    c.check(c.backward(), wanted)
    c.scale = 0.0
    assert (c.forward()[0].result() == 0).all()


def test_equal_keys(lib):  # noqa: F811
    """One key for every token, beta near one: t is as far from small as it gets."""
    for type in ("bf16", "fp32"):
        c = Delta(lib, type, 1, 130, 1, 1, 64, 16, decay=8.0)
        c.k[:] = c.k[:, :1]
        c.beta[:] = 1 - c.beta / 64
        c.beta = c.beta.float().to(F)
        c.kr, c.br = Rows((1, 130, 64), c.t, 0, 0, c.k), Rows((1, 130, 1), torch.float32, 0, 0, c.beta)
        wanted = c.wanted()
        o, last = c.forward(keep=True)
        c.check({"o": o, "state": last}, wanted)
        c.check(c.backward(), wanted)


@pytest.mark.parametrize("type", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("B, Hk, H, K, V, pad, offset", [(3, 2, 4, 128, 128, 0, 0), (1, 1, 1, 1, 1, 0, 0), (5, 1, 3, 100, 72, 8, 8), (2, 2, 2, 64, 300, 3, 1),
                                                         (40, 4, 8, 16, 24, 0, 0), (2, 1, 2, 33, 7, 1, 0)])
def test_single_tokens(lib, type, B, Hk, H, K, V, pad, offset):  # noqa: F811
    c = Delta(lib, type, B, 1, Hk, H, K, V, None, pad, offset)
    want = ref.delta_tokens(c.q, c.k, c.v, c.g, c.beta, c.state, c.n, c.scale)
    o, last, state = c.rows(H * V, c.t), Rows((B, H, K, V), torch.float32), Rows((B, H, K, V), torch.float32, 0, 0, c.state)
    call = lambda into: lib.delta_step_gated(c.qr.ptr, c.kr.ptr, c.vr.ptr, c.gr.ptr, c.br.ptr, state.ptr, o.ptr, into, B, Hk, H, K, V, c.qr.ld, c.kr.ld,  # noqa: E731
                                             c.vr.ld, c.gr.ld, c.br.ld, o.ld, c.scale, operand(lib, type), stream())
    call(last.ptr)
    # sums of K terms, the decay (its argument rounded, below 16 here) and a handful more, on both ways to a result
    a = torch.exp(c.g[:, 0])[..., None, None] * c.state.abs()
    kk, qq = (x[:, 0].abs().repeat_interleave(H // Hk, 1) for x in (c.k, c.q))
    size_u = c.beta[:, 0, :, None] * (c.v[:, 0].abs() + torch.einsum("bhkv,bhk->bhv", a, kk))
    size_o = c.scale * (torch.einsum("bhkv,bhk->bhv", a, qq) + size_u * (kk * qq).sum(-1, keepdim=True))
    check(last.result(), want[1], a + kk[..., None] * size_u[:, :, None], K + 40, "state")
    check(o.result().reshape(B, H, V), want[0][:, 0], size_o, 2 * K + 40, "o")
    first, out = last.result(), o.result()
    call(state.ptr)                                            # in place
    assert torch.equal(state.result(), first) and torch.equal(o.result(), out)


def test_a_sequence_in_pieces_and_tokens(lib):  # noqa: F811
    """A prompt, its continuation from the state (in place), then token by token: what one call gives."""
    whole = Delta(lib, "fp32", 2, 150, 1, 2, 64, 48)
    wanted = whole.wanted(grads=False)
    B, L, Hk, H, K, V = whole.dims
    o = Rows((B, L, H * V), torch.float32)
    state = Rows((B, H, K, V), torch.float32, 0, 0, whole.state)
    for lo, hi in ((0, 100), (100, 147)):
        part = Delta(lib, "fp32", B, hi - lo, Hk, H, K, V)
        for name, width in (("q", Hk * K), ("k", Hk * K), ("v", H * V), ("g", H), ("beta", H)):
            setattr(part, {"q": "qr", "k": "kr", "v": "vr", "g": "gr", "beta": "br"}[name],
                    Rows((B, hi - lo, width), torch.float32, 0, 0, getattr(whole, name)[:, lo:hi]))
        out, _ = part.forward(last=state, state=state.ptr)
        o.view().view(B, L, H * V)[:, lo:hi] = out.result()
    for t in range(147, 150):
        row = lambda r, w: r.ptr + t * w * 4  # noqa: E731
        lib.delta_step_gated(row(whole.qr, K), row(whole.kr, K), row(whole.vr, H * V), row(whole.gr, H), row(whole.br, H), state.ptr, row(o, H * V), state.ptr,
                             B, Hk, H, K, V, L * K, L * K, L * H * V, L * H, L * H, L * H * V, whole.scale, lib.OPERAND_FP32, stream())
    whole.check({"o": o, "state": state}, wanted)


def test_no_token_at_all(lib):  # noqa: F811
    c = Delta(lib, "bf16", 2, 70, 1, 1, 32, 16, lengths=[0, 0])
    o, last = c.forward(keep=True)
    assert (o.result() == 0).all() and torch.equal(last.result().double().cpu(), c.state)
    got = c.backward()
    for name in ("dq", "dk", "dv", "dg", "dbeta"):
        assert (got[name].result() == 0).all(), name
    assert torch.equal(got["dstate"].result().double().cpu(), c.dlast)


def test_delta_captured_and_on_another_stream(lib):  # noqa: F811
    """Forward and backward in a graph replayed on new inputs, and two calls at once on two streams with their own workspaces."""
    c, d = Delta(lib, "bf16", 2, 140, 1, 2, 64, 64), Delta(lib, "bf16", 2, 140, 1, 2, 64, 64, seed=800)
    op = lib.OPERAND_BF16
    ws = [workspace(max(lib.delta_fwd_gated_workspace_size(*c.dims, op), lib.delta_bwd_gated_workspace_size(*c.dims, op))) for _ in range(2)]
    want = []
    for x in (c, d):
        o, last = x.forward(keep=True)
        want.append([o.result(), last.result()] + [r.result() for r in x.backward().values()])
    side = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = []
    for x, s, w in zip((c, d), side, ws):
        with torch.cuda.stream(s):
            o, last = x.forward(keep=True, ws=w)
            got.append([o, last, *x.backward(ws=w).values()])
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        assert all(torch.equal(a.result(), b) for a, b in zip(g, w))
    out = [c.rows(128, c.t), Rows((2, 2, 64, 64), torch.float32)]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.forward(keep=True, o=out[0], last=out[1], ws=ws[0])
        grads = c.backward(ws=ws[0])
    for x in ("qr", "kr", "vr", "gr", "br", "dr"):
        getattr(c, x).view().copy_(getattr(d, x).view())
    c.sd.copy_(d.sd), c.dld.copy_(d.dld)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out[0].result(), want[1][0]) and torch.equal(out[1].result(), want[1][1])
    assert all(torch.equal(a.result(), b) for a, b in zip(grads.values(), want[1][2:]))


@pytest.mark.parametrize("columns", ["32", "64"])
@pytest.mark.parametrize("case", [("bf16", 2, 200, 2, 4, 128, 128, [200, 65]), ("fp16", 1, 150, 1, 2, 100, 96, None), ("fp32", 1, 130, 1, 1, 64, 72, None)],
                         ids=lambda c: f"{c[0]}-{c[5]}x{c[6]}")
def test_walks_of_either_width(lib, monkeypatch, case, columns):  # noqa: F811
    """Blocks of 32 and of 64 columns, whatever the rule says."""
    monkeypatch.setenv("CONV2D_B200_DELTA_COLUMNS", columns)
    c = Delta(lib, *case)
    wanted = c.wanted()
    o, last = c.forward(keep=True)
    c.check({"o": o, "state": last}, wanted)
    c.check(c.backward(), wanted)


def test_one_workspace_for_calls_one_after_the_other(lib):  # noqa: F811
    """Two graphs that share a workspace, and calls of other sizes on it, in turn; nothing is expected of what it holds."""
    c, d = Delta(lib, "bf16", 1, 200, 1, 2, 64, 64), Delta(lib, "fp32", 2, 70, 1, 1, 128, 40, seed=810)
    op = {"bf16": lib.OPERAND_BF16, "fp32": lib.OPERAND_FP32}
    need = max(f(*x.dims, op[x.type]) for x in (c, d) for f in (lib.delta_fwd_gated_workspace_size, lib.delta_bwd_gated_workspace_size))
    ws = workspace(need)
    ws.fill_(0xff)
    want, outs, graphs = [], [], []
    for x in (c, d):
        o, last = x.forward(keep=True, ws=ws)
        want.append([o.result(), last.result()] + [r.result() for r in x.backward(ws=ws).values()])
    torch.cuda.synchronize()
    for x in (c, d):
        o, last = x.rows(x.dims[3] * x.dims[5], x.t), Rows((x.dims[0], x.dims[3], x.dims[4], x.dims[5]), torch.float32)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            x.forward(keep=True, o=o, last=last, ws=ws)
            grads = x.backward(ws=ws)
        graphs.append(graph), outs.append([o, last, *grads.values()])
    for i in (0, 1, 1, 0):
        ws.fill_(0xff)
        graphs[i].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a.result(), b) for a, b in zip(outs[i], want[i]))


@pytest.mark.parametrize("V, columns", [(65536, None), (4100, "32")])
def test_many_columns(lib, monkeypatch, V, columns):  # noqa: F811
    if columns:
        monkeypatch.setenv("CONV2D_B200_DELTA_COLUMNS", columns)
    c = Delta(lib, "bf16", 1, 70 if V < 65536 else 3, 1, 1, 5, V)
    wanted = c.wanted()
    o, last = c.forward(keep=True)
    c.check({"o": o, "state": last}, wanted)
    c.check(c.backward(), wanted)


def test_an_expired_wait_is_reported(lib, monkeypatch):  # noqa: F811
    """With no patience at all every wait gives up: the kernels wait for what they have under way, return, and the status says so, once; the next calls are right."""
    c = Delta(lib, "bf16", 2, 140, 1, 2, 64, 64)
    wanted = c.wanted()
    c.forward(keep=True)
    torch.cuda.synchronize()
    for call in (c.forward, c.backward):
        monkeypatch.setenv("CONV2D_B200_DELTA_MAX_POLLS", "0")
        call()
        with pytest.raises(lib.Conv2dError) as e:
            lib.conv2d_get_status(0, stream())
        assert e.value.status == 8                              # CONV2D_ERR_DEVICE_TIMEOUT
        torch.cuda.synchronize()
        lib.conv2d_get_status(0, stream())
        monkeypatch.delenv("CONV2D_B200_DELTA_MAX_POLLS")
    o, last = c.forward(keep=True)
    c.check({"o": o, "state": last}, wanted)
    c.check(c.backward(), wanted)
    lib.conv2d_get_status(0, stream())


def test_delta_beyond_32_bit_offsets(lib):  # noqa: F811
    """Rows so far apart that the last sequence lies beyond 2^31 elements."""
    B, L, K, V = 3, 70, 64, 32
    ld = (1 << 31) // (2 * L) + 8
    c = Delta(lib, "bf16", B, L, 1, 1, K, V)
    buf = torch.zeros(B * L * ld, dtype=torch.bfloat16, device="cuda")
    place = lambda x, at: buf.as_strided((B * L, x.shape[-1]), (ld, 1), at).copy_(x.reshape(B * L, -1))  # noqa: E731
    place(c.q, 0), place(c.k, 128), place(c.v, 256)
    o, last = Rows((B, L, V), c.t), Rows((B, 1, K, V), torch.float32)
    need = lib.delta_fwd_gated_workspace_size(*c.dims)
    ws = workspace(need)
    at = lambda n: buf.data_ptr() + 2 * n  # noqa: E731
    lib.delta_fwd_gated(at(0), at(128), at(256), c.gr.ptr, c.br.ptr, c.sd.data_ptr(), 0, at(512), last.ptr, 0, B, L, 1, 1, K, V, ld, ld, ld, 1, 1, ld, c.scale,
                        lib.OPERAND_BF16, ws.data_ptr(), need, stream())
    o.view().copy_(buf.as_strided((B * L, V), (ld, 1), 512))
    c.check({"o": o, "state": last}, c.wanted(grads=False))


# --------------------------------------------------------------------------------------------------------------- RMS norm

RMS = [  # type, M, C, G, residual, gate, pad, offset
    ("bf16", 3, 4096, 1, True, False, 0, 0),
    ("bf16", 17, 128, 1, False, False, 0, 0),
    ("bf16", 5, 2048, 16, False, True, 8, 8),
    ("fp16", 9, 144, 1, True, True, 0, 0),
    ("fp16", 33, 96, 4, True, True, 0, 0),
    ("fp16", 4, 1001, 7, False, True, 3, 1),
    ("fp32", 6, 520, 5, True, False, 0, 0),
    ("fp32", 2, 16384, 1, True, True, 0, 0),
    ("bf16", 2, 16384, 2, False, False, 1, 0),
    ("fp32", 1, 1, 1, True, True, 0, 0),
    ("bf16", 700, 40, 5, True, False, 0, 0),
    ("fp32", 3, 6, 6, True, True, 2, 2),
    ("fp16", 2, 11000, 1, True, False, 0, 0),
    ("bf16", 21, 1792, 32, True, True, 0, 0),
    ("bf16", 5, 1084, 1, True, False, 0, 0),
    ("fp16", 6, 1162, 7, False, True, 0, 0),
    ("fp32", 3, 16383, 129, True, True, 1, 1),
    ("fp16", 2, 16320, 60, True, True, 0, 4),
    ("bf16", 2, 16383, 1, True, False, 0, 1),
    ("fp32", 9, 90, 5, True, True, 0, 2),
    # (several rows a block, the last ones fewer)
    ("bf16", 3001, 1280, 1, True, False, 0, 0),
    ("fp16", 6001, 520, 5, False, True, 0, 0),
    ("fp32", 4003, 300, 3, True, True, 1, 1),
    ("bf16", 5003, 264, 1, False, True, 0, 0),
    ("fp32", 1300, 4096, 32, False, False, 0, 0),
    ("bf16", 1501, 8200, 1, True, True, 0, 0),
]


@pytest.mark.parametrize("case", RMS, ids=lambda c: "-".join(map(str, c)))
def test_rms_norm(lib, case):  # noqa: F811
    type, M, C, G, residual, gate, pad, offset = case
    t, eps = TYPES[type], 1e-5
    x, res, z = draw(900, M, C, dtype=t), draw(901, M, C, scale=3.0, dtype=t), draw(902, M, C, scale=2.0, dtype=t)
    gamma, dy, dh = draw(903, C // G, scale=0.3, shift=1.0).float().to(F), draw(904, M, C, dtype=t), draw(905, M, C, dtype=t)
    h = (x + res).float().to(t).to(F) if residual else x         # (a sum of two is rounded to 24 bits before it is rounded to its type)
    R = lambda v=None, w=t: Rows((M, C), w, pad, offset, v)  # noqa: E731
    xr, rr, zr, dyr, dhr, yr, hr, dxr, dzr = R(x), R(res), R(z), R(dy), R(dh), R(), R(), R(), R()
    gr, rstd, dg = cuda(gamma), Rows((M, G), torch.float32), Rows((C // G,), torch.float32)
    lib.norm_fwd_rms(xr.ptr, rr.ptr if residual else 0, zr.ptr if gate else 0, gr.data_ptr(), yr.ptr, hr.ptr if residual else 0, 0, 0, rstd.ptr, M, C, G, 0,
                     xr.ld, rr.ld, zr.ld, yr.ld, hr.ld, 0, eps, operand(lib, type), stream())
    (y, size), r = ref.rms_fwd(h, z if gate else None, gamma, G, eps)
    n = C // G
    adds = min(n, 16) + 12                                     # a thread's elements one after the other, then trees over lanes and warps; the sum is positive
    check(yr.result(), y, size, adds + 16, "y")
    check(rstd.result(), r, r, adds + 4, "rstd")
    if residual:
        assert torch.equal(hr.result().double().cpu(), h)
    need = lib.norm_bwd_rms_workspace_size(M, C, G)
    ws = workspace(need)
    kept = hr if residual else xr
    for _ in range(2):
        lib.norm_bwd_rms(kept.ptr, zr.ptr if gate else 0, gr.data_ptr(), rstd.ptr, dyr.ptr, dhr.ptr if residual else 0, dxr.ptr, dzr.ptr if gate else 0, dg.ptr,
                         M, C, G, kept.ld, zr.ld, dyr.ld, dhr.ld, dxr.ld, dzr.ld, operand(lib, type), ws.data_ptr(), need, stream())
    dx, dz, dgamma = ref.rms_bwd(h, z if gate else None, gamma, G, eps, dy, dh if residual else None)
    check(dxr.result(), *dx, 3 * adds + 40, "dx")
    if gate:
        check(dzr.result(), *dz, adds + 40, "dz")
    check(dg.result(), *dgamma, adds + 40 + M * G, "dgamma")    # whatever the order of its M * G terms
    # without the scale, without its gradient, in place of the residual and of dy: the same values
    one = torch.ones(n, device="cuda")
    lib.norm_fwd_rms(xr.ptr, rr.ptr if residual else 0, zr.ptr if gate else 0, one.data_ptr(), yr.ptr, hr.ptr if residual else 0, 0, 0, 0, M, C, G, -5,
                     xr.ld, rr.ld, zr.ld, yr.ld, hr.ld, -1, eps, operand(lib, type), stream())
    want, into = yr.result(), rr if residual else R()
    lib.norm_fwd_rms(xr.ptr, rr.ptr if residual else 0, zr.ptr if gate else 0, 0, yr.ptr, into.ptr if residual else 0, 0, 0, 0, M, C, G, 0,
                     xr.ld, rr.ld, zr.ld, yr.ld, into.ld, 0, eps, operand(lib, type), stream())
    assert torch.equal(yr.result(), want) and (not residual or torch.equal(into.result().double().cpu(), h))
    want = dxr.result()
    lib.norm_bwd_rms(kept.ptr, zr.ptr if gate else 0, gr.data_ptr(), rstd.ptr, dyr.ptr, dhr.ptr if residual else 0, dyr.ptr, dzr.ptr if gate else 0, 0,
                     M, C, G, kept.ld, zr.ld, dyr.ld, dhr.ld, dyr.ld, dzr.ld, operand(lib, type), 0, 0, stream())
    assert torch.equal(dyr.result(), want)


@pytest.mark.parametrize("type, M, C, G, block, pad, gate", [("bf16", 5, 4096, 1, 128, 0, False), ("bf16", 7, 4096, 1, 4096, 0, False), ("fp16", 3, 1000, 1, 128, 8, True),
                                                             ("fp16", 4, 288, 6, 128, 0, False), ("bf16", 2, 77, 7, 10, 1, False), ("fp32", 3, 96, 3, 7, 0, True),
                                                             ("fp32", 2, 260, 1, 64, 0, False), ("bf16", 9, 24, 3, 1, 0, False), ("bf16", 300, 64, 1, 64, 0, True),
                                                             ("bf16", 4, 72, 1, 128, 0, False), ("fp16", 2, 45, 3, 1 << 30, 2, True),
                                                             ("bf16", 6001, 512, 1, 128, 0, False), ("fp32", 5003, 256, 1, 256, 0, False),
                                                             ("fp16", 4001, 500, 1, 100, 0, True)])
def test_output_in_8_bits(lib, type, M, C, G, block, pad, gate):  # noqa: F811
    t = TYPES[type]
    x, z = draw(910, M, C, dtype=t), draw(911, M, C, dtype=t)
    x[0], gamma = 0, draw(912, C // G, shift=1.0).float().to(F)
    xr, zr, y8, n = Rows((M, C), t, pad, 0, x), Rows((M, C), t, pad, 0, z), torch.full((M, C + pad + 3), 9, dtype=torch.uint8, device="cuda"), -(-C // block)
    wide = min(block, C)
    gr, scales, yr = cuda(gamma), Rows((M, n), torch.float32), Rows((M, C), t)
    for y in (0, yr.ptr):                                      # with and without an output of the type
        lib.norm_fwd_rms(xr.ptr, 0, zr.ptr if gate else 0, gr.data_ptr(), y, 0, y8.data_ptr(), scales.ptr, 0, M, C, G, block, xr.ld, 0, zr.ld, C, 0, C + pad + 3,
                         1e-5, operand(lib, type), stream())
    (want, size), _ = ref.rms_fwd(x, z if gate else None, gamma, G, 1e-5)
    check(yr.result(), want, size, 50, "y")
    assert (y8[:, C:] == 9).all()
    blocks = torch.nn.functional.pad(want, (0, n * wide - C)).reshape(M, n, wide)
    s = (blocks.abs().amax(-1) / 448).clamp(min=2.0 ** -126)
    grow = torch.nn.functional.pad(size, (0, n * wide - C)).reshape(M, n, wide).amax(-1) / 448
    check(scales.result(), s, torch.maximum(grow, s), 52, "scales")
    values = y8[:, :C].view(torch.float8_e4m3fn).double().cpu() * scales.result().double().cpu().repeat_interleave(wide, 1)[:, :C]
    spread = s.repeat_interleave(wide, 1)[:, :C]
    # half a step: 2^-4 of the value, 2^-10 of a scale below the smallest normal code; 60 roundings before
    assert ((values - want).abs() <= 2.0 ** -4 * want.abs() * (1 + 2.0 ** -17) + 2.0 ** -10 * spread + 60 * 2.0 ** -24 * (size + 448 * spread)).all()
    assert (values[0] == 0).all() and (scales.result()[0] == 2.0 ** -126).all()


def test_rms_extremes_and_graphs(lib):  # noqa: F811
    """Rows of zeros, of the largest numbers and with values that are not finite leave other rows alone; eps zero; a captured call sees new inputs."""
    M, C = 6, 256
    x = draw(920, M, C, dtype=torch.bfloat16).to(torch.bfloat16).cuda()
    x[1], x[2], x[3, 5], x[4, 7] = 0, 2.0 ** 60, float("nan"), float("inf")
    y, rstd = torch.empty_like(x), torch.empty(M, 1, device="cuda")
    call = lambda eps: lib.norm_fwd_rms(x.data_ptr(), 0, 0, 0, y.data_ptr(), 0, 0, 0, rstd.data_ptr(), M, C, 1, 0, C, 0, 0, C, 0, 0, eps,  # noqa: E731
                                        lib.OPERAND_BF16, stream())
    call(1e-6)
    assert (y[1] == 0).all() and (y[2] == 1).all() and y[3].isnan().all()
    for i in (0, 5):
        (want, size), _ = ref.rms_fwd(x[i:i + 1].double().cpu(), None, torch.ones(C, dtype=F), 1, 1e-6)
        check(y[i:i + 1], want, size, 40, "y")
    call(0.0)
    assert torch.isfinite(y[0]).all() and (y[2] == 1).all()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(1e-6)
    x[:] = draw(921, M, C).to(torch.bfloat16).cuda()
    graph.replay()
    (want, size), _ = ref.rms_fwd(x.double().cpu(), None, torch.ones(C, dtype=F), 1, 1e-6)
    check(y, want, size, 40, "y")


@pytest.mark.parametrize("type, M, C, G", [("bf16", 1500, 2048, 1), ("fp32", 700, 96, 3), ("fp16", 3, 5000, 1)])
def test_rms_training_captured_in_place_and_on_two_streams(lib, type, M, C, G):  # noqa: F811
    """Forward and backward as a training step calls them, h in place of x and dx in place of dh: eager on two streams at once, and in a graph replayed on other inputs."""
    t, op, eps = TYPES[type], operand(lib, type), 1e-5
    need = lib.norm_bwd_rms_workspace_size(M, C, G)

    class Step:
        def __init__(self, seed):
            new = lambda i, *s: draw(seed + i, *s).to(t).cuda()  # noqa: E731
            self.x, self.res, self.dy, self.dh = (new(i, M, C) for i in range(4))
            self.gamma = draw(seed + 4, C // G, shift=1.0).float().cuda()
            self.y, self.rstd, self.dgamma, self.ws = torch.empty_like(self.x), torch.empty(M, G, device="cuda"), torch.empty(C // G, device="cuda"), workspace(need)
            self.given = [v.clone() for v in (self.x, self.res, self.dy, self.dh, self.gamma)]

        def reset(self, other=None):
            for v, w in zip((self.x, self.res, self.dy, self.dh, self.gamma), (other or self).given):
                v.copy_(w)

        def run(self, on):
            p = lambda v: v.data_ptr()  # noqa: E731
            lib.norm_fwd_rms(p(self.x), p(self.res), 0, p(self.gamma), p(self.y), p(self.x), 0, 0, p(self.rstd), M, C, G, 0, C, C, 0, C, C, 0, eps, op, on)
            lib.norm_bwd_rms(p(self.x), 0, p(self.gamma), p(self.rstd), p(self.dy), p(self.dh), p(self.dh), 0, p(self.dgamma), M, C, G, C, 0, C, C, C, 0, op,
                             p(self.ws), need, on)

        def results(self):
            return [v.clone() for v in (self.x, self.y, self.rstd, self.dh, self.dgamma)]

    steps = [Step(950), Step(970)]
    want = []
    for s in steps:
        h = (s.given[0].float() + s.given[1].float()).to(t)
        s.run(stream())
        want.append(s.results())
        assert torch.equal(s.x, h)
        kept = h.double().cpu()
        (y, size), _ = ref.rms_fwd(kept, None, s.given[4].double().cpu(), G, eps)
        dx, _, _ = ref.rms_bwd(kept, None, s.given[4].double().cpu(), G, eps, s.given[2].double().cpu(), s.given[3].double().cpu())
        adds = min(C // G, 16) + 12
        check(s.y, y, size, adds + 16, "y")
        check(s.dh, *dx, 3 * adds + 40, "dx")
        s.reset()
    torch.cuda.synchronize()
    sides = [torch.cuda.Stream(), torch.cuda.Stream()]
    for s, side in zip(steps, sides):
        s.run(side.cuda_stream)
    torch.cuda.synchronize()
    for s, w in zip(steps, want):
        assert all(torch.equal(a, b) for a, b in zip(s.results(), w))
        s.reset()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        steps[0].run(stream())
    for i in (1, 0):
        steps[0].reset(steps[i])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(steps[0].results(), want[i]))


# ---------------------------------------------------------------------------------------------------------------- a layer

def test_a_layer_of_them_with_the_convolution(lib):  # noqa: F811
    """Norm with the residual, causal convolution of queries, keys and values in one tensor, norm of the heads of queries and keys by slices of it, delta rule,
    norm of heads with a gate: forward and backward, as a layer would call them, against automatic differentiation in 64 bits."""
    B, L, Hk, H, K, V, taps, eps = 2, 90, 1, 2, 64, 32, 4, 1e-6
    C, Q, D = 2 * Hk * K + H * V, Hk * K, H * V
    f32, op, f = torch.float32, lib.OPERAND_FP32, stream
    new = lambda *s: torch.empty(s, device="cuda")  # noqa: E731
    x, res, w = draw(930, B * L, C), draw(931, B * L, C), draw(932, C, taps, scale=0.5)
    z, gamma, out_gamma = draw(933, B * L, D), draw(934, C, shift=1.0, scale=0.1), draw(935, V, shift=1.0, scale=0.1)
    g, beta = -torch.nn.functional.softplus(draw(936, B * L, H)), torch.sigmoid(draw(937, B * L, H))
    dy, dh = draw(938, B * L, D), draw(939, B * L, C)
    # queries and keys of length one: their mean square is 1 / K
    leaves = {n: v.float().to(F).requires_grad_() for n, v in dict(x=x, w=w, z=z, gamma=gamma, out_gamma=out_gamma, g=g, beta=beta).items()}
    hs = (leaves["x"].float() + res.float()).to(F)
    h = leaves["x"] + res.float().to(F) + (hs - leaves["x"] - res.float().to(F)).detach()
    rms = lambda v, d: v * (v.reshape(*v.shape[:-1], -1, d).square().mean(-1, keepdim=True) + eps).rsqrt().expand(*v.shape[:-1], v.shape[-1] // d, d).reshape(v.shape)  # noqa: E731
    n = rms(h, C) * leaves["gamma"]
    padded = torch.cat([torch.zeros(B, taps - 1, C, dtype=F), n.reshape(B, L, C)], 1)
    a = sum(padded[:, i:i + L] * leaves["w"][:, i] for i in range(taps))
    a = a * torch.sigmoid(a)
    q, k = rms(a[..., :Q], K) * K ** -0.5, rms(a[..., Q:2 * Q], K) * K ** -0.5
    o, _ = ref.delta_tokens(q.reshape(B, L, Hk, K), k.reshape(B, L, Hk, K), a[..., 2 * Q:].reshape(B, L, H, V), leaves["g"].reshape(B, L, H), leaves["beta"].reshape(B, L, H),
                            torch.zeros(B, H, K, V, dtype=F), [L] * B, K ** -0.5)
    zz = leaves["z"].reshape(B, L, H, V)
    y = rms(o.reshape(B, L, D), V).reshape(B, L, H, V) * leaves["out_gamma"] * zz * torch.sigmoid(zz)
    want = dict(zip(leaves, torch.autograd.grad((y, h), list(leaves.values()), (dy.reshape(B, L, H, V), dh))))

    p = lambda t: t.data_ptr()  # noqa: E731
    d = {n: v.detach().float().cuda() for n, v in leaves.items()}
    rd, dyd, dhd, unit = cuda(res), cuda(dy), cuda(dh), torch.full((K,), K ** -0.5, device="cuda")
    hd, nd, cd, qk = new(B * L, C), new(B * L, C), new(B * L, C), new(B * L, 2 * Q)
    od, yd, r0, r1, r2 = new(B * L, D), new(B * L, D), new(B * L, 1), new(B * L, 2 * Hk), new(B * L, H)
    dims = (B, L, Hk, H, K, V, op)
    kept = workspace(lib.delta_states_size(*dims))
    ws = workspace(max(lib.delta_fwd_gated_workspace_size(*dims), lib.delta_bwd_gated_workspace_size(*dims), lib.norm_bwd_rms_workspace_size(B * L, C, 1),
                       lib.norm_bwd_rms_workspace_size(B * L, D, H), lib.conv1d_bwd_causal_workspace_size(B, L, C, taps)))
    W = (p(ws), ws.numel())
    lib.norm_fwd_rms(p(d["x"]), p(rd), 0, p(d["gamma"]), p(nd), p(hd), 0, 0, p(r0), B * L, C, 1, 0, C, C, 0, C, C, 0, eps, op, f())
    lib.conv1d_fwd_causal(p(nd), p(d["w"]), 0, 0, 0, p(cd), 0, B, L, C, taps, C, C, op, lib.ACT_SILU, f())
    lib.norm_fwd_rms(p(cd), 0, 0, p(unit), p(qk), 0, 0, 0, p(r1), B * L, 2 * Q, 2 * Hk, 0, C, 0, 0, 2 * Q, 0, 0, eps, op, f())
    vp = p(cd) + 4 * 2 * Q
    lib.delta_fwd_gated(p(qk), p(qk) + 4 * Q, vp, p(d["g"]), p(d["beta"]), 0, 0, p(od), 0, p(kept), B, L, Hk, H, K, V, 2 * Q, 2 * Q, C, H, H, D, K ** -0.5, op, *W, f())
    lib.norm_fwd_rms(p(od), 0, p(d["z"]), p(d["out_gamma"]), p(yd), 0, 0, 0, p(r2), B * L, D, H, 0, D, 0, D, D, 0, 0, eps, op, f())
    do, dz, dog, dqk, dc, dg, db = new(B * L, D), new(B * L, D), new(V), new(B * L, 2 * Q), new(B * L, C), new(B * L, H), new(B * L, H)
    dn, dw, dx, dgm = new(B * L, C), new(C, taps), new(B * L, C), new(C)
    lib.norm_bwd_rms(p(od), p(d["z"]), p(d["out_gamma"]), p(r2), p(dyd), 0, p(do), p(dz), p(dog), B * L, D, H, D, D, D, 0, D, D, op, *W, f())
    lib.delta_bwd_gated(p(qk), p(qk) + 4 * Q, 0, p(kept), p(do), 0, p(dqk), p(dqk) + 4 * Q, p(dc) + 4 * 2 * Q, p(dg), p(db), 0, B, L, Hk, H, K, V, 2 * Q, 2 * Q, D,
                        2 * Q, 2 * Q, C, H, H, K ** -0.5, op, *W, f())
    lib.norm_bwd_rms(p(cd), 0, p(unit), p(r1), p(dqk), 0, p(dc), 0, 0, B * L, 2 * Q, 2 * Hk, C, 0, 2 * Q, 0, C, 0, op, 0, 0, f())
    lib.conv1d_bwd_causal(p(nd), p(d["w"]), 0, 0, 0, p(dc), 0, p(dn), p(dw), 0, 0, B, L, C, taps, C, C, C, op, lib.ACT_SILU, *W, f())
    lib.norm_bwd_rms(p(hd), 0, p(d["gamma"]), p(r0), p(dn), p(dhd), p(dx), 0, p(dgm), B * L, C, 1, C, 0, C, C, C, 0, op, *W, f())
    got = dict(y=yd, x=dx, w=dw, z=dz, gamma=dgm, out_gamma=dog, g=dg, beta=db)
    want["y"] = y.detach()
    # every stage is off by a few 2^-20 of what it computes (products of up to 128 terms) and passes that on; the norms divide by what may be a tenth of a typical
    # row, once in each of three stages either way: 2^-20 * 16 * 8 in norm
    for name, v in got.items():
        ref_v = want[name].reshape(v.shape)
        off = (v.double().cpu() - ref_v).norm() / ref_v.norm()
        assert off < 2.0 ** -13, (name, float(off))
