"""The gated delta rule where its kernels go round: several pieces for every block of the gradients, several heads of a shared key for a block of the first kernel, walks
of 64 columns by the rule itself; empty and short sequences between long ones, one to five blocks of columns."""
import pytest
import torch

from test_gpu_recurrent import Delta
from test_gpu_sequence import Rows, lib  # noqa: F401

pytestmark = pytest.mark.gpu

# B * H * ceil(L / 64) is 448 to 640 everywhere, more than three for each of a B200's 148 SMs
CASES = [  # type, B, L, Hk, H, K, V, lengths, pad, offset
    ("bf16", 6, 832, 2, 6, 16, 32, [832, 0, 700, 65, 1, 800], 0, 0),
    ("bf16", 10, 1000, 1, 3, 128, 96, [1000, 1000, 0, 0, 0, 64, 999, 1, 128, 640], 0, 0),
    ("bf16", 16, 500, 2, 4, 64, 128, [500, 0, 450, 500, 64, 65, 0, 1, 500, 321, 500, 500, 0, 128, 500, 63], 0, 0),
    ("bf16", 4, 2048, 4, 4, 64, 64, None, 0, 0),
    ("bf16", 10, 3000, 1, 1, 24, 160, [3000, 0, 0, 2900, 1, 3000, 64, 0, 3000, 1500], 0, 0),
    ("fp16", 5, 1030, 2, 6, 64, 128, [1030, 0, 1025, 513, 0], 0, 0),
    ("fp16", 5, 1000, 3, 6, 100, 64, None, 8, 8),
    ("fp32", 12, 777, 1, 3, 64, 64, [777, 0, 0, 700, 1, 64, 777, 128, 0, 650, 777, 777], 0, 0),
    ("fp32", 8, 640, 3, 6, 40, 50, [640, 0, 640, 1, 600, 64, 0, 639], 1, 1),
    ("fp32", 5, 1024, 3, 6, 128, 32, None, 0, 0),
    ("fp32", 10, 700, 1, 5, 128, 100, [700, 700, 64, 0, 0, 0, 0, 1, 300, 700], 0, 0),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: f"{c[0]}-{'x'.join(map(str, c[1:7]))}-{c[8]}")
def test_blocks_of_several_pieces_and_heads(lib, case):  # noqa: F811
    type, B, L, Hk, H, K, V, lengths, pad, offset = case
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    assert B * H * -(-L // 64) > 3 * sms
    c = Delta(lib, type, B, L, Hk, H, K, V, lengths, pad, offset, seed=1200)
    wanted = c.wanted()
    o, last = c.forward(keep=True)
    c.check({"o": o, "state": last}, wanted)
    first = c.backward()
    c.check(first, wanted)
    again, end = c.forward(keep=True)
    assert torch.equal(again.result(), o.result()) and torch.equal(end.result(), last.result())
    for name, x in c.backward().items():
        assert torch.equal(x.result(), first[name].result()), name


def test_a_sequence_does_not_see_its_batch(lib):  # noqa: F811
    """The same sequences one by one and in a batch whose blocks take several pieces and heads: the same bits."""
    B, L, Hk, H, K, V = 7, 900, 2, 6, 32, 32
    lengths = [900, 0, 257, 900, 64, 1, 850]
    c = Delta(lib, "bf16", B, L, Hk, H, K, V, lengths, seed=1220)
    o, last = c.forward(keep=True)
    grads = {n: x.result().reshape(B, -1) for n, x in c.backward().items()}
    o, last = o.result(), last.result()
    for b in (0, 2, 6):
        one = Delta(lib, "bf16", 1, L, Hk, H, K, V, [lengths[b]], seed=1220)
        for x in ("qr", "kr", "vr", "gr", "br", "dr"):
            rows = getattr(c, x)
            setattr(one, x, Rows((1, L, rows.width), rows.buf.dtype, 0, 0, rows.view().reshape(B, L, -1)[b]))
        one.sd, one.dld = c.sd[b:b + 1].contiguous(), c.dld[b:b + 1].contiguous()
        oo, ll = one.forward(keep=True)
        assert torch.equal(oo.result()[0], o[b]) and torch.equal(ll.result()[0], last[b])
        for n, x in one.backward().items():
            assert torch.equal(x.result().reshape(-1), grads[n][b]), n


@pytest.mark.parametrize("type", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("K, V, share, pad", [(128, 128, 1, 0), (64, 96, 3, 0), (33, 20, 2, 1)])
def test_a_gate_without_a_state_has_no_gradient(lib, type, K, V, share, pad):  # noqa: F811
    """The first decay of a sequence that begins without a state has nothing to decay: its gradient is zero, not what rounding leaves of sums."""
    lengths = [1, 2, 64, 65, 130, 0]
    c = Delta(lib, type, 6, 130, 2, 2 * share, K, V, lengths, pad, pad, state=False, seed=1240)
    c.beta[3, :40] = 0
    c.br = Rows((6, 130, 2 * share), torch.float32, pad, pad, torch.where((torch.arange(130)[None] < torch.tensor(lengths)[:, None])[..., None], c.beta, float("nan")))
    wanted = c.wanted()
    o, last = c.forward(keep=True)
    c.check({"o": o, "state": last}, wanted)
    grads = c.backward()
    c.check(grads, wanted)
    dg = grads["dg"].result()
    assert (dg[:, 0] == 0).all()
    assert (o.result()[3, :40] == 0).all()


@pytest.mark.parametrize("type, K, V", [("bf16", 64, 96), ("fp32", 128, 32), ("fp16", 33, 20)])
@pytest.mark.parametrize("what", ["qr", "kr", "vr", "gr", "br", "dr"])
def test_what_is_not_finite_stays_in_its_head(lib, type, K, V, what):  # noqa: F811
    """A NaN and an infinity in one sequence, seen by the value heads of one key head at most: all other results, and the pieces before it, are the same bits."""
    B, L, Hk, share = 9, 1030, 1, 3
    H = Hk * share
    lengths = [1030, 0, 1030, 700, 1, 64, 1030, 1000, 129]
    results = []
    for spoil in (False, True):
        c = Delta(lib, type, B, L, 2 * Hk, 2 * H, K, V, lengths, seed=1260)
        if spoil:
            rows = getattr(c, what).view().view(B, L, -1)
            width = rows.shape[-1] // 2                         # of the first half of the heads
            rows[2, 70, width - 1], rows[2, 300, 0] = float("nan"), float("inf")
        o, last = c.forward(keep=True)
        grads = c.backward()
        results.append({"o": o.result().reshape(B, L, 2, -1), "state": last.result().reshape(B, 1, 2, -1),
                        **{n: x.result().reshape(B, 1 if n == "dstate" else L, 2, -1) for n, x in grads.items()}})
    bits = lambda x: x.view(torch.int32 if x.element_size() == 4 else torch.int16)  # noqa: E731
    for name, x in results[0].items():
        y = results[1][name]
        one, two = bits(x).clone(), bits(y).clone()
        assert torch.equal(one[:, :, 1], two[:, :, 1]), name   # the other half of the heads
        if name == "o":
            assert torch.equal(one[2, :64], two[2, :64])
        one[2, :, 0], two[2, :, 0] = 0, 0
        assert torch.equal(one, two), name                     # the other sequences
    assert not all(torch.isfinite(x[2].float()).all() for x in results[1].values())
