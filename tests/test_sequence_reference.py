"""The plain forms that the operators along a sequence are tested against: their gradients are those of automatic differentiation of the
definition, and those follow differences.  CPU, 64 bits."""
import pytest
import torch

import sequence_reference as ref

F = torch.float64


def rand(gen, *shape, scale=1.0):
    return torch.randn(shape, generator=gen, dtype=F) * scale


@pytest.mark.parametrize("act", ["none", "relu", "silu", "gelu"])
def test_conv_gradients(act):
    gen = torch.Generator().manual_seed(11)
    B, L, D, K, lengths = 3, 9, 4, 4, [9, 5, 2]
    leaves = [rand(gen, B, L, D), rand(gen, D, K), rand(gen, D), rand(gen, B, K - 1, D)]
    dy, dends = rand(gen, B, L, D), rand(gen, B, K - 1, D)

    def loss(x, w, bias, state):
        y, _, ends = ref.conv_fwd(x, w, bias, state, lengths, act)
        return sum((y[b, :n] * dy[b, :n]).sum() for b, n in enumerate(lengths)) + (ends * dends).sum()

    grads = torch.autograd.grad(loss(*[v.requires_grad_() for v in leaves]), leaves)
    with torch.no_grad():
        formula = ref.conv_bwd(*leaves, lengths, act, dy, dends)
        for got, want, leaf in zip(formula, grads, leaves):
            torch.testing.assert_close(got[0], want, rtol=1e-12, atol=1e-12)
            along = rand(gen, *leaf.shape)
            at = [v.detach().clone() for v in leaves]
            i = [k for k, v in enumerate(leaves) if v is leaf][0]
            h = 1e-6
            at[i] = leaf.detach() + h * along
            up = loss(*at)
            at[i] = leaf.detach() - h * along
            assert abs((up - loss(*at)) / (2 * h) - (want * along).sum()) < 1e-6


@pytest.mark.parametrize("soft, gated", [(True, True), (False, True), (True, False)])
def test_scan_gradients(soft, gated):
    gen = torch.Generator().manual_seed(12)
    B, L, D, N, G, lengths = 2, 7, 6, 3, 2, [7, 4]
    names = ["u", "ddelta_in", "A", "B", "C", "skip", "z", "bias", "state"]
    leaves = [rand(gen, B, L, D), rand(gen, B, L, D, scale=0.5), -torch.exp(rand(gen, D, N)), rand(gen, B, L, G, N), rand(gen, B, L, G, N),
              rand(gen, D), rand(gen, B, L, D), rand(gen, D), rand(gen, B, D, N)]
    dy, dlast = rand(gen, B, L, D), rand(gen, B, D, N)

    def loss(u, delta, A, Bm, Cm, skip, z, bias, state):
        (y, _), (h, _) = ref.scan_fwd(u, delta, A, Bm, Cm, skip, z if gated else None, bias, state, lengths, soft)
        return sum((y[b, :n] * dy[b, :n]).sum() for b, n in enumerate(lengths)) + (h * dlast).sum()

    for v in leaves:
        v.requires_grad_()
    grads = torch.autograd.grad(loss(*leaves), leaves, allow_unused=True)
    with torch.no_grad():
        u, delta, A, Bm, Cm, skip, z, bias, state = leaves
        out = ref.scan_bwd(u, delta, A, Bm, Cm, skip, z if gated else None, bias, state, lengths, soft, dy, dlast)
        formula = [out[k][0] for k in ("du", "ddelta", "dA", "dB", "dC", "dskip", "dz", "dbias", "dstate")]
        for i, (name, got, want, leaf) in enumerate(zip(names, formula, grads, leaves)):
            if want is None:
                assert name == "z" and not gated
                continue
            torch.testing.assert_close(got, want, rtol=1e-10, atol=1e-10, msg=name)
            along, h, at = rand(gen, *leaf.shape), 1e-6, [v.detach().clone() for v in leaves]
            at[i] = leaf.detach() + h * along
            up = loss(*at)
            at[i] = leaf.detach() - h * along
            # 1e-6 for the third derivatives, and the roundings of the loss (a sum of about 100 terms, each known to 2^-53 of itself at
            # best, whose sizes add up to no less than |loss|: without softplus steps of both signs let it grow to 1e9) over the step
            rounding = 100 * 2.0 ** -53 * abs(float(up)) / h
            assert abs((up - loss(*at)) / (2 * h) - (want * along).sum()) < 1e-6 * (1 + abs(float((want * along).sum()))) + rounding


@pytest.mark.parametrize("act", ["none", "relu", "silu", "gelu"])
@pytest.mark.parametrize("N, S, C, G", [(2, 5, 6, 3), (3, 1, 8, 2), (1, 4, 5, 1)])
def test_norm_gradients(act, N, S, C, G):
    gen = torch.Generator().manual_seed(13)
    leaves = [rand(gen, N, S, C).requires_grad_(), rand(gen, C).requires_grad_(), rand(gen, C).requires_grad_()]
    dy = rand(gen, N, S, C)
    (y, _), *_ = ref.norm_fwd(*leaves, G, 1e-5, act)
    want = torch.nn.functional.group_norm(leaves[0].transpose(1, 2), G, leaves[1], leaves[2], 1e-5).transpose(1, 2)
    torch.testing.assert_close(y, ref.act(want, act), rtol=1e-10, atol=1e-10)
    grads = torch.autograd.grad((y * dy).sum(), leaves)
    with torch.no_grad():
        got = ref.norm_bwd(*leaves, G, 1e-5, act, dy)
    for i in range(3):
        torch.testing.assert_close(got[i][0], grads[i], rtol=1e-9, atol=1e-9)
