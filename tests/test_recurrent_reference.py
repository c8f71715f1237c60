"""The plain forms against the definitions: pieces against tokens, gradients against automatic differentiation and differences."""
import pytest
import torch

import recurrent_reference as ref

F = torch.float64


def case(seed, B, L, Hk, H, K, V, state=True):
    gen = torch.Generator().manual_seed(seed)
    n = lambda *s: torch.randn(*s, generator=gen, dtype=F)  # noqa: E731
    unit = lambda x: x / x.norm(dim=-1, keepdim=True)  # noqa: E731
    return (unit(n(B, L, Hk, K)), unit(n(B, L, Hk, K)), n(B, L, H, V), -torch.nn.functional.softplus(n(B, L, H)), torch.sigmoid(n(B, L, H)),
            n(B, H, K, V) if state else torch.zeros(B, H, K, V, dtype=F))


@pytest.mark.parametrize("B, L, Hk, H, K, V, lengths", [(2, 130, 1, 2, 5, 7, [130, 65]), (2, 3, 2, 2, 4, 3, [0, 3]), (1, 64, 1, 1, 8, 2, [64])])
def test_pieces_are_the_recurrence_and_its_gradients(B, L, Hk, H, K, V, lengths):
    x = case(1, B, L, Hk, H, K, V)
    leaves = [y.clone().requires_grad_() for y in x]
    o, last = ref.delta_tokens(*leaves, lengths, 0.3)
    gen = torch.Generator().manual_seed(2)
    dout, dlast = torch.randn(o.shape, generator=gen, dtype=F), torch.randn(last.shape, generator=gen, dtype=F)
    real = (torch.arange(L)[None] < torch.tensor(lengths)[:, None])[..., None, None]
    dout = torch.where(real, dout, 0)
    grads = torch.autograd.grad((o, last), leaves, (dout, dlast))
    r = ref.delta_pieces(*x, lengths, 0.3, dout, dlast)
    want = dict(zip(("o", "state", "dq", "dk", "dv", "dg", "dbeta", "dstate"), (torch.where(real, o, 0).detach(), last.detach()) + grads))
    for name, w in want.items():
        assert torch.allclose(r[name], w, rtol=1e-9, atol=1e-9), name


def test_differences_agree_with_the_gradients_of_gates_and_keys():
    x = case(3, 1, 70, 1, 1, 4, 3)
    gen = torch.Generator().manual_seed(4)
    dout, dlast = torch.randn(1, 70, 1, 3, generator=gen, dtype=F), torch.randn(1, 1, 4, 3, generator=gen, dtype=F)
    r = ref.delta_pieces(*x, [70], 0.5, dout, dlast)

    def loss(x):
        o, s = ref.delta_tokens(*x, [70], 0.5)
        return (o * dout).sum() + (s * dlast).sum()

    for i, name in enumerate(("dq", "dk", "dv", "dg", "dbeta", "dstate")):
        for at in (0, 7, x[i].numel() // 2, x[i].numel() - 1):
            step = torch.zeros(x[i].numel(), dtype=F)
            step[at] = 1e-6
            up, down = list(x), list(x)
            up[i], down[i] = x[i] + step.reshape(x[i].shape), x[i] - step.reshape(x[i].shape)
            slope = (loss(up) - loss(down)) / 2e-6
            # central differences: step^2 of the third derivative, and 2^-52 of the loss over the step
            assert abs(slope - r[name].flatten()[at]) < 1e-6 * (1 + abs(slope)), name


@pytest.mark.parametrize("G, gate, residual", [(1, False, True), (3, True, False), (2, True, True)])
def test_rms_gradients(G, gate, residual):
    gen = torch.Generator().manual_seed(5)
    n = lambda *s: torch.randn(*s, generator=gen, dtype=F)  # noqa: E731
    h, z, gamma, dy, dh = n(4, 12).requires_grad_(), n(4, 12).requires_grad_(), n(12 // G).requires_grad_(), n(4, 12), n(4, 12)
    (y, _), _ = ref.rms_fwd(h, z if gate else None, gamma, G, 1e-3)
    total = (y * dy).sum() + ((h * dh).sum() if residual else 0)
    want = torch.autograd.grad(total, (h, gamma) + ((z,) if gate else ()))
    with torch.no_grad():
        dx, dz, dg = ref.rms_bwd(h, z if gate else None, gamma, G, 1e-3, dy, dh if residual else None)
    assert torch.allclose(dx[0], want[0], atol=1e-12) and torch.allclose(dg[0], want[1], atol=1e-12)
    assert (dz is None) == (not gate) and (not gate or torch.allclose(dz[0], want[2], atol=1e-12))
