"""Plain 64-bit forms of the gated delta rule and of RMS norm, and what rounding may do to the library's results.

Delta rule.  `delta_tokens` is the definition, token by token.  `delta_pieces` computes the same and the gradients from the formulas of pieces of 64 tokens, and
can be told to err: every product of matrices is then off by u * (|a| @ |b|) * r, r drawn from -1 .. 1, where the kernels' are off by at most that.
What comes of such errors, further products included, is what rounding may do to a result.  u for a product of n terms: operands in three bf16
parts are off by 2^-24 each (a rounding of 2^-8, of the rest of it again, and again) and what is left out, products of later parts, is 3 * 2^-24;
the sum of n terms in fp32 by at most n 2^-24, of which errors of either sign leave about sqrt(n): taken as 16 * 2^-24 for n <= 128.  Exponentials of sums of decays
are off by 2^-22 and by 2^-24 of their argument, which is below 90 where they are not zero: 2^-17, but only of what is nearly nothing; u covers 16 * 2^-24 of it.
A check allows half a step of the result's type and, of errors drawn three times, four times the largest for each head: in norm, and (eight times) for a
single value.
"""
from __future__ import annotations

import torch

from sequence_reference import TYPES  # noqa: F401

F = torch.float64
U = 5 * 2.0 ** -24 + 2.0 ** -20
PIECE = 64


def delta_tokens(q, k, v, g, beta, state, lengths, scale):
    """q, k [B][L][Hk][K], v [B][L][H][V], g, beta [B][L][H], state [B][H][K][V].  Returns o and the last state."""
    B, L, H, V = v.shape
    share = H // q.shape[2]
    S, outs = state, []
    n = torch.tensor(lengths)
    for t in range(L):
        on = (t < n)[:, None, None]
        kt, qt = (torch.where(on, x[:, t], 0).repeat_interleave(share, 1) for x in (k, q))
        vt, gt, bt = torch.where(on, v[:, t], 0), torch.where(on[..., 0], g[:, t], 0), torch.where(on[..., 0], beta[:, t], 0)
        S = S * torch.exp(gt)[..., None, None]
        u = bt[..., None] * (vt - torch.einsum("bhkv,bhk->bhv", S, kt))
        S = S + kt[..., None] * u[..., None, :]
        outs.append(scale * torch.einsum("bhkv,bhk->bhv", S, qt))
    return torch.stack(outs, 1), S


class Errs:
    """Products that are off by at most u of the sum of their terms' sizes."""

    def __init__(self, u=0.0, seed=0):
        self.u, self.gen = u, torch.Generator().manual_seed(seed)

    def mm(self, a, b):
        c = a @ b
        return c + self.u * (a.abs() @ b.abs()) * (2 * torch.rand(c.shape, generator=self.gen, dtype=F) - 1) if self.u else c


def delta_pieces(q, k, v, g, beta, state, lengths, scale, dout=None, dlast=None, errs=None):
    """A dict of o, state (the last) and, with dout, dq, dk, dv, dg, dbeta, dstate."""
    B, L, H, V = v.shape
    Hk, K = q.shape[2:]
    share, n = H // Hk, -(-L // PIECE)
    e = errs or Errs()
    real = torch.arange(L)[None] < torch.tensor(lengths)[:, None]

    def pieces(x, heads):
        x = torch.where(real.reshape(B, L, *(1,) * (x.dim() - 2)), x, 0)
        x = torch.cat([x, x.new_zeros(B, n * PIECE - L, *x.shape[2:])], 1).reshape(B, n, PIECE, *x.shape[2:])
        return x.transpose(2, 3).transpose(1, 2).repeat_interleave(H // heads, 1)

    def back(x, heads):
        x = torch.stack(x, 2)                                     # [B][H][n][64][..]
        x = x.reshape(B, heads, H // heads, *x.shape[2:]).sum(2)
        return x.transpose(1, 2).transpose(2, 3).reshape(B, n * PIECE, heads, *x.shape[4:])[:, :L]

    q, k, v = pieces(q, Hk), pieces(k, Hk), pieces(v, H)
    g, beta = pieces(g, H), pieces(beta, H)[..., None]
    G = torch.cumsum(torch.clamp(g, min=-10000.0), -1)
    low = torch.ones(PIECE, PIECE, dtype=torch.bool).tril()
    D = torch.exp(torch.where(low, G[..., :, None] - G[..., None, :], -torch.inf))
    begin, end = torch.exp(G)[..., None], torch.exp(G[..., -1:] - G)[..., None]
    S, kept, out = state, [], []
    for c in range(n):
        kc, qc = k[:, :, c], q[:, :, c]
        A, P = D[:, :, c].tril(-1) * e.mm(kc, kc.mT), D[:, :, c] * e.mm(qc, kc.mT)
        t = torch.linalg.solve_triangular(torch.eye(PIECE, dtype=F) + A * beta[:, :, c].mT, A, upper=False, unitriangular=True)
        t = t + e.u * t.abs() * (2 * torch.rand(t.shape, generator=e.gen, dtype=F) - 1)
        R = v[:, :, c] - begin[:, :, c] * e.mm(kc, S)
        E = R - e.mm(t, beta[:, :, c] * R)
        kept.append((S, E, t, P))
        out.append(scale * (begin[:, :, c] * e.mm(qc, S) + e.mm(P, beta[:, :, c] * E)))
        S = begin[:, :, c, -1:] * S + e.mm(kc.mT, end[:, :, c] * beta[:, :, c] * E)
    r = {"o": back(out, H), "state": S}
    if dout is None:
        return r
    dout = pieces(dout, H)
    dS = torch.zeros_like(S) if dlast is None else dlast
    got = {x: [None] * n for x in ("dq", "dk", "dv", "dg", "dbeta")}
    for c in reversed(range(n)):
        kc, qc, do, be = k[:, :, c], q[:, :, c], dout[:, :, c], beta[:, :, c]
        S, E, t, P = kept[c]
        eg, ed, Dc = begin[:, :, c], end[:, :, c], D[:, :, c]
        dU = scale * e.mm(P.mT, do) + ed * e.mm(kc, dS)
        W = dU - e.mm(t.mT, be * dU)
        dv = be * W
        p = Dc * scale * e.mm(do, E.mT) * be.mT
        y = -Dc.tril(-1) * e.mm(dv, E.mT) * be.mT
        dq = scale * eg * e.mm(do, S.mT) + e.mm(p, kc)
        plus = e.mm(y, kc) - eg * e.mm(dv, S.mT)
        kd = ed * be * e.mm(E, dS.mT)
        minus = e.mm(p.mT, qc) + e.mm(y.mT, kc) + kd
        dG = (qc * dq + kc * (plus - minus)).sum(-1)
        inner = eg[..., -1, 0] * (S * dS).sum((-1, -2)) + (kc * kd).sum((-1, -2))
        got["dq"][c], got["dk"][c], got["dv"][c] = dq, plus + minus, dv
        got["dg"][c], got["dbeta"][c] = dG.flip(-1).cumsum(-1).flip(-1) + inner[..., None], (W * E).sum(-1)
        dS = eg[..., -1:, :] * dS + e.mm(qc.mT, scale * eg * do) - e.mm(kc.mT, eg * dv)
    for x in got:
        r[x] = back(got[x], Hk if x in ("dq", "dk") else H)
        r[x] = torch.where(real.reshape(B, L, *(1,) * (r[x].dim() - 2)), r[x], 0)
    r["dstate"] = dS
    return r


def delta_allowed(*args, **kw):
    """The 64-bit results and, three times, those of products that err as the kernels' may."""
    ref = delta_pieces(*args, **kw)
    return ref, [delta_pieces(*args, **kw, errs=Errs(U, 100 + i)) for i in range(3)]


def check_delta(got, name, ref, wrong):
    """got: the library's result for ref[name]; heads are its third dimension from the front of tokens, the second of states."""
    half, tiny = torch.finfo(got.dtype).eps / 2, torch.finfo(got.dtype).tiny
    got, want = got.double().cpu(), ref[name]
    assert got.shape == want.shape and torch.isfinite(got).all(), f"{name}: not finite"
    heads = 1 if name in ("state", "dstate") else 2
    one = lambda x: x.movedim(heads, 0).reshape(x.shape[heads], -1)  # noqa: E731
    off, w = one(got - want), one(want)
    errs = torch.stack([one(r[name]) - w for r in wrong])
    far = errs.norm(dim=-1).amax(0)
    limit = half * w.norm(dim=-1) + 4 * far + tiny
    assert (off.norm(dim=-1) <= limit).all(), f"{name}: off by {(off.norm(dim=-1) / limit).max():.2f} of what is allowed in norm"
    single = half * w.abs() + 8 * errs.abs().amax((0, 2))[:, None] + tiny
    assert (off.abs() <= single).all(), f"{name}: a value off by {(off.abs() / single).max():.2f} of what is allowed"


# --------------------------------------------------------------------------------------------------------------- RMS norm

def rms_fwd(h, z, gamma, G, eps):
    """h [M][C] as stored, z or None, gamma [C/G].  Returns (y, size), rstd."""
    M, C = h.shape
    x = h.reshape(M, G, C // G)
    r = (x.square().mean(-1, keepdim=True) + eps).rsqrt()
    y = x * r * gamma
    if z is None:
        return (y.reshape(M, C), y.abs().reshape(M, C)), r[..., 0]
    z = z.reshape(M, G, C // G)
    s = torch.sigmoid(z)
    # (the exponential's argument is rounded: |z| 2^-24 relative)
    return ((y * z * s).reshape(M, C), ((y * z * s).abs() * (1 + z.abs())).reshape(M, C)), r[..., 0]


def rms_bwd(h, z, gamma, G, eps, dy, dh):
    """(dx, size), (dz, size), (dgamma, size)"""
    M, C = h.shape
    heads = lambda x: x.reshape(M, G, C // G)  # noqa: E731
    x, dy = heads(h), heads(dy)
    r = (x.square().mean(-1, keepdim=True) + eps).rsqrt()
    m = x * r
    gate, more, dz = 1.0, 1.0, None
    if z is not None:
        z = heads(z)
        s = torch.sigmoid(z)
        gate, more = z * s, 1 + z.abs()
        dz = dy * gamma * m * s * (1 + z * (1 - s))
        dz = dz.reshape(M, C), ((dy * gamma * m).abs() * s * more * more).reshape(M, C)
    n = dy * gate * gamma
    dx = r * (n - m * (n * m).mean(-1, keepdim=True))
    size = r * (n.abs() * more + m.abs() * ((n * m).abs() * more).mean(-1, keepdim=True))
    dx, size = dx.reshape(M, C), size.reshape(M, C)
    if dh is not None:
        dx, size = dx + dh, size + dh.abs()
    return (dx, size), dz, ((dy * gate * m).sum((0, 1)), ((dy * gate * m).abs() * more).sum((0, 1)))
