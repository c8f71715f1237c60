"""Plain 64-bit forms of the operators along a sequence, and what rounding may do to the library's results.

Every reference returns, beside each result, the same expression over absolute values ("size"): a computation in fp32 that makes n roundings on the
way to a result is off by at most about n * 2^-24 * size.  A result of type t is then rounded once more, by at most
eps(t) / 2 of its value.
"""
from __future__ import annotations

import math

import torch

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
U = 2.0 ** -24


def act(v, name):
    if name == "silu":
        return v * torch.sigmoid(v)
    if name == "relu":
        return torch.relu(v)
    if name == "gelu":
        return v * 0.5 * torch.erfc(-v / math.sqrt(2.0))
    return v


def slope(v, name):
    if name == "silu":
        s = torch.sigmoid(v)
        return s * (1 + v * (1 - s))
    if name == "relu":
        return (v > 0).double()
    if name == "gelu":
        return 0.5 * torch.erfc(-v / math.sqrt(2.0)) + v * torch.exp(-0.5 * v * v) / math.sqrt(2 * math.pi)
    return torch.ones_like(v)


def check(got, ref, size, roundings, what):
    """got: the library's result; |got - ref| <= half a step of its type + roundings * 2^-24 * size."""
    half = torch.finfo(got.dtype).eps / 2
    tiny = torch.finfo(got.dtype).tiny           # below the smallest normal number steps are absolute
    got, ref, size = got.double().cpu(), ref.double().cpu(), size.double().cpu()
    assert torch.isfinite(got).all(), f"{what}: not finite"
    bound = half * ref.abs() + (1 + half) * roundings * U * size + tiny
    off = (got - ref).abs()
    if not (off <= bound).all():
        i = int(torch.argmax(off - bound))
        raise AssertionError(f"{what}: off by {off.flatten()[i]:.3e}, allowed {bound.flatten()[i]:.3e}, at {i}: "
                             f"{got.flatten()[i]:.9g} for {ref.flatten()[i]:.9g}; {int((off > bound).sum())} of {off.numel()}")


# ------------------------------------------------------------------------------------------------------------ convolution

def conv_fwd(x, w, bias, state, lengths, name):
    """x [B][L][D] in 64 bits.  Returns y, its size, the state behind each sequence."""
    B, L, D = x.shape
    K = w.shape[1]
    y, size, ends = torch.zeros_like(x), torch.zeros_like(x), torch.zeros(B, K - 1, D, dtype=x.dtype)
    for b in range(B):
        n = lengths[b]
        xe = torch.cat([state[b], x[b, :n]])
        ends[b] = xe[n:n + K - 1]
        if n:
            a = bias + sum(xe[k:k + n] * w[:, k] for k in range(K))
            m = bias.abs() + sum((xe[k:k + n] * w[:, k]).abs() for k in range(K))
            y[b, :n] = act(a, name)
            size[b, :n] = m + y[b, :n].abs() * (1 + a.abs())      # the exponential's argument is rounded: |a| 2^-24 relative
    return y, size, ends


def conv_bwd(x, w, bias, state, lengths, name, dy, dends):
    """Gradients dx, dw, dbias, dstate, each as (value, size)."""
    B, L, D = x.shape
    K = w.shape[1]
    dx, dst = (torch.zeros_like(x), torch.zeros_like(x)), (torch.zeros_like(state), torch.zeros_like(state))
    dw, db = (torch.zeros_like(w), torch.zeros_like(w)), (torch.zeros_like(bias), torch.zeros_like(bias))
    for b in range(B):
        n = lengths[b]
        xe = torch.cat([state[b], x[b, :n]])
        a = bias + sum(xe[k:k + n] * w[:, k] for k in range(K))
        m = bias.abs() + sum((xe[k:k + n] * w[:, k]).abs() for k in range(K))
        g = dy[b, :n] * slope(a, name)
        gs = dy[b, :n].abs() * ((1 if name != "none" else 0) * m + 2 + a.abs())      # |act''| <= 1
        de, des = torch.zeros_like(xe), torch.zeros_like(xe)
        for k in range(K):
            de[k:k + n] += g * w[:, k]
            des[k:k + n] += gs * w[:, k].abs()
            dw[0][:, k] += (g * xe[k:k + n]).sum(0)
            dw[1][:, k] += (gs * xe[k:k + n].abs()).sum(0)
        de[n:] += dends[b]
        des[n:] += dends[b].abs()
        db[0].add_(g.sum(0))
        db[1].add_(gs.sum(0))
        for i, v in enumerate((de, des)):
            dst[i][b], dx[i][b, :n] = v[:K - 1], v[K - 1:]
    return dx, dw, db, dst


# ------------------------------------------------------------------------------------------------------------------- scan

def _steps(delta, bias, soft):
    s = delta + bias
    return torch.nn.functional.softplus(s, threshold=700.0) if soft else s


def scan_fwd(u, delta, A, Bm, Cm, skip, z, bias, state, lengths, soft):
    """u, delta, z [B][L][D]; Bm, Cm [B][L][G][N].  Returns (y, size), (last state, size)."""
    B, L, D = u.shape
    G, N = Bm.shape[2:]
    s = _steps(delta, bias, soft)
    Be, Ce = Bm.repeat_interleave(D // G, 2), Cm.repeat_interleave(D // G, 2)
    y, ysize = torch.zeros_like(u), torch.zeros_like(u)
    h, hs = state.clone(), state.abs()
    for t in range(L):
        on = torch.tensor([t < n for n in lengths])[:, None, None]
        a = torch.exp(s[:, t, :, None] * A)
        b = (s[:, t] * u[:, t])[..., None] * Be[:, t]
        new = a * h + b
        # the step size and the exponential's argument are rounded: (1 + |s A|) a 2^-24 of what the state was
        news = a * (1 + (s[:, t, :, None] * A).abs()) * hs + b.abs()
        h, hs = torch.where(on, new, h), torch.where(on, news, hs)
        v = (Ce[:, t] * h).sum(-1) + skip * u[:, t]
        vs = (Ce[:, t].abs() * hs).sum(-1) + (skip * u[:, t]).abs()
        gate = act(z[:, t], "silu") if z is not None else torch.ones_like(v)
        gates = gate.abs() * (1 + z[:, t].abs()) if z is not None else gate
        y[:, t], ysize[:, t] = torch.where(on[..., 0], v * gate, 0), torch.where(on[..., 0], vs * gates, 0)
    return (y, ysize), (h, hs)


def scan_bwd(u, delta, A, Bm, Cm, skip, z, bias, state, lengths, soft, dy, dlast):
    """Gradients by name, each as (value, size), from the formulas walked backwards."""
    B, L, D = u.shape
    G, N = Bm.shape[2:]
    E = D // G
    s = _steps(delta, bias, soft)
    real = torch.arange(L)[None, :] < torch.tensor(lengths)[:, None]
    s = torch.where(real[..., None], s, 0)
    u = torch.where(real[..., None], u, 0)
    sig = torch.sigmoid(z) if z is not None else None
    gate = z * sig if z is not None else torch.ones_like(u)
    dy = torch.where(real[..., None], dy, 0)
    Bm, Cm = torch.where(real[..., None, None], Bm, 0), torch.where(real[..., None, None], Cm, 0)
    out = {}
    for which in (0, 1):
        if which:       # the same over absolute values; a factor for each rounded argument of an exponential
            grow = 1 + (s[..., None] * A).abs()
            decay = torch.exp(s[..., None] * A) * grow
            s_, u_, B_, C_, k_, A_, g_ = s.abs(), u.abs(), Bm.abs(), Cm.abs(), skip.abs(), A.abs(), (dy * gate).abs() * (1 + (z.abs() if z is not None else 0))
            h, e = state.abs(), dlast.abs()
        else:
            decay = torch.exp(s[..., None] * A)
            s_, u_, B_, C_, k_, A_, g_ = s, u, Bm, Cm, skip, A, dy * gate
            h, e = state.clone(), dlast.clone()
        Be, Ce = B_.repeat_interleave(E, 2), C_.repeat_interleave(E, 2)
        hist = [h]
        for t in range(L):
            h = decay[:, t] * h + (s_[:, t] * u_[:, t])[..., None] * Be[:, t]
            hist.append(h)
        r = {k: torch.zeros_like(u) for k in ("du", "ddelta", "dz")}
        r["dB"], r["dC"], r["dA"] = torch.zeros_like(Bm), torch.zeros_like(Cm), torch.zeros_like(A)
        r["dskip"] = (g_ * u_).sum((0, 1))
        for t in range(L - 1, -1, -1):
            v = (Ce[:, t] * hist[t + 1]).sum(-1) + k_ * u_[:, t]
            e = e + Ce[:, t] * g_[:, t, :, None]
            q = e * decay[:, t] * hist[t]
            eB = (e * Be[:, t]).sum(-1)
            r["dA"] += (q * s_[:, t, :, None]).sum(0)
            r["dC"][:, t] = (g_[:, t, :, None] * hist[t + 1]).reshape(B, G, E, N).sum(2)
            r["dB"][:, t] = (e * (s_[:, t] * u_[:, t])[..., None]).reshape(B, G, E, N).sum(2)
            r["du"][:, t] = s_[:, t] * eB + k_ * g_[:, t]
            r["ddelta"][:, t] = (q * A_).sum(-1) + u_[:, t] * eB
            if z is not None:
                ds = sig[:, t] * (1 + z[:, t] * (1 - sig[:, t]))
                r["dz"][:, t] = (dy[:, t].abs() * v * sig[:, t] * (1 + z[:, t].abs()) * (1 + z[:, t].abs())) if which else dy[:, t] * v * ds
            e = decay[:, t] * e
        if soft:
            r["ddelta"] *= torch.sigmoid(delta + bias) * ((1 + (delta + bias).abs()) if which else 1)
        for k in ("du", "ddelta", "dz"):
            r[k] = torch.where(real[..., None], r[k], 0)
        r["dbias"] = r["ddelta"].sum((0, 1))
        r["dstate"] = e
        for k, val in r.items():
            out.setdefault(k, []).append(val)
    return out


# ------------------------------------------------------------------------------------------------------------- group norm

def norm_fwd(x, gamma, beta, G, eps, name):
    """x [N][S][C].  Returns (y, size), (mean, size), (rstd, size), and x^ with its size."""
    N, S, C = x.shape
    xg = x.reshape(N, S, G, C // G)
    mean = xg.mean((1, 3), keepdim=True)
    var = ((xg - mean) ** 2).mean((1, 3), keepdim=True)
    rstd = (var + eps) ** -0.5
    xn = (xg - mean) * rstd
    # mean is known to 2^-24 of the largest element, the spread to 2^-24 of (largest element) * spread
    big = xg.abs().amax((1, 3), keepdim=True)
    xns = (big + xg.abs()) * rstd * (1 + xn.abs()) + xn.abs()
    v = xn * gamma.reshape(G, -1) + beta.reshape(G, -1)
    y = act(v, name)
    ys = 1.2 * (xns * gamma.abs().reshape(G, -1) + beta.abs().reshape(G, -1)) + y.abs() * (1 + v.abs())
    flat = lambda q: q.reshape(N, S, C)  # noqa: E731
    return (flat(y), flat(ys)), (mean.reshape(N, G), big.reshape(N, G)), (rstd.reshape(N, G), (rstd * (1 + big * rstd)).reshape(N, G)), (xn, xns, v)


def norm_bwd(x, gamma, beta, G, eps, name, dy):
    """(dx, size), (dgamma, size), (dbeta, size)."""
    N, S, C = x.shape
    _, _, (rstd, _), (xn, xns, v) = norm_fwd(x, gamma, beta, G, eps, name)
    rstd = rstd.reshape(N, 1, G, 1)
    g, dyg = gamma.reshape(G, -1), dy.reshape(N, S, G, C // G)
    d = dyg * slope(v, name)
    ds = dyg.abs() * (2 + v.abs() + (xns * g.abs() if name in ("silu", "gelu") else 0))
    if name == "relu":
        # the argument is known to 64 roundings of its terms (mean and spread, each a tree of sums, and four operations): where that
        # is more than the argument itself, rounding decides whether the slope is 0 or 1, and the term is off by all of |dy|
        unsure = v.abs() <= 64 * U * (xns * g.abs() + beta.reshape(G, -1).abs())
        ds = ds + torch.where(unsure, dyg.abs() / (64 * U), 0)
    dn, dns = d * g, ds * g.abs()
    m1, m2 = dn.mean((1, 3), keepdim=True), (dn * xn).mean((1, 3), keepdim=True)
    m1s = dns.mean((1, 3), keepdim=True)
    m2s = (dns * xn.abs() + dn.abs() * xns).mean((1, 3), keepdim=True)
    dx = rstd * (dn - m1 - xn * m2)
    dxs = rstd * (dns + m1s + xn.abs() * m2s + xns * m2.abs() + (dn.abs() + m1.abs() + (xn * m2).abs()) * (1 + xns.amax((1, 3), keepdim=True)))
    dgamma, dgs = (d * xn).sum((0, 1)), (ds * xn.abs() + d.abs() * xns).sum((0, 1))
    return ((dx.reshape(N, S, C), dxs.reshape(N, S, C)), (dgamma.reshape(C), dgs.reshape(C)), (d.sum((0, 1)).reshape(C), ds.sum((0, 1)).reshape(C)))
