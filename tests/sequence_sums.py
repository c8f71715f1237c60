"""Checks of whole tensors against the 64-bit forms, narrow enough that a lost row, part, segment or channel set shows.

A bound of so many roundings of the sum of absolute terms holds for every single value, but for sums of thousands of terms of either sign it is wider than the sum
itself.  Roundings are independent of each other, so the error of a whole tensor is smaller: with `units` of 2^-24 for each term and sqrt(n) for the n additions
of a sum it is that of a random walk, whose steps are roundings of partial sums; those are taken to be at most 8 times the result, as a root mean square over the
tensor.  So |got - ref| <= (half a step of the type) |ref| + (units + 8 sqrt(n)) 2^-24 |ref| in the 2-norm; where a result is a small difference of large
terms, their norm stands in the place of |ref|."""
from __future__ import annotations

import torch

import sequence_reference as ref
from sequence_reference import TYPES, U

F = torch.float64


def distance(got, want, units, scale=None):
    """|got - want| and what it may be."""
    info = torch.finfo(got.dtype)
    got, want = got.double().cpu().flatten(), want.double().cpu().flatten()
    by = float((want if scale is None else scale).norm())
    return float((got - want).norm()), info.eps / 2 * float(want.norm()) + units * U * by + info.tiny * want.numel() ** 0.5


def close(got, want, units, what, scale=None):
    off, allowed = distance(got, want, units, scale)
    assert off <= allowed, f"{what}: off by {off:.3e} in the 2-norm, allowed {allowed:.3e}, of {float(want.norm()):.3e}"


def values(seed, *shape, scale=1.0, shift=0.0, dtype=torch.float32):
    gen = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=gen) * scale + shift).to(dtype).to(F)


# ------------------------------------------------------------------------------------------------------------ convolution

CONV = [  # type, B, L, D, K, activation, lengths
    ("fp32", 2, 3000, 24, 4, "silu", None),
    ("bf16", 3, 1100, 72, 4, "silu", [1100, 7, 640]),
    ("fp16", 1, 2500, 33, 3, "gelu", None),
    ("fp32", 2, 19, 12, 8, "silu", [2, 19]),
    ("bf16", 40, 65, 130, 5, "none", None),
]


class Conv:
    def __init__(self, case, drop=None):
        self.type, self.B, self.L, self.D, self.K, self.act, lengths = case
        self.t = TYPES[self.type]
        self.n = [self.L] * self.B if lengths is None else lengths
        B, L, D, K, t = self.B, self.L, self.D, self.K, self.t
        self.x, self.w, self.bias = values(700, B, L, D, dtype=t), values(701, D, K, scale=0.6, dtype=t), values(702, D, scale=0.3, dtype=t)
        self.state, self.dy, self.dends = values(703, B, K - 1, D, dtype=t), values(704, B, L, D, dtype=t), values(705, B, K - 1, D, dtype=t)
        if drop is not None:
            self.dy[drop] = 0
        # K products and sums and an activation, twice
        self.units = {"y": 2 * K + 30, "dx": 4 * K + 60, "dstate": 4 * K + 60}
        for k in ("dw", "dbias"):
            self.units[k] = 4 * K + 60 + 8 * (B * L) ** 0.5
        self.sums = ("dw", "dbias")

    def reference(self):
        y, _, _ = ref.conv_fwd(self.x, self.w, self.bias, self.state, self.n, self.act)
        dx, dw, db, ds = ref.conv_bwd(self.x, self.w, self.bias, self.state, self.n, self.act, self.dy, self.dends)
        return {"y": y, "dx": dx[0], "dw": dw[0], "dbias": db[0], "dstate": ds[0]}

    def types(self):
        return {k: torch.float32 if k in self.sums else self.t for k in self.units}


# ------------------------------------------------------------------------------------------------------------------- scan

SCAN = [  # type, B, L, D, N, G, lengths
    ("fp32", 1, 4000, 24, 16, 1, None),                  # thousands of rows, cut into segments
    ("bf16", 3, 2100, 32, 16, 2, [2100, 0, 1333]),
    ("fp32", 1, 90, 4, 100, 1, [89]),
    ("fp32", 2, 70, 10, 20, 2, None),
    ("fp16", 4, 300, 70, 32, 1, None),
    ("bf16", 2, 2000, 64, 64, 1, [2000, 1500]),          # four channel sets a block and segments, as the sizes decide
    ("fp32", 20, 40, 128, 64, 1, None),                  # four channel sets a block, whole
    ("fp32", 20, 40, 100, 128, 1, None),
]
SETS = [  # with four channel sets a block asked for: 32 channels (16 with more than 64 states) a block, the last one with 1, 2 or 3 sets, one partly filled
    ("fp32", 2, 70, 37, 64, 1, [70, 33]),
    ("bf16", 1, 100, 2 * 43, 40, 2, None),
    ("fp32", 2, 50, 49, 64, 1, None),
    ("fp32", 3, 40, 64, 33, 1, [40, 0, 17]),
    ("fp32", 1, 64, 3 * 18, 100, 3, None),
    ("fp16", 2, 37, 23, 128, 1, [36, 37]),
    ("fp32", 1, 33, 27, 65, 1, None),
    ("bf16", 2, 50, 100, 20, 1, [50, 49]),
]


class Scan:
    def __init__(self, case, drop=None):
        self.type, self.B, self.L, self.D, self.N, self.G, lengths = case
        self.t, B, L, D, N, G = TYPES[self.type], *case[1:6]
        self.n = [L] * B if lengths is None else lengths
        t = self.t
        self.u, self.z, self.delta = values(710, B, L, D, dtype=t), values(711, B, L, D, dtype=t), values(712, B, L, D, scale=0.7, dtype=t)
        self.bias, self.A = values(713, D, scale=0.3, shift=-2.0), -torch.exp(values(714, D, N, scale=0.7)).float().to(F)
        self.Bm, self.Cm = values(715, B, L, G, N, dtype=t), values(716, B, L, G, N, dtype=t)
        self.skip, self.state, self.dy, self.dlast = values(717, D), values(718, B, D, N), values(719, B, L, D, dtype=t), values(720, B, D, N)
        if drop is not None:
            self.dy[drop] = 0
        # A step is off by 8 units (decay, its argument, two products, a sum); states and what is carried back remember 100 rows at most, as steps are 0.1 and more
        # and A is -0.1 and below: 80 for either, 40 for step sizes, gates and outputs
        many = 200
        self.units = {k: many + 8 * N ** 0.5 for k in ("y", "state", "du", "ddelta", "dz", "dstate")}
        for k in ("dB", "dC"):
            self.units[k] = many + 8 * (D // G) ** 0.5
        for k in ("dA", "dskip", "dbias"):
            self.units[k] = many + 8 * (B * L + N) ** 0.5
        self.sums = ("dA", "dskip", "dbias")

    def inputs(self):
        return self.u, self.delta, self.A, self.Bm, self.Cm, self.skip, self.z, self.bias, self.state, self.n, True

    def reference(self):
        (y, _), (h, _) = ref.scan_fwd(*self.inputs())
        out = {k: v[0] for k, v in ref.scan_bwd(*self.inputs(), self.dy, self.dlast).items()}
        return {"y": y, "state": h, **out}

    def types(self):
        return {k: torch.float32 if k in self.sums + ("state", "dstate") else self.t for k in self.units}


# ------------------------------------------------------------------------------------------------------------- group norm

NORM = [  # type, N, S, C, G, activation, shift of the mean
    ("fp32", 3, 1, 32, 4, "silu", 0.5),
    ("bf16", 70, 1, 96, 3, "none", 0.5),
    ("bf16", 9, 1, 4096, 1, "gelu", 0.0),
    ("fp32", 2, 1, 20000, 1, "silu", 0.0),
    ("fp16", 3, 200, 40, 4, "gelu", -2.0),
    ("fp32", 1, 1000, 36, 9, "relu", 0.5),
    ("fp32", 2, 333, 300, 30, "silu", 0.0),
    ("bf16", 1, 4000, 512, 2, "silu", 0.3),
    ("fp32", 1, 30000, 24, 1, "silu", 0.0),
    ("bf16", 2, 3, 2304, 1, "none", 0.0),
    ("fp32", 1, 50, 16, 2, "none", 1000.0),
    ("fp16", 300, 49, 80, 8, "silu", 0.5),
    ("fp32", 2500, 1, 64, 4, "gelu", 0.2),
    ("fp32", 600, 2, 64, 4, "silu", 0.2),
]


class Norm:
    eps = 1e-5

    def __init__(self, case, drop=None):
        self.type, self.N, self.S, self.C, self.G, self.act, shift = case
        self.t, N, S, C, G = TYPES[self.type], *case[1:5]
        self.x = values(730, N, S, C, shift=shift, dtype=self.t)
        self.gamma, self.beta, self.dy = values(731, C, scale=0.3, shift=1.0), values(732, C, scale=0.3), values(733, N, S, C, dtype=self.t)
        if self.act == "relu":      # where rounding decides on which side of zero an argument lies, the slope is anything: no gradient comes in there
            v = ref.norm_fwd(self.x, self.gamma, self.beta, G, self.eps, "none")[0][0]
            self.dy[v.abs() < 1e-4] = 0
        if drop is not None:
            self.dy[drop] = 0
        # mean and spread are trees over chains of at most S C / G additions; 60 for the operations of an element; the mean itself is rounded, after a few
        # operations on values of its size: 8 |shift| of an element's spread
        near = 60 + 8 * (S * C // G) ** 0.5 + 8 * abs(shift)
        self.units = {"y": near, "mean": near, "rstd": near, "dx": 3 * near, "dgamma": 2 * near + 8 * (N * S) ** 0.5, "dbeta": 2 * near + 8 * (N * S) ** 0.5}
        self.sums = ("dgamma", "dbeta")

    def reference(self):
        (y, _), (m, _), (r, _), _ = ref.norm_fwd(self.x, self.gamma, self.beta, self.G, self.eps, self.act)
        dx, dg, db = ref.norm_bwd(self.x, self.gamma, self.beta, self.G, self.eps, self.act, self.dy)
        return {"y": y, "mean": m, "rstd": r, "dx": dx[0], "dgamma": dg[0], "dbeta": db[0]}

    def scales(self, want):
        """mean: of values of either sign, its error is that of the values."""
        return {"mean": want["mean"].abs() + 1 / want["rstd"]}

    def types(self):
        return {k: torch.float32 if k in self.sums + ("mean", "rstd") else self.t for k in self.units}


def rows_of(c):
    """Some rows that hold a token: the last, the first and one in between (of large cases the last)."""
    if isinstance(c, Norm):
        return [(c.N - 1, c.S - 1), (0, 0), (c.N // 2, c.S // 3)]
    b = max(range(c.B), key=lambda i: c.n[i])
    rows = [(b, c.n[b] - 1), (b, 0), (b, c.n[b] // 2)]
    return rows[:1] if c.L >= 1000 else rows
