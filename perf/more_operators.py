"""Workloads of the operators of a recurrent language model's layer: RMS norm with the residual's addition, a gate and an output in 8 bits,
and the gated delta rule over prompts, single tokens and training steps.

A case is a dict with
  op     "norm" | "delta"
  mode   "prompt" (forward; the delta rule leaves the state that single tokens continue from), "step" (one token of every sequence),
         "train" (forward and backward)
  type   "bf16" | "fp16" | "fp32"
  norm   M rows of C channels in G groups, each normalised by itself; residual, gate: whether there is one; block: columns that share a scale
         of the output in 8 bits (0: output of the type)
  delta  B L, Hk heads of queries and keys, H heads of values, K and V their lengths, ragged (sequences of different lengths in one padded batch)
"""
import math

import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
_BYTES = {"bf16": 2, "fp16": 2, "fp32": 4}
_EPS = 1e-6
_CHUNK = 64


def _norm(mode, type, M, C, G=1, residual=True, gate=False, block=0, **kw):
    return dict(op="norm", mode=mode, type=type, M=M, C=C, G=G, residual=residual, gate=gate, block=block, **kw)


def _delta(mode, type, B, L, Hk, H, K, V, ragged=False, **kw):
    return dict(op="delta", mode=mode, type=type, B=B, L=L, Hk=Hk, H=H, K=K, V=V, ragged=ragged, **kw)


def listed():
    return [
        # the entry of a layer for a few conversations, its projection in 8 bits: all launch latency
        _norm("step", "bf16", 8, 4096, block=128, name="norm_step"),
        # the entry of a layer for prompts, one scale a token
        _norm("prompt", "bf16", 8192, 4096, block=4096, name="norm_prompt"),
        # the entry of a layer in a training step
        _norm("train", "bf16", 16384, 2048, name="norm_train"),
        # the exit of the mixer in a training step: every head by itself, with its gate, rows off every tile
        _norm("train", "fp16", 4111, 2304, G=18, residual=False, gate=True, name="norm_heads_train"),
        # decoding for a few users
        _delta("step", "bf16", 4, 1, 16, 32, 128, 128, name="delta_step"),
        # decoding for a full server: every state is read and written once
        _delta("step", "bf16", 256, 1, 16, 32, 128, 128, name="delta_step_many"),
        # prompts of different lengths in one padded batch
        _delta("prompt", "fp16", 3, 1917, 8, 16, 128, 128, ragged=True, name="delta_prompt_ragged"),
        # one long document
        _delta("prompt", "bf16", 1, 16384, 16, 32, 128, 128, name="delta_prompt_long"),
        # a layer of a training step
        _delta("train", "bf16", 4, 2048, 16, 16, 128, 128, name="delta_train"),
        # a small model in full precision: shared heads, sizes off every tile
        _delta("train", "fp32", 2, 777, 2, 6, 60, 90, name="delta_train_odd"),
        # a short training step of a small model
        _delta("train", "fp16", 2, 500, 4, 8, 64, 64, name="delta_train_small"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _extent(rng, lo, hi):
    """A size of the range, a multiple of 64, of 8 or of nothing."""
    n, unit = _log(rng, lo, hi), rng.choice((64, 8, 1))
    return max(lo, n // unit * unit)


def draw(rng):
    type = rng.choice(("bf16", "bf16", "fp16", "fp32"))
    mode = rng.choice(("prompt", "step", "train"))
    if rng.random() < 0.4:
        block, residual, gate = 0, rng.random() < 0.6, rng.random() < 0.3
        G = 1 if rng.random() < 0.6 else rng.choice((2, 6, 16, 32))
        C = G * _extent(rng, 64 if G == 1 else 16, 8192 if G == 1 else 256)
        if mode != "train" and type != "fp32" and rng.random() < 0.5:
            block = rng.choice((C, 128, 128))
        M = _log(rng, 1, 256) if mode == "step" else max(1, min(_log(rng, 1, 16384), ((8 if type == "fp32" else 16) << 20) // C))
        return _norm(mode, type, M, C, G=G, residual=residual, gate=gate, block=block)
    K, V = rng.choice((16, 32, 64, 64, 128, 128, rng.randint(5, 128))), rng.choice((16, 64, 64, 128, 128, 256, rng.randint(3, 256)))
    Hk = _log(rng, 1, 16)
    H = Hk * rng.choice((1, 1, 2, 3))
    B = _log(rng, 1, 256 if mode == "step" else 8)
    if mode == "step":
        B = max(1, min(B, (128 << 20) // (H * K * V)))
        return _delta(mode, type, B, 1, Hk, H, K, V)
    most = {"prompt": 64, "train": 16}[mode] << 20              # elements of the values; in fp32 half
    L = max(1, min(_log(rng, 1, 16384), (most >> (type == "fp32")) // (B * H * max(K, V))))
    return _delta(mode, type, B, L, Hk, H, K, V, ragged=mode == "prompt" and rng.random() < 0.5)


# ---------------------------------------------------------------------------------------------------------------- inputs

def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    t = _TYPES[case["type"]]

    def normal(*shape, scale=1.0, shift=0.0, dtype=t):
        return torch.empty(shape, device="cuda").normal_(generator=gen).mul_(scale).add_(shift).to(dtype)

    def unit(*shape):
        return torch.empty(shape, device="cuda").uniform_(generator=gen)

    s = dict(case=case)
    train = case["mode"] == "train"
    if case["op"] == "norm":
        M, C, G = case["M"], case["C"], case["G"]
        s["x"] = normal(M, C)
        # the residual of a deep layer, a few channels of it much larger than the others
        s["residual"] = (normal(M, C, scale=2.0, dtype=torch.float32) * torch.exp(normal(C, dtype=torch.float32))).to(t) if case["residual"] else None
        s["z"] = normal(M, C) if case["gate"] else None
        s["gamma"] = normal(C // G, scale=0.2, shift=1.0, dtype=torch.float32)
        s["h"] = torch.empty_like(s["x"]) if case["residual"] else None
        s["rstd"] = torch.empty(M, G, device="cuda")
        s["y"] = s["y8"] = s["scales"] = None
        if case["block"]:
            s["y8"] = torch.empty(M, C, dtype=torch.float8_e4m3fn, device="cuda")
            s["scales"] = torch.empty(M, -(-C // case["block"]), device="cuda")
        else:
            s["y"] = torch.empty_like(s["x"])
        if train:
            s["dy"] = normal(M, C)
            s["dh"] = normal(M, C) if case["residual"] else None
            s["dx"], s["dgamma"] = torch.empty_like(s["x"]), torch.empty(C // G, device="cuda")
            s["dz"] = torch.empty_like(s["x"]) if case["gate"] else None
        return s
    B, L, Hk, H, K, V = (case[n] for n in ("B", "L", "Hk", "H", "K", "V"))
    step = case["mode"] == "step"
    rows = (B,) if step else (B, L)

    def direction(x):
        return (x / x.square().sum(-1, keepdim=True).add_(_EPS).sqrt_()).to(t)

    s["lengths"] = None
    if case["ragged"]:
        s["lengths"] = (unit(B) * L).floor().add_(1).clamp_(max=L).to(torch.int32)
        s["lengths"][0] = L
    s["q"], s["k"] = (direction(normal(*rows, Hk, K, dtype=torch.float32)) for _ in range(2))
    s["v"] = normal(*rows, H, V)
    # log decays: rates of 1 to 16 by steps of 0.001 to 0.1, moved by the token
    rate, dt = 1 + 15 * unit(H), torch.exp(unit(H) * (math.log(0.1) - math.log(0.001)) + math.log(0.001))
    s["g"] = -rate * torch.log1p(torch.exp(normal(*rows, H, dtype=torch.float32) + dt + torch.log(-torch.expm1(-dt))))
    s["beta"] = 1 / (1 + torch.exp(-normal(*rows, H, dtype=torch.float32)))
    s["state"] = normal(B, H, K, V, scale=0.3, dtype=torch.float32) if step else None
    s["o"] = torch.empty_like(s["v"])
    s["state_out"] = None if train else torch.empty(B, H, K, V, device="cuda")
    if train:
        s["do"] = normal(*rows, H, V)
        for name in ("q", "k", "v", "g", "beta"):
            s["d" + name] = torch.empty_like(s[name])
    return s


# --------------------------------------------------------------------------------------------------- the framework's calls

def _p(x):
    return 0 if x is None else x.data_ptr()


def _kept(s, name, nbytes):
    """A buffer that a program keeps between calls of one size."""
    if name not in s:
        s[name] = torch.empty(max(nbytes, 16), dtype=torch.uint8, device="cuda")
    return s[name].data_ptr()


def _own(s):
    import paper_1705_10591_b200 as lib

    c = s["case"]
    stream = torch.cuda.current_stream().cuda_stream
    type = {"bf16": lib.OPERAND_BF16, "fp16": lib.OPERAND_FP16, "fp32": lib.OPERAND_FP32}[c["type"]]
    train = c["mode"] == "train"
    if c["op"] == "norm":
        M, C, G = c["M"], c["C"], c["G"]
        lib.norm_fwd_rms(_p(s["x"]), _p(s["residual"]), _p(s["z"]), _p(s["gamma"]), _p(s["y"]), _p(s["h"]), _p(s["y8"]), _p(s["scales"]),
                         _p(s["rstd"]) if train else 0, M, C, G, c["block"], C, C, C, C, C, C, _EPS, type, stream)
        if not train:
            return tuple(s[n] for n in ("y", "y8", "scales", "h") if s[n] is not None)
        if "ws_bytes" not in s:
            s["ws_bytes"] = lib.norm_bwd_rms_workspace_size(M, C, G)
        n = s["ws_bytes"]
        lib.norm_bwd_rms(_p(s["h"] if c["residual"] else s["x"]), _p(s["z"]), _p(s["gamma"]), _p(s["rstd"]), _p(s["dy"]), _p(s["dh"]), _p(s["dx"]),
                         _p(s["dz"]), _p(s["dgamma"]), M, C, G, C, C, C, C, C, C, type, _kept(s, "ws", n), n, stream)
        return tuple(s[n] for n in ("y", "h", "dx", "dz", "dgamma") if s[n] is not None)
    B, L, Hk, H, K, V = (c[n] for n in ("B", "L", "Hk", "H", "K", "V"))
    scale = K ** -0.5
    if c["mode"] == "step":
        lib.delta_step_gated(_p(s["q"]), _p(s["k"]), _p(s["v"]), _p(s["g"]), _p(s["beta"]), _p(s["state"]), _p(s["o"]), _p(s["state_out"]),
                             B, Hk, H, K, V, Hk * K, Hk * K, H * V, H, H, H * V, scale, type, stream)
        return s["o"], s["state_out"]
    if "ws_bytes" not in s:
        s["ws_bytes"] = lib.delta_fwd_gated_workspace_size(B, L, Hk, H, K, V, type)
        if train:
            s["ws_bytes"] = max(s["ws_bytes"], lib.delta_bwd_gated_workspace_size(B, L, Hk, H, K, V, type))
            s["kept_bytes"] = lib.delta_states_size(B, L, Hk, H, K, V, type)
    n = s["ws_bytes"]
    ws, kept = _kept(s, "ws", n), _kept(s, "kept", s["kept_bytes"]) if train else 0
    lib.delta_fwd_gated(_p(s["q"]), _p(s["k"]), _p(s["v"]), _p(s["g"]), _p(s["beta"]), 0, _p(s["lengths"]), _p(s["o"]), _p(s["state_out"]), kept,
                        B, L, Hk, H, K, V, Hk * K, Hk * K, H * V, H, H, H * V, scale, type, ws, n, stream)
    if not train:
        return s["o"], s["state_out"]
    lib.delta_bwd_gated(_p(s["q"]), _p(s["k"]), _p(s["lengths"]), kept, _p(s["do"]), 0, _p(s["dq"]), _p(s["dk"]), _p(s["dv"]), _p(s["dg"]),
                        _p(s["dbeta"]), 0, B, L, Hk, H, K, V, Hk * K, Hk * K, H * V, Hk * K, Hk * K, H * V, H, H, scale, type, ws, n, stream)
    return (s["o"],) + tuple(s["d" + name] for name in ("q", "k", "v", "g", "beta"))


# --------------------------------------------------------------------------------------------------------- the plain forms

def _plain_norm(s):
    c = s["case"]
    M, C, G, t = c["M"], c["C"], c["G"], _TYPES[c["type"]]
    h = s["x"] if s["residual"] is None else (s["x"].float() + s["residual"].float()).to(t)
    x = h.float().reshape(M, G, C // G)
    rstd = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + _EPS)
    xn = x * rstd
    n = xn * s["gamma"]
    gate = 1.0
    if s["z"] is not None:
        z = s["z"].float().reshape(M, G, C // G)
        sig = 1 / (1 + torch.exp(-z))
        gate = z * sig
    y = (n * gate).reshape(M, C)
    if c["block"]:
        blocks = -(-C // c["block"])
        padded = torch.cat([y, y.new_zeros(M, blocks * c["block"] - C)], dim=1).reshape(M, blocks, -1)
        scales = (padded.abs().amax(-1) / 448).clamp(min=2.0 ** -126)
        y8 = (padded / scales[..., None]).reshape(M, -1)[:, :C].to(torch.float8_e4m3fn)
        return (y8, scales) + (() if s["residual"] is None else (h,))
    if c["mode"] != "train":
        return (y.to(t),) + (() if s["residual"] is None else (h,))
    dy = s["dy"].float().reshape(M, G, C // G)
    dn = dy * gate * s["gamma"]
    dx = rstd * (dn - xn * (dn * xn).mean(-1, keepdim=True)).reshape(M, G, -1)
    dx = dx.reshape(M, C)
    if s["residual"] is not None:
        dx = dx + s["dh"].float()
    out = (y.to(t),) + (() if s["residual"] is None else (h,)) + (dx.to(t),)
    if s["z"] is not None:
        out += ((dy * n * sig * (1 + z * (1 - sig))).reshape(M, C).to(t),)
    return out + ((dy * gate * xn).sum((0, 1), dtype=torch.float64).float(),)


def _compose(m, n):
    """S_c = m_c S_{c-1} + n_c along dimension 2, from zero: neighbours are joined to a sequence of half the length, which gives every second
    value; the others follow from those."""
    L = m.shape[2]
    if L == 1:
        return n
    half = L // 2
    odd = _compose(m[:, :, 1::2] @ m[:, :, 0:2 * half:2], m[:, :, 1::2] @ n[:, :, 0:2 * half:2] + n[:, :, 1::2])
    S = torch.empty_like(n)
    S[:, :, 1::2] = odd
    S[:, :, 0] = n[:, :, 0]
    S[:, :, 2::2] = m[:, :, 2::2] @ odd[:, :, :(L - 1) // 2] + n[:, :, 2::2]
    return S


def _inverse(a):
    """(1 + a)^-1 of strictly lower triangular matrices, by halves."""
    n = a.shape[-1]
    if n == 1:
        return torch.ones_like(a)
    m = n // 2
    first, last = _inverse(torch.stack([a[..., :m, :m], a[..., m:, m:]])).unbind(0)
    top = torch.cat([first, torch.zeros_like(a[..., :m, m:])], dim=-1)
    return torch.cat([top, torch.cat([-last @ (a[..., m:, :m] @ first), last], dim=-1)], dim=-2)


def _plain_step(s):
    c = s["case"]
    t, share = _TYPES[c["type"]], c["H"] // c["Hk"]
    q, k = (s[n].float().repeat_interleave(share, dim=1)[..., None] for n in ("q", "k"))
    S = s["state"] * torch.exp(s["g"])[..., None, None]
    u = s["beta"][..., None] * (s["v"].float() - (S * k).sum(2))
    S = S + k * u[:, :, None]
    return ((S * q).sum(2) * c["K"] ** -0.5).to(t), S


def _plain_delta(s):
    c = s["case"]
    B, L, H, K, V, t = c["B"], c["L"], c["H"], c["K"], c["V"], _TYPES[c["type"]]
    share, scale = H // c["Hk"], K ** -0.5
    n = -(-L // _CHUNK)
    real = torch.ones((B, L), dtype=torch.bool, device="cuda")
    if s["lengths"] is not None:
        real = torch.arange(L, device="cuda")[None] < s["lengths"][:, None]

    def chunks(x, heads):                                       # [B][H][chunks][tokens][..], zero behind the sequences
        x = torch.where(real.reshape(B, L, *(1,) * (x.dim() - 2)), x, torch.zeros((), dtype=x.dtype, device="cuda")).float()
        x = torch.cat([x, x.new_zeros(B, n * _CHUNK - L, *x.shape[2:])], dim=1).reshape(B, n, _CHUNK, *x.shape[2:])
        return x.transpose(2, 3).transpose(1, 2).repeat_interleave(H // heads, dim=1)

    def rows(x, heads, type):                                   # back, the heads that share one summed
        x = x.reshape(B, heads, H // heads, *x.shape[2:]).sum(2)
        x = x.transpose(1, 2).transpose(2, 3).reshape(B, n * _CHUNK, heads, *x.shape[4:])[:, :L]
        return torch.where(real.reshape(B, L, *(1,) * (x.dim() - 2)), x, torch.zeros((), device="cuda")).to(type)

    q, k, v = chunks(s["q"], c["Hk"]), chunks(s["k"], c["Hk"]), chunks(s["v"], H)
    beta = chunks(s["beta"], H)[..., None]
    G = torch.cumsum(chunks(s["g"], H).double(), dim=-1)
    low = torch.ones(_CHUNK, _CHUNK, dtype=torch.bool, device="cuda").tril()
    decay = torch.exp(torch.where(low, G[..., :, None] - G[..., None, :], -torch.inf)).float()
    begin, end = torch.exp(G).float()[..., None], torch.exp(G[..., -1:] - G).float()[..., None]
    whole = begin[..., -1:, :]
    A = decay.tril(-1) * (k @ k.mT)
    T = _inverse(A * beta.mT)
    W, X = T @ (begin * k), T @ v
    kd = end * k
    m = whole * torch.eye(K, device="cuda") - (beta * kd).mT @ W
    after = _compose(m, (beta * kd).mT @ X)
    S = torch.cat([torch.zeros_like(after[:, :, :1]), after[:, :, :-1]], dim=2)
    E = X - W @ S
    U = beta * E
    P = decay * (q @ k.mT)
    o = scale * (begin * (q @ S) + P @ U)
    if c["mode"] != "train":
        return rows(o, H, t), after[:, :, -1]
    do = chunks(s["do"], H) * scale
    # the gradient of the state behind each chunk: the same recurrence from the other end
    into = (begin * q).mT @ do - W.mT @ (beta * (P.mT @ do))
    dS = _compose(m.mT.flip(2), into.flip(2)).flip(2)           # of the state before each chunk
    dS = torch.cat([dS[:, :, 1:], torch.zeros_like(dS[:, :, :1])], dim=2)
    del m, into
    dU = P.mT @ do + kd @ dS
    dv = T.mT @ (beta * dU)
    dbeta = ((dU - A.mT @ dv) * E).sum(-1)
    p, y = decay * (do @ U.mT), decay.tril(-1) * -(dv @ U.mT)
    dq = begin * (do @ S.mT) + p @ k
    plus, minus = y @ k - begin * (dv @ S.mT), p.mT @ q + y.mT @ k + end * (U @ dS.mT)
    dG = (q * dq + k * plus - k * minus).sum(-1, dtype=torch.float64)
    dg = dG.flip(-1).cumsum(-1).flip(-1) + (after * dS).sum((-1, -2), dtype=torch.float64)[..., None]
    return (rows(o, H, t), rows(dq, c["Hk"], t), rows(plus + minus, c["Hk"], t), rows(dv, H, t), rows(dg, H, torch.float32),
            rows(dbeta, H, torch.float32))


def run(s):
    if own:
        return _own(s)
    if s["case"]["op"] == "norm":
        return _plain_norm(s)
    return _plain_step(s) if s["case"]["mode"] == "step" else _plain_delta(s)


# -------------------------------------------------------------------------------------------------------------- yardsticks

def work(case):
    size = _BYTES[case["type"]]
    train = case["mode"] == "train"
    if case["op"] == "norm":
        n, M, C, G = case["M"] * case["C"], case["M"], case["C"], case["G"]
        tensors = 2 + 2 * case["residual"] + case["gate"]               # x, y; the residual before and after; the gate
        if train:                                                       # dy, dx; the gradients of the sum and of the gate
            tensors += 2 + case["residual"] + case["gate"]
            return {"bytes": n * tensors * size + 8 * C // G, "flops": n * (16 + 12 * case["gate"])}
        if case["block"]:
            return {"bytes": n * ((tensors - 1) * size + 1) + 4 * M * -(-C // case["block"]) + 4 * C // G, "flops": n * (8 + 5 * case["gate"])}
        return {"bytes": n * tensors * size + 4 * C // G, "flops": n * (5 + 5 * case["gate"])}
    B, L, Hk, H, K, V = (case[n] for n in ("B", "L", "Hk", "H", "K", "V"))
    tokens, state = B * L, 4 * B * H * K * V
    qk, vo, gates = tokens * Hk * K * size, tokens * H * V * size, 8 * tokens * H
    if case["mode"] == "step":
        return {"bytes": 2 * qk + 2 * vo + gates + 2 * state, "flops": 7 * tokens * H * K * V}
    # token by token: decay, product with the key, update, product with the query
    flops = 7 * tokens * H * K * V
    if train:                                                           # q, k, v, do and three gradients; o; gates and theirs
        return {"bytes": 4 * qk + 4 * vo + 2 * gates, "flops": 3 * flops}
    return {"bytes": 2 * qk + 2 * vo + gates + state, "flops": flops}


def exact(case, seed):
    """The definitions in 64 bits, token by token; gradients by automatic differentiation of them."""
    s = prepare(case, seed)
    c, f, t = case, torch.float64, _TYPES[case["type"]]
    train = c["mode"] == "train"

    def leaf(x):
        return x.to(f).requires_grad_(train)

    if c["op"] == "norm":
        M, C, G = c["M"], c["C"], c["G"]
        h = s["x"]
        if c["residual"]:
            h = (s["x"].to(f) + s["residual"].to(f)).to(t)
        x, gamma = leaf(h), leaf(s["gamma"])
        y = x.reshape(M, G, C // G)
        y = y * (y.pow(2).sum(-1, keepdim=True) / (C // G) + _EPS).rsqrt() * gamma
        z = None
        if c["gate"]:
            z = leaf(s["z"])
            y = y * torch.nn.functional.silu(z.reshape(M, G, C // G))
        y = y.reshape(M, C)
        sums = (h.to(f),) if c["residual"] else ()
        if c["block"]:
            scales = torch.stack([b.abs().amax(1) for b in y.split(c["block"], dim=1)], dim=1).div(448).clamp(min=2.0 ** -126)
            codes = y / scales.repeat_interleave(c["block"], dim=1)[:, :C]
            return (codes.float().to(torch.float8_e4m3fn).to(f), scales) + sums
        if not train:
            return (y,) + sums
        grads = torch.autograd.grad(y, (x, gamma) + ((z,) if c["gate"] else ()), s["dy"].to(f))
        dx = grads[0] + s["dh"].to(f) if c["residual"] else grads[0]
        return (y.detach(),) + sums + (dx,) + grads[2:] + (grads[1],)

    B, L, Hk, H, K, V = (c[n] for n in ("B", "L", "Hk", "H", "K", "V"))
    if B * L * H * K * V > (1 << 31 if train else 1 << 34):
        return None
    scale, share = K ** -0.5, H // Hk
    S = torch.zeros(B, H, K, V, dtype=f, device="cuda") if s["state"] is None else s["state"].to(f)
    q, k, v, g, beta = (s[n].to(f).reshape(B, L, *s[n].shape[1 if c["mode"] == "step" else 2:]) for n in ("q", "k", "v", "g", "beta"))

    def token(S, q, k, v, g, beta):
        q, k = q.repeat_interleave(share, dim=1), k.repeat_interleave(share, dim=1)
        S = S * g.exp()[..., None, None]
        u = beta[..., None] * (v - torch.einsum("bhkv,bhk->bhv", S, k))
        S = S + k[..., None] * u[..., None, :]
        return S, scale * torch.einsum("bhkv,bhk->bhv", S, q)

    if not train:
        o = torch.zeros(B, L, H, V, dtype=f, device="cuda")
        ends = torch.full((B,), L, device="cuda") if s["lengths"] is None else s["lengths"]
        for i in range(L):
            alive = (ends > i)[:, None, None, None]
            new, out = token(S, q[:, i], k[:, i], v[:, i], g[:, i], beta[:, i])
            S = torch.where(alive, new, S)
            o[:, i] = torch.where(alive[..., 0], out, 0)
        return o.reshape(s["v"].shape), S
    # differentiated in pieces of the sequence, from the last one back, so that one piece's graph is held at a time
    piece = max(1, (1 << 29) // (B * H * K * V))

    def through(S, *x):
        outs = []
        for i in range(x[0].shape[1]):
            S, out = token(S, *(y[:, i] for y in x))
            outs.append(out)
        return S, torch.stack(outs, dim=1)

    pieces, outs = [], []
    for lo in range(0, L, piece):
        x = [y[:, lo:lo + piece].detach().requires_grad_() for y in (q, k, v, g, beta)]
        pieces.append((S, x, s["do"][:, lo:lo + piece].to(f)))
        with torch.no_grad():
            S, o = through(S, *x)
        outs.append(o)
    back, parts = torch.zeros_like(S), []
    for S0, x, do in reversed(pieces):
        with torch.enable_grad():
            S0 = S0.detach().requires_grad_()
            S1, o = through(S0, *x)
            grads = torch.autograd.grad((o, S1), tuple(x) + (S0,), (do, back))
        parts.insert(0, grads[:5])
        back = grads[5]
    return (torch.cat(outs, dim=1),) + tuple(torch.cat(x, dim=1) for x in zip(*parts))
