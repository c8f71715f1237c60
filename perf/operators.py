"""Workloads of the sequence operators: short causal convolution, selective state space scan, group norm with an activation.

All tensors are channels last.  A case is a dict with
  op     "conv" | "scan" | "norm"
  mode   "prompt" (forward over whole sequences, with the state that single tokens continue from), "step" (one token of every
         sequence), "train" (forward and backward), "apply" (forward of the norm)
  type   "bf16" | "fp16" | "fp32"
  conv   B L D K, act, ragged (sequences of different lengths in one padded batch)
  scan   B L D N G, ragged
  norm   N S C G, act
"""
import math

import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
_BYTES = {"bf16": 2, "fp16": 2, "fp32": 4}
_EPS = 1e-5


def _conv(mode, type, B, L, D, K, act="silu", ragged=False, **kw):
    return dict(op="conv", mode=mode, type=type, B=B, L=L, D=D, K=K, act=act, ragged=ragged, **kw)


def _scan(mode, type, B, L, D, N, G=1, ragged=False, **kw):
    return dict(op="scan", mode=mode, type=type, B=B, L=L, D=D, N=N, G=G, ragged=ragged, **kw)


def _norm(mode, type, N, S, C, G, act="silu", **kw):
    return dict(op="norm", mode=mode, type=type, N=N, S=S, C=C, G=G, act=act, **kw)


def listed():
    return [
        # one token for each of a few conversations: all launch latency
        _conv("step", "bf16", 8, 1, 4096, 4, name="conv_step"),
        # prompts of different lengths in one padded batch, channels that no power of two divides
        _conv("prompt", "fp16", 3, 1083, 1928, 4, ragged=True, name="conv_prompt_ragged"),
        # a layer of a training step on long sequences
        _conv("train", "bf16", 4, 4096, 4096, 4, name="conv_train"),
        # decoding for a few users: the state is read and written once
        _scan("step", "bf16", 8, 1, 4096, 16, name="scan_step"),
        # decoding for a full server
        _scan("step", "bf16", 256, 1, 4096, 16, name="scan_step_many"),
        # prompts of different lengths in one padded batch
        _scan("prompt", "bf16", 3, 1917, 2048, 16, ragged=True, name="scan_prompt_ragged"),
        # one long document
        _scan("prompt", "bf16", 1, 16384, 4096, 16, name="scan_prompt_long"),
        # a layer of a training step
        _scan("train", "bf16", 4, 2048, 2048, 16, name="scan_train"),
        # a small model in full precision: grouped inputs of the state, sizes off every tile
        _scan("train", "fp32", 2, 777, 300, 20, G=3, name="scan_train_odd"),
        # the heads of a token mixer, normalised per token
        _norm("apply", "bf16", 8192, 1, 4096, 32, act="none", name="norm_tokens"),
        # feature maps between the convolutions of a decoder of images
        _norm("apply", "fp16", 8, 64 * 64, 512, 32, name="norm_maps"),
        # a layer of a training step on the feature maps of an image network
        _norm("train", "bf16", 32, 56 * 56, 256, 32, name="norm_train"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _extent(rng, lo, hi):
    """A size of the range, a multiple of 64, of 8 or of nothing."""
    n, unit = _log(rng, lo, hi), rng.choice((64, 8, 1))
    return max(lo, n // unit * unit)


def draw(rng):
    type = rng.choice(("bf16", "bf16", "fp16", "fp32"))
    op = rng.choice(("conv", "scan", "norm"))
    if op == "conv":
        mode = rng.choice(("prompt", "step", "train"))
        D, B, K = _extent(rng, 64, 8192), _log(rng, 1, 256 if mode == "step" else 8), rng.choice((2, 3, 4, 4, 4, 7))
        most = (32 if type == "fp32" else 64) << 20
        L = 1 if mode == "step" else min(_log(rng, 1, 16384), most // (B * D))
        return _conv(mode, type, B, L, D, K, act=rng.choice(("none", "silu", "silu")), ragged=mode == "prompt" and rng.random() < 0.5)
    if op == "scan":
        mode = rng.choice(("prompt", "step", "train"))
        G, N = rng.choice((1, 1, 2, 4)), rng.choice((4, 8, 16, 16, 16, 19, 32, 64))
        D, B = G * _extent(rng, 32, 4096 // G), _log(rng, 1, 256 if mode == "step" else 8)
        most = (192 if mode == "train" else 768) << 20
        L = 1 if mode == "step" else max(1, min(_log(rng, 1, 16384), most // (B * D * N)))
        if mode == "step":
            B = max(1, min(B, (16 << 20) // (D * N)))
        return _scan(mode, type, B, L, D, N, G=G, ragged=mode == "prompt" and rng.random() < 0.5)
    mode = rng.choice(("apply", "train"))
    G = rng.choice((1, 8, 16, 32))
    C = G * _log(rng, 4, max(4, 4096 // G))
    S = 1 if rng.random() < 0.3 else _log(rng, 4, 16384)
    most = (16 if type == "fp32" else 24) << 20
    S = min(S, most // C)
    N = max(1, min(_log(rng, 1, 16384 if S == 1 else 32), most // (S * C)))
    return _norm(mode, type, N, S, C, G, act=rng.choice(("none", "relu", "silu", "gelu")))


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
        N, S, C, G = case["N"], case["S"], case["C"], case["G"]
        s["x"] = normal(N, S, C, scale=1.5, shift=0.3)
        s["gamma"] = normal(C, scale=0.2, shift=1.0, dtype=torch.float32)
        s["beta"] = normal(C, scale=0.2, dtype=torch.float32)
        s["y"] = torch.empty_like(s["x"])
        s["mean"], s["rstd"] = torch.empty(N, G, device="cuda"), torch.empty(N, G, device="cuda")
        if train:
            s["dy"] = normal(N, S, C)
            s["dx"] = torch.empty_like(s["x"])
            s["dgamma"], s["dbeta"] = torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
        return s
    B, L, D = case["B"], case["L"], case["D"]
    step = case["mode"] == "step"
    rows = (B, D) if step else (B, L, D)
    s["lengths"] = None
    if case["ragged"]:
        s["lengths"] = (unit(B) * L).floor().add_(1).clamp_(max=L).to(torch.int32)
        s["lengths"][0] = L
    if case["op"] == "conv":
        K = case["K"]
        s["x"] = normal(*rows)
        s["w"] = normal(D, K, scale=1.0 / math.sqrt(K))
        s["bias"] = normal(D, scale=0.1)
        s["state"] = normal(B, K - 1, D) if step else None
        s["y"] = torch.empty_like(s["x"])
        s["state_out"] = None if train else torch.empty((B, K - 1, D), dtype=t, device="cuda")
        if train:
            s["dy"] = normal(*rows)
            s["dx"] = torch.empty_like(s["x"])
            s["dw"], s["dbias"] = torch.empty(D, K, device="cuda"), torch.empty(D, device="cuda")
        return s
    N, G = case["N"], case["G"]
    s["u"], s["z"] = normal(*rows), normal(*rows)
    s["delta"] = normal(*rows, scale=0.5)
    # steps of 0.001 to 0.1, spread over their logarithm, as the bias of the step sizes is initialised
    dt = torch.exp(unit(D) * (math.log(0.1) - math.log(0.001)) + math.log(0.001))
    s["delta_bias"] = dt + torch.log(-torch.expm1(-dt))
    s["A"] = -torch.arange(1, N + 1, device="cuda", dtype=torch.float32) * torch.exp(0.1 * normal(D, N, dtype=torch.float32))
    s["Bm"] = normal(*rows[:-1], G, N)
    s["Cm"] = normal(*rows[:-1], G, N)
    s["Dskip"] = normal(D, scale=0.1, shift=1.0, dtype=torch.float32)
    s["state"] = normal(B, D, N, scale=0.3, dtype=torch.float32) if step else None
    s["y"] = torch.empty_like(s["u"])
    s["state_out"] = None if train else torch.empty(B, D, N, device="cuda")
    if train:
        s["dy"] = normal(*rows)
        for name in ("u", "delta", "z", "Bm", "Cm", "A", "Dskip", "delta_bias"):
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
    if c["op"] == "norm":
        N, S, C, G = c["N"], c["S"], c["C"], c["G"]
        act = {"none": lib.ACT_NONE, "relu": lib.ACT_RELU, "silu": lib.ACT_SILU, "gelu": lib.ACT_GELU}[c["act"]]
        if "ws_bytes" not in s:
            s["ws_bytes"] = max(lib.norm_fwd_groups_workspace_size(N, S, C, G), lib.norm_bwd_groups_workspace_size(N, S, C, G))
        n = s["ws_bytes"]
        ws = _kept(s, "ws", n)
        lib.norm_fwd_groups(_p(s["x"]), _p(s["gamma"]), _p(s["beta"]), _p(s["y"]), _p(s["mean"]), _p(s["rstd"]), N, S, C, G, C, C, _EPS,
                            type, act, ws, n, stream)
        if c["mode"] == "apply":
            return s["y"], s["mean"], s["rstd"]
        lib.norm_bwd_groups(_p(s["x"]), _p(s["gamma"]), _p(s["beta"]), _p(s["mean"]), _p(s["rstd"]), _p(s["dy"]), _p(s["dx"]),
                            _p(s["dgamma"]), _p(s["dbeta"]), N, S, C, G, C, C, C, type, act, ws, n, stream)
        return s["y"], s["dx"], s["dgamma"], s["dbeta"]
    B, L, D = c["B"], c["L"], c["D"]
    if c["op"] == "conv":
        K = c["K"]
        act = {"none": lib.ACT_NONE, "silu": lib.ACT_SILU}[c["act"]]
        if c["mode"] == "step":
            lib.conv1d_step_causal(_p(s["x"]), _p(s["w"]), _p(s["bias"]), _p(s["state"]), _p(s["y"]), _p(s["state_out"]), B, D, K, D, D,
                                   type, act, stream)
            return s["y"], s["state_out"]
        lib.conv1d_fwd_causal(_p(s["x"]), _p(s["w"]), _p(s["bias"]), 0, _p(s["lengths"]), _p(s["y"]), _p(s["state_out"]), B, L, D, K, D, D,
                              type, act, stream)
        if c["mode"] == "prompt":
            return s["y"], s["state_out"]
        if "ws_bytes" not in s:
            s["ws_bytes"] = lib.conv1d_bwd_causal_workspace_size(B, L, D, K)
        n = s["ws_bytes"]
        lib.conv1d_bwd_causal(_p(s["x"]), _p(s["w"]), _p(s["bias"]), 0, 0, _p(s["dy"]), 0, _p(s["dx"]), _p(s["dw"]), _p(s["dbias"]), 0,
                              B, L, D, K, D, D, D, type, act, _kept(s, "ws", n), n, stream)
        return s["y"], s["dx"], s["dw"], s["dbias"]
    N, G = c["N"], c["G"]
    if c["mode"] == "step":
        lib.scan_step_selective(_p(s["u"]), _p(s["delta"]), _p(s["A"]), _p(s["Bm"]), _p(s["Cm"]), _p(s["Dskip"]), _p(s["z"]),
                                _p(s["delta_bias"]), _p(s["state"]), _p(s["y"]), _p(s["state_out"]), B, D, N, G, D, D, G * N, G * N, D, D,
                                type, lib.FLAG_SCAN_SOFTPLUS, stream)
        return s["y"], s["state_out"]
    train = c["mode"] == "train"
    if "ws_bytes" not in s:
        s["ws_bytes"] = lib.scan_fwd_selective_workspace_size(B, L, D, N, G)
        if train:
            s["ws_bytes"] = max(s["ws_bytes"], lib.scan_bwd_selective_workspace_size(B, L, D, N, G))
            s["states_bytes"] = lib.scan_states_size(B, L, D, N)
    n = s["ws_bytes"]
    ws, states = _kept(s, "ws", n), _kept(s, "states", s["states_bytes"]) if train else 0
    lib.scan_fwd_selective(_p(s["u"]), _p(s["delta"]), _p(s["A"]), _p(s["Bm"]), _p(s["Cm"]), _p(s["Dskip"]), _p(s["z"]), _p(s["delta_bias"]),
                           0, _p(s["lengths"]), _p(s["y"]), _p(s["state_out"]), states, B, L, D, N, G, D, D, G * N, G * N, D, D,
                           type, lib.FLAG_SCAN_SOFTPLUS, ws, n, stream)
    if not train:
        return s["y"], s["state_out"]
    lib.scan_bwd_selective(_p(s["u"]), _p(s["delta"]), _p(s["A"]), _p(s["Bm"]), _p(s["Cm"]), _p(s["Dskip"]), _p(s["z"]), _p(s["delta_bias"]),
                           0, states, _p(s["dy"]), 0, _p(s["du"]), _p(s["ddelta"]), _p(s["dA"]), _p(s["dBm"]), _p(s["dCm"]), _p(s["dDskip"]),
                           _p(s["dz"]), _p(s["ddelta_bias"]), 0, B, L, D, N, G, D, D, G * N, G * N, D, D, D, D, G * N, G * N, D,
                           type, lib.FLAG_SCAN_SOFTPLUS, ws, n, stream)
    return (s["y"],) + tuple(s["d" + name] for name in ("u", "delta", "A", "Bm", "Cm", "Dskip", "z", "delta_bias"))


# --------------------------------------------------------------------------------------------------------- the plain forms

def _act(v, act):
    if act == "none":
        return v
    if act == "relu":
        return torch.where(v < 0, torch.zeros_like(v), v)
    if act == "silu":
        return v / (1 + torch.exp(-v))
    return v * 0.5 * (1 + torch.erf(v * math.sqrt(0.5)))


def _dact(v, act):
    """The derivative of the activation at v."""
    if act == "none":
        return torch.ones_like(v)
    if act == "relu":
        return (v > 0).to(v.dtype)
    if act == "silu":
        sig = 1 / (1 + torch.exp(-v))
        return sig * (1 + v * (1 - sig))
    return 0.5 * (1 + torch.erf(v * math.sqrt(0.5))) + v * torch.exp(-0.5 * v * v) * (1 / math.sqrt(2 * math.pi))


def _real_rows(s, L):
    """[B][L][1]: which rows belong to their sequence."""
    B = s["case"]["B"]
    if s["lengths"] is None:
        return torch.ones((B, L, 1), dtype=torch.bool, device="cuda")
    return (torch.arange(L, device="cuda")[None, :] < s["lengths"][:, None])[..., None]


def _plain_conv(s):
    c = s["case"]
    B, L, D, K, t = c["B"], c["L"], c["D"], c["K"], _TYPES[c["type"]]
    w, bias = s["w"].float(), s["bias"].float()
    if c["mode"] == "step":
        window = torch.cat([s["state"], s["x"][:, None]], dim=1)
        y = _act((window.float() * w.t()).sum(1) + bias, c["act"])
        return y.to(t), window[:, 1:].contiguous()
    real = _real_rows(s, L)
    x = torch.where(real, s["x"], torch.zeros_like(s["x"])).float()
    xe = torch.cat([x.new_zeros(B, K - 1, D), x], dim=1)
    windows = xe.unfold(1, K, 1)                                     # [B][L][D][K]
    a = (windows * w).sum(-1) + bias
    y = torch.where(real, _act(a, c["act"]), torch.zeros_like(a))
    if c["mode"] == "prompt":
        ends = torch.full((B,), L, device="cuda") if s["lengths"] is None else s["lengths"].long()
        rows = ends[:, None] + torch.arange(K - 1, device="cuda")
        return y.to(t), torch.gather(xe, 1, rows[..., None].expand(B, K - 1, D)).to(t)
    g = s["dy"].float() * _dact(a, c["act"])
    ge = torch.cat([g, g.new_zeros(B, K - 1, D)], dim=1)
    dx = (ge.unfold(1, K, 1) * w.flip(1)).sum(-1)
    dw = (windows * g[..., None]).sum((0, 1), dtype=torch.float64)
    return y.to(t), dx.to(t), dw.float(), g.sum((0, 1), dtype=torch.float64).float()


def _recurrence(a, b):
    """h_t = a_t h_{t-1} + b_t along dimension 1, from zero: neighbours are joined to a sequence of half the length, which gives every
    second value; the others follow from those."""
    L = a.shape[1]
    if L == 1:
        return b
    m = L // 2
    odd = _recurrence(a[:, 1::2] * a[:, 0:2 * m:2], a[:, 1::2] * b[:, 0:2 * m:2] + b[:, 1::2])
    h = torch.empty_like(b)
    h[:, 1::2] = odd
    h[:, 0] = b[:, 0]
    h[:, 2::2] = a[:, 2::2] * odd[:, :(L - 1) // 2] + b[:, 2::2]
    return h


def _plain_scan(s):
    c = s["case"]
    B, D, N, G, t = c["B"], c["D"], c["N"], c["G"], _TYPES[c["type"]]
    L, E = c["L"], D // G
    real = _real_rows(s, L)

    def rows(x):                                                     # [B][L][G][E], zero behind the sequences
        x = x.reshape(B, L, D)
        return torch.where(real, x, torch.zeros_like(x)).float().reshape(B, L, G, E)

    u, z = rows(s["u"]), rows(s["z"])
    raw = rows(s["delta"]) + s["delta_bias"].reshape(G, E)
    dt = torch.log1p(torch.exp(-raw.abs())) + torch.where(raw > 0, raw, torch.zeros_like(raw))
    dt = torch.where(real[..., None], dt, torch.zeros_like(dt))
    A = s["A"].reshape(G, E, N)
    keep = real[..., None]
    Bm = torch.where(keep, s["Bm"].reshape(B, L, G, N), 0).float()[:, :, :, None]
    Cm = torch.where(keep, s["Cm"].reshape(B, L, G, N), 0).float()[:, :, :, None]
    a = torch.exp(dt[..., None] * A)
    b = (dt * u)[..., None] * Bm
    if s["state"] is not None:
        b[:, 0] += a[:, 0] * s["state"].reshape(B, G, E, N)
    h = _recurrence(a, b)
    v = (h * Cm).sum(-1) + s["Dskip"].reshape(G, E) * u
    sig = 1 / (1 + torch.exp(-z))
    y = torch.where(real, (v * z * sig).reshape(B, L, D), torch.zeros((), device="cuda"))
    if c["mode"] != "train":
        return y.reshape(s["u"].shape).to(t), h[:, -1].reshape(B, D, N).clone()
    dy = rows(s["dy"])
    g = dy * z * sig
    dz = dy * v * sig * (1 + z * (1 - sig))
    del b
    # e_t = C_t g_t + a_{t+1} e_{t+1}: the same recurrence from the other end
    after = torch.cat([a[:, 1:], torch.zeros_like(a[:, :1])], dim=1)
    e = _recurrence(after.flip(1), (Cm * g[..., None]).flip(1)).flip(1)
    del after
    dC = (g[..., None] * h).sum(3)
    before = torch.cat([torch.zeros_like(h[:, :1]), h[:, :-1]], dim=1)
    q = e * a * before
    del a, h, before
    dA = (q * dt[..., None]).sum((0, 1), dtype=torch.float64)
    eB = (e * Bm).sum(-1)
    ddt = (q * A).sum(-1) + u * eB
    du = dt * eB + s["Dskip"].reshape(G, E) * g
    dB = (e * (dt * u)[..., None]).sum(3)
    ddelta = ddt / (1 + torch.exp(-raw))
    return (y.to(t), du.reshape(B, L, D).to(t), ddelta.reshape(B, L, D).to(t), dA.reshape(D, N).float(), dB.to(t), dC.to(t),
            (g * u).sum((0, 1), dtype=torch.float64).reshape(D).float(), dz.reshape(B, L, D).to(t),
            ddelta.sum((0, 1), dtype=torch.float64).reshape(D).float())


def _plain_norm(s):
    c = s["case"]
    N, S, C, G, t = c["N"], c["S"], c["C"], c["G"], _TYPES[c["type"]]
    x = s["x"].float().reshape(N, S, G, C // G)
    gamma, beta = s["gamma"].reshape(G, C // G), s["beta"].reshape(G, C // G)
    mean = x.mean((1, 3), keepdim=True)
    xc = x - mean
    rstd = 1 / torch.sqrt((xc * xc).mean((1, 3), keepdim=True) + _EPS)
    xn = xc * rstd
    v = xn * gamma + beta
    y = _act(v, c["act"]).reshape(N, S, C).to(t)
    if c["mode"] == "apply":
        return y, mean.reshape(N, G), rstd.reshape(N, G)
    d = s["dy"].float().reshape(N, S, G, C // G) * _dact(v, c["act"])
    dn = d * gamma
    dx = rstd * (dn - dn.mean((1, 3), keepdim=True) - xn * (dn * xn).mean((1, 3), keepdim=True))
    return (y, dx.reshape(N, S, C).to(t), (d * xn).sum((0, 1), dtype=torch.float64).reshape(C).float(),
            d.sum((0, 1), dtype=torch.float64).reshape(C).float())


def run(s):
    if own:
        return _own(s)
    return {"conv": _plain_conv, "scan": _plain_scan, "norm": _plain_norm}[s["case"]["op"]](s)


# -------------------------------------------------------------------------------------------------------------- yardsticks

def work(case):
    size = _BYTES[case["type"]]
    train = case["mode"] == "train"
    if case["op"] == "norm":
        n, small = case["N"] * case["S"] * case["C"], 4 * (2 * case["C"] + 2 * case["N"] * case["G"])
        if train:         # x, dy in; y, dx out; the gradients of the scale and the shift
            return {"bytes": 4 * n * size + 16 * case["C"], "flops": 26 * n}
        return {"bytes": 2 * n * size + small, "flops": 9 * n}
    B, L, D = case["B"], case["L"], case["D"]
    n = B * L * D
    if case["op"] == "conv":
        K = case["K"]
        weights, state = D * (K + 1), B * (K - 1) * D
        if train:         # x, dy in; y, dx out; the gradients of the filters
            return {"bytes": (4 * n + weights) * size + 4 * weights, "flops": n * (6 * K + 12)}
        return {"bytes": (2 * n + weights + (2 if case["mode"] == "step" else 1) * state) * size, "flops": n * (2 * K + 4)}
    N, G = case["N"], case["G"]
    bc, params, state = 2 * B * L * G * N, 4 * (D * N + 2 * D), 4 * B * D * N
    if train:             # u, delta, z, dy in; y and three gradients out; B, C and theirs
        return {"bytes": (8 * n + 2 * bc) * size + 2 * params, "flops": n * (26 * N + 40)}
    return {"bytes": (4 * n + bc) * size + params + (2 if case["mode"] == "step" else 1) * state, "flops": n * (7 * N + 12)}


def exact(case, seed):
    """The definitions in 64 bits, token by token and tap by tap; gradients by automatic differentiation of them."""
    s = prepare(case, seed)
    c, f = case, torch.float64
    train = c["mode"] == "train"
    act = {"none": lambda v: v, "relu": torch.relu, "silu": lambda v: v * torch.sigmoid(v),
           "gelu": lambda v: v * 0.5 * torch.erfc(-v / math.sqrt(2.0))}[c.get("act", "none")]

    def leaf(x):
        return x.to(f).requires_grad_(train)

    if c["op"] == "norm":
        N, S, C, G = c["N"], c["S"], c["C"], c["G"]
        x, gamma, beta = leaf(s["x"]), leaf(s["gamma"]), leaf(s["beta"])
        flat = x.reshape(N, S, G, C // G).transpose(1, 2).reshape(N, G, -1)
        var, mean = torch.var_mean(flat, dim=-1, unbiased=False, keepdim=True)
        xn = ((flat - mean) * (var + _EPS).rsqrt()).reshape(N, G, S, C // G).transpose(1, 2).reshape(N, S, C)
        y = act(xn * gamma + beta)
        if not train:
            return y, mean[..., 0], (var + _EPS).rsqrt()[..., 0]
        return (y.detach(),) + torch.autograd.grad(y, (x, gamma, beta), s["dy"].to(f))

    B, L, D = c["B"], c["L"], c["D"]
    lengths = [L] * B if s["lengths"] is None else s["lengths"].tolist()
    if c["op"] == "conv":
        K = c["K"]
        x, w, bias = leaf(s["x"].reshape(B, L, D)), leaf(s["w"]), leaf(s["bias"])
        first = torch.zeros(B, K - 1, D, dtype=f, device="cuda") if s["state"] is None else s["state"].to(f)
        xe = torch.cat([first, x], dim=1)
        a = bias
        for k in range(K):
            a = a + xe[:, k:k + L] * w[:, k]
        y = act(a)
        if train:
            return (y.detach(),) + torch.autograd.grad(y, (x, w, bias), s["dy"].to(f))
        for i, n in enumerate(lengths):
            y[i, n:] = 0
        return y.reshape(s["x"].shape), torch.stack([xe[i, n:n + K - 1] for i, n in enumerate(lengths)])

    N, G = c["N"], c["G"]
    if B * L * D * N > (1 << 28 if train else 1 << 31):
        return None
    u, delta, z = (leaf(s[k].reshape(B, L, D)) for k in ("u", "delta", "z"))
    A, skip, shift = leaf(s["A"]), leaf(s["Dskip"]), leaf(s["delta_bias"])
    Bm, Cm = (leaf(s[k].reshape(B, L, G, N)) for k in ("Bm", "Cm"))
    h = torch.zeros(B, D, N, dtype=f, device="cuda") if s["state"] is None else s["state"].to(f)
    if not train:
        y = torch.zeros(B, L, D, dtype=f, device="cuda")
        alive = torch.tensor(lengths, device="cuda")
        for i in range(L):
            dt = torch.nn.functional.softplus(delta[:, i] + shift, threshold=100.0)[..., None]
            new = torch.exp(dt * A) * h + dt * u[:, i, :, None] * Bm[:, i].repeat_interleave(D // G, dim=1)
            h = torch.where((alive > i)[:, None, None], new, h)
            out = (h * Cm[:, i].repeat_interleave(D // G, dim=1)).sum(-1) + skip * u[:, i]
            y[:, i] = torch.where((alive > i)[:, None], out * z[:, i] * torch.sigmoid(z[:, i]), 0)
        return y.reshape(s["u"].shape), h
    # differentiated in pieces of the sequence, from the last one back, so that one piece's graph is held at a time
    piece = max(1, (1 << 25) // (B * D * N))
    weights = (A, skip, shift)

    def through(h, u, delta, z, Bm, Cm):
        outs = []
        for i in range(u.shape[1]):
            dt = torch.nn.functional.softplus(delta[:, i] + shift, threshold=100.0)[..., None]
            h = torch.exp(dt * A) * h + dt * u[:, i, :, None] * Bm[:, i].repeat_interleave(D // G, dim=1)
            outs.append(((h * Cm[:, i].repeat_interleave(D // G, dim=1)).sum(-1) + skip * u[:, i]) * z[:, i] * torch.sigmoid(z[:, i]))
        return h, torch.stack(outs, dim=1)

    pieces, ys = [], []
    for lo in range(0, L, piece):
        rows = [x[:, lo:lo + piece].detach().requires_grad_() for x in (u, delta, z, Bm, Cm)]
        pieces.append((h, rows, s["dy"][:, lo:lo + piece].to(f)))
        with torch.no_grad():
            h, y = through(h, *rows)
        ys.append(y)
    total, back, parts = [torch.zeros_like(x) for x in weights], torch.zeros_like(h), []
    for h0, rows, dy in reversed(pieces):
        with torch.enable_grad():
            h0 = h0.detach().requires_grad_()
            h1, y = through(h0, *rows)
            grads = torch.autograd.grad((y, h1), tuple(rows) + weights + (h0,), (dy, back))
        parts.insert(0, grads[:5])
        total = [sum_ + grad for sum_, grad in zip(total, grads[5:8])]
        back = grads[8]
    du, ddelta, dz, dB, dC = (torch.cat(x, dim=1) for x in zip(*parts))
    return torch.cat(ys, dim=1), du, ddelta, total[0], dB, dC, total[1], dz, total[2]
