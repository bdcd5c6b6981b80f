"""Performance cases of the operators of a latent transformer's block: layer norm with a weight and bias for each
sequence, rotary positions over several axes, the gated feed-forward product and dropout.

A denoiser over a latent cut into patches (an image, a video) or over an action sequence calls them beside attention and
torch's matrix products: in a sampler on all points of a window at once, in training with their gradients, and for
single tokens.  With ``own`` false the operators are computed in their plain form, by elementary operations in 32 bits.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
_BYTES = {"f32": 4.0, "bf16": 2.0}
_EPS = 1e-6


# ------------------------------------------------------------------------------------- the cases
def _norm(**kw):
    """groups: sequences with a weight and bias of their own (1: all rows share one); pad: what the rows' buffer is wider;
    keep: the rows' statistics are returned, as training needs them."""
    return dict({"do": "norm", "rows": 16, "width": 1024, "groups": 1, "dtype": "f32", "pad": 0, "keep": False}, **kw)


def _rotary(**kw):
    """grid: tokens along each axis; sections: pairs of a head that turn by each axis, as 'a,b,c'; order: 'runs' (an axis's
    pairs side by side) or 'turns' (the axes take pairs in turn)."""
    return dict({"do": "rotary", "batch": 1, "grid": "24,24", "heads": 16, "kv_heads": 16, "dim": 64, "sections": "16,16",
                 "order": "runs", "pairs": "half", "dtype": "f32", "fused": True}, **kw)


def _dropout(**kw):
    return dict({"do": "dropout", "rows": 16, "width": 1024, "dtype": "f32", "p": 0.1, "residual": False, "pad": 0}, **kw)


def _gated(**kw):
    """weights: 'in_out' ([in, out], as the product x @ w takes them) or 'out_in'; keep: gate and up are stored for the
    backward pass."""
    return dict({"do": "gated", "rows": 1, "width": 1024, "hidden": 4096, "dtype": "bf16", "act": "silu",
                 "weights": "in_out", "keep": False}, **kw)


def listed():
    return [
        # one action sequence (16 steps) at the policy's width: the smallest call, where latency is everything
        _norm(name="norm_action_sequence"),
        # a sampler's window of 64 points of a 96x96 latent in patches of 4x4, each point with its own timestep
        _norm(name="norm_latent_window", rows=64 * 576, groups=64, dtype="bf16"),
        # training on 16 sequences of 777 tokens, modulated by their timesteps: an odd width, rows cut from a wider buffer
        _norm(name="norm_backward_odd", do="norm_backward", rows=16 * 777, width=1001, groups=16, dtype="bf16", pad=7),
        # one latent in patches of 4x4, in float32: height and width
        _rotary(name="rotary_image"),
        # gradient through a video's positions: 16 frames of 32x32 patches, pairs side by side, the axes in turn
        _rotary(name="rotary_video_backward", do="rotary_backward", grid="16,32,32", heads=32, kv_heads=8, dim=128,
                sections="16,24,24", order="turns", pairs="interleaved", dtype="bf16"),
        # a training step's smallest call: one action sequence
        _dropout(name="dropout_action_sequence"),
        # training on latents: the feed-forward's result, dropped out and added to the residual stream
        _dropout(name="dropout_latent_residual", rows=64 * 576, dtype="bf16", residual=True),
        # a control loop: one token
        _gated(name="gated_token"),
        # serving: the next token of 24 sequences, weights as a linear layer holds them
        _gated(name="gated_token_batch", rows=24, act="gelu_tanh", weights="out_in"),
        # every point of a policy's whole-chain window, 100 sequences of 16 actions, in float32; an odd hidden width
        _gated(name="gated_policy_window", rows=1600, hidden=2731, dtype="f32"),
        # a window of 64 points of a latent in 4x4 patches
        _gated(name="gated_latent_window", rows=64 * 576, act="gelu"),
        # training on latents in 2x2 patches (48x48 tokens)
        _gated(name="gated_latent_backward", do="gated_backward", rows=4 * 2304, hidden=2736),
    ]


#: Multiply-adds (rows x width x hidden) of a drawn gated case: no more than the listed window has.
_MOST_PRODUCTS = 64 * 576 * 1024 * 4096


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "norm_backward", "rotary", "rotary_backward", "dropout", "gated", "gated", "gated_backward"])
    dtype = rng.choice(["f32", "bf16", "bf16"])
    if kind.startswith("norm") or kind == "dropout":
        width = rng.choice([rng.randint(40, 8192), 8 * rng.randint(8, 1024), 128 * rng.randint(1, 64)])
        rows = _log(rng, 1, max(2, 32_000_000 // width))
        pad = rng.choice([0, 0, 8, 5])
        if kind == "dropout":
            return _dropout(rows=rows, width=width, dtype=dtype, pad=pad, p=rng.choice([0.1, 0.5, rng.uniform(0.01, 0.6)]),
                            residual=rng.random() < 0.5)
        groups = rng.choice([1, 1, rng.randint(2, 64)])
        span = max(1, rows // groups)
        return _norm(do=kind, rows=groups * span, width=width, groups=groups, dtype=dtype, pad=pad, keep=rng.random() < 0.5)
    if kind.startswith("rotary"):
        axes = rng.choice([2, 2, 3, 3, 1])
        dim = rng.choice([32, 64, 64, 80, 96, 128, 128, 2 * rng.randint(12, 64)])
        pairs = rng.choice([dim // 2, dim // 2, max(axes, dim // 4)])
        cuts = sorted(rng.sample(range(1, pairs), axes - 1))
        sections = [b - a for a, b in zip([0] + cuts, cuts + [pairs])]
        if rng.random() < 0.5:
            sections = [pairs // axes + (1 if i < pairs % axes else 0) for i in range(axes)]
        kv = rng.choice([1, 2, 4, 8])
        heads = kv * rng.choice([1, 2, 4, 7, 8])
        batch = _log(rng, 1, 64)
        most = min(32768, max(2, 64_000_000 // (batch * (heads + kv) * dim)))
        side = most ** (1.0 / axes)
        grid = [max(1, int(_log(rng, 1, max(1.5, side)))) for _ in range(axes)]
        return _rotary(do=kind, batch=batch, grid=",".join(map(str, grid)), heads=heads, kv_heads=kv, dim=dim,
                       sections=",".join(map(str, sections)), order=rng.choice(["runs", "turns"]),
                       pairs=rng.choice(["half", "interleaved"]), dtype=dtype, fused=rng.random() < 0.5)
    width = rng.choice([8 * _log(rng, 8, 512), 64 * _log(rng, 1, 64), _log(rng, 40, 4096)])
    hidden = rng.choice([4 * width, 8 * ((8 * width // 3 + 7) // 8), 2 * width, _log(rng, 64, 8192)])
    most = _MOST_PRODUCTS // (4 if dtype == "f32" else 1)
    if kind == "gated_backward":
        most //= 2
    most = min(most // (width * hidden), 400_000_000 // (width + 3 * hidden))
    return _gated(do=kind, rows=_log(rng, 1, max(2, min(40000, most))), width=width, hidden=hidden, dtype=dtype,
                  act=rng.choice(["silu", "silu", "gelu", "gelu_tanh", "sigmoid", "relu"]),
                  weights=rng.choice(["in_out", "out_in"]), keep=kind == "gated" and rng.random() < 0.5)


# ---------------------------------------------------------------------------------------- inputs
def _ints(text):
    return [int(v) for v in text.split(",")]


def _tokens(c):
    return math.prod(_ints(c["grid"]))


def _axis_of_pair(c):
    """The axis that each pair turns by, and the pair's number among its axis's."""
    left, axis, at = _ints(c["sections"]), [], []
    took = [0] * len(left)
    while sum(left):
        for a in range(len(left)):
            n = min(left[a], 1) if c["order"] == "turns" else left[a]
            axis += [a] * n
            at += range(took[a], took[a] + n)
            took[a] += n
            left[a] -= n
    return axis, at


def _table(c, device):
    """cos and sin of every coordinate and pair: each axis's pairs turn by 10000^(-i / its pairs)."""
    axis, at = _axis_of_pair(c)
    per = _ints(c["sections"])
    f = torch.tensor([10000.0 ** (-i / per[a]) for a, i in zip(axis, at)], device=device, dtype=torch.float64)
    a = torch.arange(max(_ints(c["grid"])), device=device, dtype=torch.float64)[:, None] * f
    return torch.stack([a.cos(), a.sin()], 2).to(torch.float32)


def _randn(g, *shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(*shape, device="cuda", generator=g) * scale).to(dtype)


def _norm_state(c, g):
    n, d, t, G = c["rows"], c["width"], _TYPES[c["dtype"]], c["groups"]

    def rows():                                    # rows of a buffer that may be wider
        return _randn(g, n, d + c["pad"], dtype=t)[:, :d]
    # a residual stream has a few features much larger than the rest, and an offset in some
    gain = torch.exp(0.8 * torch.randn(d, device="cuda", generator=g))
    shift = 0.5 * gain * torch.randn(d, device="cuda", generator=g)
    # a block's modulation: scale and shift of each sequence, side by side in one product's result
    m = 0.2 * torch.randn(G, 2 * d, device="cuda", generator=g)
    s = {"weight": (1.0 + m)[:, :d], "bias": m[:, d:]}
    if G == 1:
        s = {k: v[0].clone() for k, v in s.items()}
    if c["do"] == "norm":
        s["x"] = rows()
        s["residual"] = (rows().float() * gain + shift).to(t)
        s["sum"], s["y"] = (torch.empty(n, d, device="cuda", dtype=t) for _ in range(2))
        s["mean"], s["rstd"] = (torch.empty(n, device="cuda") if c["keep"] else None for _ in range(2))
        return s
    s["sum"] = rows()
    s["sum"].copy_(s["sum"].float() * gain + shift)
    h = s["sum"].double()
    s["mean"] = h.mean(1).float()
    s["rstd"] = torch.rsqrt(h.var(1, unbiased=False) + _EPS).float()
    del h
    s["dy"], s["dsum"] = rows() * 0.1, rows() * 0.1
    s["dx"] = torch.empty(n, d, device="cuda", dtype=t)
    s["dweight"], s["dbias"] = (torch.empty(s["weight"].shape, device="cuda") for _ in range(2))
    return s


def _rotary_state(c, g):
    B, n, t = c["batch"], _tokens(c), _TYPES[c["dtype"]]
    H, K, D = c["heads"], c["kv_heads"], c["dim"]
    if c["fused"]:                                 # side by side, as one product makes them
        q, k = torch.split(_randn(g, B, n, H + K, D, dtype=t), [H, K], dim=2)
    else:
        q, k = _randn(g, B, n, H, D, dtype=t), _randn(g, B, n, K, D, dtype=t)
    at = torch.meshgrid(*[torch.arange(m, device="cuda", dtype=torch.int32) for m in _ints(c["grid"])], indexing="ij")
    return {"q": q, "k": k, "positions": torch.stack([a.flatten() for a in at], 1), "table": _table(c, "cuda"),
            "q_out": torch.empty(B, n, H, D, device="cuda", dtype=t), "k_out": torch.empty(B, n, K, D, device="cuda", dtype=t)}


def _gated_state(c, g):
    n, D, F, t = c["rows"], c["width"], c["hidden"], _TYPES[c["dtype"]]
    shape = (D, F) if c["weights"] == "in_out" else (F, D)
    wg, wu = (_randn(g, *shape, dtype=t, scale=D ** -0.5) for _ in range(2))
    if c["weights"] == "out_in":                   # a linear layer's weights, seen as [in, out]
        wg, wu = wg.t(), wu.t()
    s = {"x": _randn(g, n, D, dtype=t), "w_gate": wg, "w_up": wu}
    new = lambda: torch.empty(n, F, device="cuda", dtype=t)  # noqa: E731
    if c["do"] == "gated":
        s["h"] = new()
        s["gate"], s["up"] = (new(), new()) if c["keep"] else (None, None)
        return s
    x = s["x"].float()                             # what the forward pass of the training step left
    s["gate"], s["up"] = ((x @ w.float()).to(t) for w in (wg, wu))
    s["dh"] = _randn(g, n, F, dtype=t, scale=0.1)
    s["dx"] = torch.empty(n, D, device="cuda", dtype=t)
    s["dw_gate"], s["dw_up"] = (torch.empty_like(w) for w in (wg, wu))
    return s


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(seed)
    if c["do"].startswith("norm"):
        s = _norm_state(c, g)
    elif c["do"].startswith("rotary"):
        s = _rotary_state(c, g)
    elif c["do"].startswith("gated"):
        s = _gated_state(c, g)
    else:
        n, d, t = c["rows"], c["width"], _TYPES[c["dtype"]]
        s = {"x": _randn(g, n, d + c["pad"], dtype=t)[:, :d], "y": torch.empty(n, d, device="cuda", dtype=t),
             "residual": _randn(g, n, d, dtype=t) if c["residual"] else None, "seed": 1 + seed * 0x9E3779B97F4A7C15 % 2**63,
             "site": seed % 37, "step": seed % 1009}
    return dict(s, case=c)


# --------------------------------------------------------------------------------- the plain forms
def _of_rows(s, name):
    """Weight or bias as [groups, 1, width]."""
    return s[name].reshape(s["case"]["groups"], 1, s["case"]["width"])


def _plain_norm(s):
    c = s["case"]
    t, G, d = _TYPES[c["dtype"]], c["groups"], c["width"]
    h = s["x"].float() + s["residual"].float()
    mean = h.mean(1, keepdim=True)
    off = h - mean
    rstd = torch.rsqrt(off.square().mean(1, keepdim=True) + _EPS)
    y = (off * rstd).reshape(G, -1, d) * _of_rows(s, "weight") + _of_rows(s, "bias")
    out = h.to(t), y.reshape(-1, d).to(t)
    return (*out, mean[:, 0], rstd[:, 0]) if c["keep"] else out


def _plain_norm_backward(s):
    c = s["case"]
    G, d = c["groups"], c["width"]
    r = s["rstd"][:, None]
    n, dy = (s["sum"].float() - s["mean"][:, None]) * r, s["dy"].float()
    a = (dy.reshape(G, -1, d) * _of_rows(s, "weight")).reshape(-1, d)
    dx = s["dsum"].float() + r * (a - a.mean(1, keepdim=True) - n * (a * n).mean(1, keepdim=True))
    shape = s["weight"].shape
    return dx.to(_TYPES[c["dtype"]]), (dy * n).reshape(G, -1, d).sum(1).reshape(shape), dy.reshape(G, -1, d).sum(1).reshape(shape)


def _plain_rotary(s):
    c = s["case"]
    R = 2 * sum(_ints(c["sections"]))
    axis = torch.tensor(_axis_of_pair(c)[0], device="cuda")
    at = s["table"][s["positions"].long()[:, axis], torch.arange(R // 2, device="cuda")]      # [token, pair, 2]
    cos, sin = at[:, None, :, 0], at[:, None, :, 1]
    if c["do"] == "rotary_backward":
        sin = -sin
    got = []
    for x in (s["q"].float(), s["k"].float()):
        half = c["pairs"] == "half"
        a, b = (x[..., :R // 2], x[..., R // 2:R]) if half else (x[..., 0:R:2], x[..., 1:R:2])
        u, v = a * cos - b * sin, a * sin + b * cos
        y = torch.cat([u, v], -1) if half else torch.stack([u, v], -1).flatten(-2)
        got.append(torch.cat([y, x[..., R:]], -1).to(_TYPES[c["dtype"]]))
    return tuple(got)


def _words(seed, stream, step, blocks, device):
    """Philox4x32-10 under the key `seed`: the four words, [blocks, 4], of the counters (block, stream, step + 1)."""
    low = 0xFFFFFFFF
    q = torch.arange(blocks, device=device, dtype=torch.int64)
    c = [q & low, q >> 32, torch.full_like(q, stream), torch.full_like(q, (step + 1) & low)]
    k0, k1 = seed & low, seed >> 32

    def times(m, v):                               # high and low word of a 64-bit product
        return ((v >> 16) * m + ((v & 0xFFFF) * m >> 16)) >> 16, (v * m) & low
    for _ in range(10):
        hi0, lo0 = times(0xD2511F53, c[0])
        hi1, lo1 = times(0xCD9E8D57, c[2])
        c = [hi1 ^ c[1] ^ k0, lo1, hi0 ^ c[3] ^ k1, lo0]
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return torch.stack(c, 1)


def _plain_dropout(s):
    """Eight neighbouring values of a row take the 16-bit halves of one counter's words; a value is kept where its half is
    not under p in steps of 2^-16."""
    c = s["case"]
    n, d = c["rows"], c["width"]
    per = -(-d // 8)
    w = _words(s["seed"], s["site"], s["step"], n * per, "cuda")
    halves = torch.stack([w & 0xFFFF, w >> 16], 2).reshape(n, 8 * per)[:, :d]
    under = math.floor(c["p"] * 65536 + 0.5)
    y = torch.where(halves >= under, s["x"].float() * (65536.0 / (65536 - under)), 0.0)
    if c["residual"]:
        y = y + s["residual"].float()
    return y.to(_TYPES[c["dtype"]])


def _act(x, kind):
    if kind == "silu":
        return x / (1 + torch.exp(-x))
    if kind == "gelu":
        return 0.5 * x * (1 + torch.erf(x * math.sqrt(0.5)))
    if kind == "gelu_tanh":
        return 0.5 * x * (1 + torch.tanh(math.sqrt(2 / math.pi) * (x + 0.044715 * x * x * x)))
    return 1 / (1 + torch.exp(-x)) if kind == "sigmoid" else x.clamp_min(0)


def _act_and_slope(x, kind):
    if kind == "silu":
        e = 1 / (1 + torch.exp(-x))
        return x * e, e * (1 + x * (1 - e))
    if kind == "gelu":
        e = 0.5 * (1 + torch.erf(x * math.sqrt(0.5)))
        return x * e, e + x * torch.exp(-0.5 * x * x) / math.sqrt(2 * math.pi)
    if kind == "gelu_tanh":
        r = math.sqrt(2 / math.pi)
        t = torch.tanh(r * (x + 0.044715 * x * x * x))
        return 0.5 * x * (1 + t), 0.5 * (1 + t) + 0.5 * x * (1 - t * t) * r * (1 + 3 * 0.044715 * x * x)
    if kind == "sigmoid":
        e = 1 / (1 + torch.exp(-x))
        return e, e * (1 - e)
    return x.clamp_min(0), (x > 0).to(x.dtype)


def _plain_gated(s):
    t, x = _TYPES[s["case"]["dtype"]], s["x"].float()
    g, u = x @ s["w_gate"].float(), x @ s["w_up"].float()
    h = (_act(g, s["case"]["act"]) * u).to(t)
    return (h, g.to(t), u.to(t)) if s["case"]["keep"] else h


def _plain_gated_backward(s):
    t = _TYPES[s["case"]["dtype"]]
    a, slope = _act_and_slope(s["gate"].float(), s["case"]["act"])
    dh, xt = s["dh"].float(), s["x"].float().t()
    dg, du = dh * s["up"].float() * slope, dh * a
    dx = dg @ s["w_gate"].float().t() + du @ s["w_up"].float().t()
    return dx.to(t), (xt @ dg).to(t), (xt @ du).to(t)


# -------------------------------------------------------------------------------------------- a pass
def _run_own(s):
    import paper_2305_16317_amd as pd
    c = s["case"]
    if c["do"] == "norm":
        pd.pd_layernorm_forward(s["x"], s["y"], weight=s["weight"], bias=s["bias"], residual=s["residual"],
                                sum_out=s["sum"], mean=s["mean"], rstd=s["rstd"], eps=_EPS)
        return (s["sum"], s["y"], s["mean"], s["rstd"]) if c["keep"] else (s["sum"], s["y"])
    if c["do"] == "norm_backward":
        pd.pd_layernorm_backward(s["dy"], s["sum"], s["mean"], s["rstd"], s["dx"], weight=s["weight"],
                                 dweight=s["dweight"], dbias=s["dbias"], dsum=s["dsum"])
        return s["dx"], s["dweight"], s["dbias"]
    if c["do"].startswith("rotary"):
        pd.pd_rotary_axes_apply(s["q"], s["k"], s["positions"], s["table"], _ints(c["sections"]), s["q_out"], s["k_out"],
                                layout=pd.PD_ROTARY_HALF if c["pairs"] == "half" else pd.PD_ROTARY_INTERLEAVED,
                                order=pd.PD_AXES_RUNS if c["order"] == "runs" else pd.PD_AXES_TURNS,
                                backward=c["do"] == "rotary_backward")
        return s["q_out"], s["k_out"]
    if c["do"] == "dropout":
        pd.pd_dropout_apply(s["x"], s["y"], c["p"], s["seed"], rng_stream=s["site"], step=s["step"], residual=s["residual"])
        return s["y"]
    act = {"silu": pd.PD_ACT_SILU, "gelu": pd.PD_ACT_GELU, "gelu_tanh": pd.PD_ACT_GELU_TANH, "sigmoid": pd.PD_ACT_SIGMOID,
           "relu": pd.PD_ACT_RELU}[c["act"]]
    if c["do"] == "gated":
        pd.pd_gated_forward(s["x"], s["w_gate"], s["w_up"], s["h"], gate=s["gate"], up=s["up"], activation=act)
        return (s["h"], s["gate"], s["up"]) if c["keep"] else s["h"]
    pd.pd_gated_backward(s["dh"], s["x"], s["w_gate"], s["w_up"], s["gate"], s["up"], dx=s["dx"], dw_gate=s["dw_gate"],
                         dw_up=s["dw_up"], activation=act)
    return s["dx"], s["dw_gate"], s["dw_up"]


@torch.no_grad()
def run(state):
    if own:
        return _run_own(state)
    return {"norm": _plain_norm, "norm_backward": _plain_norm_backward, "rotary": _plain_rotary, "rotary_backward": _plain_rotary,
            "dropout": _plain_dropout, "gated": _plain_gated, "gated_backward": _plain_gated_backward}[state["case"]["do"]](state)


# --------------------------------------------------------------------------------------------- floors
def work(case):
    """Inputs once, outputs once; the products that the formulas have."""
    c, b = case, _BYTES[case["dtype"]]
    if c["do"].startswith("rotary"):
        n, heads, R = float(c["batch"]) * _tokens(c), c["heads"] + c["kv_heads"], 2 * sum(_ints(c["sections"]))
        table = max(_ints(c["grid"])) * R * 4.0 + _tokens(c) * len(_ints(c["grid"])) * 4.0
        return {"bytes": n * heads * c["dim"] * 2 * b + table, "flops": n * heads * R * 3.0}
    n = float(c["rows"]) * c["width"]
    if c["do"] == "norm":
        return {"bytes": n * 4 * b + 8.0 * c["groups"] * c["width"] + (8.0 * c["rows"] if c["keep"] else 0.0), "flops": 9 * n}
    if c["do"] == "norm_backward":
        return {"bytes": n * 4 * b + 12.0 * c["groups"] * c["width"] + 8.0 * c["rows"], "flops": 14 * n}
    if c["do"] == "dropout":
        # (of Philox's ten rounds for eight values, the four multiplications and six other operations)
        return {"bytes": n * (3 if c["residual"] else 2) * b, "flops": n * (2.0 + 100.0 / 8)}
    rows, D, F = float(c["rows"]), float(c["width"]), float(c["hidden"])
    if c["do"] == "gated":
        return {"bytes": b * (rows * D + 2 * D * F + rows * F * (3 if c["keep"] else 1)), "flops": 4 * rows * D * F}
    return {"bytes": b * (2 * rows * D + 4 * D * F + 3 * rows * F), "flops": 8 * rows * D * F}


# ------------------------------------------------------------------------- the same in 64 bits
def _exact_norm(s):
    c = s["case"]
    d = c["width"]
    group = torch.arange(c["rows"], device="cuda") // (c["rows"] // c["groups"])
    w, b = (s[k].double().reshape(-1, d)[group] for k in ("weight", "bias"))
    if c["do"] == "norm":
        h = s["x"].double() + s["residual"].double()
        mean = h.sum(1) / d
        rstd = ((h - mean[:, None]).pow(2).sum(1) / d + _EPS).pow(-0.5)
        y = torch.addcmul(b, (h - mean[:, None]) * rstd[:, None], w)
        return (h, y, mean, rstd) if c["keep"] else (h, y)
    r = s["rstd"].double()[:, None]
    n, dy = (s["sum"].double() - s["mean"].double()[:, None]) * r, s["dy"].double()
    a = dy * w
    dx = s["dsum"].double() + r * a - r * (a.sum(1, keepdim=True) + n * torch.einsum("ij,ij->i", a, n)[:, None]) / d
    dw, db = (torch.zeros(c["groups"], d, device="cuda", dtype=torch.float64).index_add_(0, group, v) for v in (dy * n, dy))
    return dx, dw.reshape(s["weight"].shape), db.reshape(s["weight"].shape)


def _exact_rotary(s):
    c = s["case"]
    axis, _ = _axis_of_pair(c)
    R, half = 2 * len(axis), c["pairs"] == "half"
    outs = [s["q"].double().clone(), s["k"].double().clone()]
    tab, pos = s["table"].double(), s["positions"].long()
    for i, a in enumerate(axis):
        cos, sin = tab[pos[:, a], i, 0][:, None], tab[pos[:, a], i, 1][:, None]
        sin = -sin if c["do"] == "rotary_backward" else sin
        lo, hi = (i, i + R // 2) if half else (2 * i, 2 * i + 1)
        for y in outs:
            u, v = y[..., lo].clone(), y[..., hi].clone()
            y[..., lo], y[..., hi] = u * cos - v * sin, u * sin + v * cos
    return tuple(outs)


def _exact_dropout(s):
    c = s["case"]
    n, d = c["rows"], c["width"]
    per, low = (d + 7) // 8, np.uint64(0xFFFFFFFF)
    c0 = np.arange(n * per, dtype=np.uint64)
    c1, c0 = c0 >> np.uint64(32), c0 & low
    c2, c3 = np.full_like(c0, s["site"]), np.full_like(c0, s["step"] + 1)
    key = [s["seed"] % 2**32, s["seed"] // 2**32]
    for r in range(10):
        a, b = c0 * np.uint64(0xD2511F53), c2 * np.uint64(0xCD9E8D57)
        k0, k1 = (np.uint64((k + r * w) % 2**32) for k, w in zip(key, (0x9E3779B9, 0xBB67AE85)))
        c0, c1, c2, c3 = (b >> np.uint64(32)) ^ c1 ^ k0, b & low, (a >> np.uint64(32)) ^ c3 ^ k1, a & low
    u = np.stack([c0, c1, c2, c3], 1).astype("<u4").view("<u2").reshape(n, 8 * per)[:, :d]
    under = int(math.floor(c["p"] * 65536 + 0.5))
    keep = torch.from_numpy(u >= under).cuda()
    y = s["x"].double() * keep / (1 - under / 65536)
    return y + s["residual"].double() if c["residual"] else y


def _exact_gated(s):
    c = s["case"]
    F64 = torch.nn.functional
    act = {"silu": F64.silu, "gelu": F64.gelu, "gelu_tanh": lambda v: F64.gelu(v, approximate="tanh"),
           "sigmoid": torch.sigmoid, "relu": torch.relu}[c["act"]]
    x, wg, wu = (s[k].double() for k in ("x", "w_gate", "w_up"))
    if c["do"] == "gated":
        g, u = torch.mm(x, wg), torch.mm(x, wu)
        h = act(g).mul_(u)
        return (h, g, u) if c["keep"] else h
    dh = s["dh"].double()
    with torch.enable_grad():
        g = s["gate"].double().requires_grad_()
        a = act(g)
        dg, = torch.autograd.grad(a, g, dh * s["up"].double())
    du = dh * a.detach()
    return torch.mm(dg, wg.t()).add_(torch.mm(du, wu.t())), torch.mm(x.t(), dg), torch.mm(x.t(), du)


@torch.no_grad()
def exact(case, seed):
    s = prepare(case, seed)
    kind = case["do"].split("_")[0]
    if kind == "gated" and case["rows"] * case["width"] * case["hidden"] > 4e11:     # (float64 products at some 50 TFLOP/s)
        return None
    return {"norm": _exact_norm, "rotary": _exact_rotary, "dropout": _exact_dropout, "gated": _exact_gated}[kind](s)
