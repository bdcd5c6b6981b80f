"""The gated product's values where they are easily lost: infinities, gelu's tail, the rounding of its gradients.

Compared with the formulas in float64 (`oracle/block.py`); the tolerances are derived where they stand."""
import math

import numpy as np
import pytest
import torch

import paper_2305_16317_amd as pd
from oracle import block as ob

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
INF = float("inf")
ACTS = {"silu": pd.PD_ACT_SILU, "gelu": pd.PD_ACT_GELU, "gelu_tanh": pd.PD_ACT_GELU_TANH, "sigmoid": pd.PD_ACT_SIGMOID,
        "relu": pd.PD_ACT_RELU}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    pd.load()


def _np(t):
    return t.detach().double().cpu().numpy()


def _rand(shape, dtype, seed, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, device="cuda", generator=g) * scale).to(dtype)


def _weight(D, F, dtype, seed, layout):
    w = _rand((D, F), dtype, seed, D ** -0.5)
    return w if layout == pd.PD_WEIGHTS_IN_OUT else w.t().contiguous().t()


def _same(got, ref, tol, what):
    """Infinities and NaN where the formula has them; the rest within tol in the root mean square."""
    got = _np(got)
    assert np.array_equal(np.isnan(got), np.isnan(ref)), (what, "NaN", np.isnan(got).sum(), np.isnan(ref).sum())
    far = np.isinf(ref)
    assert np.array_equal(got[far], ref[far]) and not np.isinf(got[~far]).any(), what
    fine = np.isfinite(ref)
    assert np.linalg.norm(got[fine] - ref[fine]) <= tol * np.linalg.norm(ref[fine]), what


def _infinite_gradients(M, layout, dtype, tol):
    """One infinity at a time: in x, in a weight of each half, in dh, in up."""
    D, F = 72, 100
    for act in ("silu", "relu"):
        for where in ("x", "w_gate", "w_up", "dh", "up"):
            a = dict(dh=_rand((M, F), dtype, 1), x=_rand((M, D), dtype, 2), w_gate=_weight(D, F, dtype, 3, layout),
                     w_up=_weight(D, F, dtype, 4, layout), gate=_rand((M, F), dtype, 5), up=_rand((M, F), dtype, 6))
            a[where][1, 7] = -INF
            dx, dw = torch.empty_like(a["x"]), [torch.empty_like(a[n]) for n in ("w_gate", "w_up")]
            pd.pd_gated_backward(*a.values(), dx=dx, dw_gate=dw[0], dw_up=dw[1], activation=ACTS[act])
            with np.errstate(invalid="ignore"):
                rx, rg, ru, _ = ob.gated_grad(*(_np(t) for t in a.values()), act)
            assert not all(np.isfinite(r).all() for r in (rx, rg, ru))
            for got, ref, what in ((dx, rx, "dx"), (dw[0], rg, "dw_gate"), (dw[1], ru, "dw_up")):
                _same(got, ref, tol, (act, where, what))


@pytest.mark.parametrize("layout", [pd.PD_WEIGHTS_IN_OUT, pd.PD_WEIGHTS_OUT_IN])
@pytest.mark.parametrize("M", [2, 20, 32, 33, 300])
def test_gradients_of_infinite_values_bfloat16(M, layout):
    """An infinite x or weight meets both parts of dgate and dup: neither is 0 or of the other sign.  (Two roundings, of
    at most 2^-8 / sqrt 3 in the root mean square each: 4e-3.)"""
    _infinite_gradients(M, layout, BF16, 4e-3)


# ------------------------------------------------------------------ the gradients' rounding
@pytest.mark.parametrize("layout", [pd.PD_WEIGHTS_IN_OUT, pd.PD_WEIGHTS_OUT_IN])
@pytest.mark.parametrize("M,D,F", [(5, 72, 100), (40, 72, 100), (129, 200, 333), (700, 1024, 264), (2304, 320, 1336)])
def test_gradients_bfloat16_are_rounded_once(M, D, F, layout):
    """dgate and dup are operands to 2^-16, and act and its slope to 1e-5: a gradient's sum is off by at most 2.5e-5 of
    its terms' root mean square.  It then rounds to another value than the formula's with a probability of that over a
    step (2^-7 of the value at most), and is a step off: sqrt(2.5e-5 2^-7) = 4.4e-4 in the root mean square at most, where
    operands rounded to bfloat16 give 1.6e-3 to 2.3e-3."""
    dh, x, g, u = _rand((M, F), BF16, 20), _rand((M, D), BF16, 21), _rand((M, F), BF16, 22), _rand((M, F), BF16, 23)
    wg, wu = _weight(D, F, BF16, 24, layout), _weight(D, F, BF16, 25, layout)
    for act in ("silu", "gelu"):
        dx, dw = torch.empty_like(x), [torch.empty_like(t) for t in (wg, wu)]
        pd.pd_gated_backward(dh, x, wg, wu, g, u, dx=dx, dw_gate=dw[0], dw_up=dw[1], activation=ACTS[act])
        refs = ob.gated_grad(*(_np(t) for t in (dh, x, wg, wu, g, u)), act)
        for got, ref, what in ((dx, refs[0], "dx"), (dw[0], refs[1], "dw_gate"), (dw[1], refs[2], "dw_up")):
            once = _np(torch.from_numpy(ref).to(BF16))
            off = np.linalg.norm(_np(got) - once) / np.linalg.norm(once)
            print(M, D, F, act, what, off, flush=True)
            assert off <= 4.4e-4, (act, what, off)


# ------------------------------------------------------------------ infinities in float32
@pytest.mark.parametrize("layout", [pd.PD_WEIGHTS_IN_OUT, pd.PD_WEIGHTS_OUT_IN])
@pytest.mark.parametrize("M", [2, 33, 161, 300])
def test_gradients_of_infinite_values_float32(M, layout):
    """(Sums of some hundred terms in float32: 5e-6.)"""
    _infinite_gradients(M, layout, F32, 5e-6)


@pytest.mark.parametrize("layout", [pd.PD_WEIGHTS_IN_OUT, pd.PD_WEIGHTS_OUT_IN])
@pytest.mark.parametrize("dtype,M", [(F32, 2), (F32, 160), (F32, 161), (F32, 700), (BF16, 2), (BF16, 300)])
def test_forward_of_infinite_values(dtype, M, layout):
    """The formula's infinities and NaN whatever the number of rows: one in x, one in a weight, and one in each."""
    D, F = 72, 100
    for act in ACTS:
        for where in ((1,), (2,), (1, 2)):
            x, w = _rand((M, D), dtype, 10), [_weight(D, F, dtype, 11 + i, layout) for i in range(2)]
            if 1 in where:
                x[1, 7] = INF
            if 2 in where:
                w[0][7, 5] = -INF
                w[1][9, 60] = INF
            h, g, u = (torch.empty((M, F), device="cuda", dtype=dtype) for _ in range(3))
            pd.pd_gated_forward(x, *w, h, gate=g, up=u, activation=ACTS[act])
            with np.errstate(invalid="ignore", over="ignore"):
                refs = ob.gated(_np(x), _np(w[0]), _np(w[1]), act)
            for got, ref, what in zip((h, g, u), refs, ("h", "gate", "up")):
                _same(got, ref, 4e-3 if dtype == BF16 else 5e-6, (act, where, what))


# ------------------------------------------------------------------ gelu's tail
def _tail_error():
    """Relative error of tail = e^(-g^2/2) t Q(t) in float32: t's two roundings (2^-24, 2^-23) times 3.8, the most that
    t Q(t) follows t by (d log / d log at t = 1); Q's fit 2.2e-8 and its sum 2^-23; the exponential's 2^-23 and four products and sums of 2^-24."""
    return 3.8 * (2.0**-24 + 2.0**-23) + 2.2e-8 + 2.0**-23 + 2.0**-23 + 4 * 2.0**-24


@pytest.mark.parametrize("dtype,rows,width", [(F32, 100, 8), (F32, 4001, 2), (BF16, 50, 8), (BF16, 4001, 2)])
def test_gelu_of_negative_gates_is_relative_to_itself(dtype, rows, width):
    """Gates from -12 to 0 through few rows and the tiles, up 1: the tail alone is left of the value.  bfloat16 adds its
    rounding (2^-8), its shorter fit (9e-6), and the exponent's rounding (up to 72 2^-23)."""
    g = torch.linspace(-12, -0.01, rows, device="cuda").to(dtype)[:, None]
    x = torch.zeros((rows, width), device="cuda", dtype=dtype)
    x[:, :1], x[:, 1] = g, 1.0
    w = torch.zeros((2, width, 8), device="cuda", dtype=dtype)
    w[0, 0], w[1, 1] = 1.0, 1.0
    h = torch.empty((rows, 8), device="cuda", dtype=dtype)
    pd.pd_gated_forward(x, w[0], w[1], h, activation=pd.PD_ACT_GELU)
    # (the formula's 1 + erf loses the tail's digits: erfc has them)
    gn = _np(g)
    ref = gn * 0.5 * np.vectorize(math.erfc)(-gn / math.sqrt(2))
    tol = 2.0**-8 + 1e-5 + 72 * 2.0**-23 if dtype == BF16 else _tail_error() + 2.0**-24
    off = np.abs(_np(h) - ref) / np.abs(ref)
    print(dtype, rows, off.max(), flush=True)
    assert off.max() <= tol


def test_gelu_slope_of_negative_gates_is_relative_to_itself():
    """Gates from -12 to -2, where the slope is g phi(g) and the tail, of which the second is at most a quarter: their
    errors are 5/3 of themselves in the difference."""
    g = torch.linspace(-12, -2, 4001, device="cuda")[:, None].contiguous()
    w = torch.zeros((2, 8, 1), device="cuda")
    w[0, 0], w[1, 1] = 1.0, 1.0
    x, one, dx = torch.zeros((4001, 8), device="cuda"), torch.ones_like(g), torch.empty((4001, 8), device="cuda")
    pd.pd_gated_backward(one, x, w[0], w[1], g, one, dx=dx, activation=pd.PD_ACT_GELU)
    gn = _np(g)
    tail = 0.5 * np.vectorize(math.erfc)(-gn / math.sqrt(2))
    ref = tail + gn * np.exp(-0.5 * gn * gn) / math.sqrt(2 * math.pi)
    off = np.abs(_np(dx)[:, :1] - ref) / np.abs(ref)
    print(off.max(), flush=True)
    assert off.max() <= 5 / 3 * _tail_error() + 2.0**-23        # (and dx's three products in parts)
    off = np.abs(_np(dx)[:, 1:2] - gn * tail) / np.abs(gn * tail)
    assert off.max() <= _tail_error() + 2.0**-23


# ------------------------------------------------------------------ operands read where they are, or laid out
@pytest.mark.parametrize("layout", [pd.PD_WEIGHTS_IN_OUT, pd.PD_WEIGHTS_OUT_IN])
@pytest.mark.parametrize("shift", [0, 1, 4, 8])
@pytest.mark.parametrize("which", ["x", "w_gate", "w_up"])
def test_operands_that_begin_anywhere(which, shift, layout):
    """Rows a multiple of 16 bytes apart, the first of which begins `shift` values after one: through the tiles, forward
    and backward, with the scratch that the binding makes."""
    M, D, F = 300, 128, 264
    def at(shape, seed, name, scale=1.0):
        n = shape[0] * (shape[1] + 8)
        buf = torch.full((n + 16,), float("nan"), device="cuda", dtype=BF16)
        v = buf[shift if name == which else 0:][:n].view(shape[0], shape[1] + 8)[:, :shape[1]]
        return v.copy_(_rand(shape, BF16, seed, scale))
    x = at((M, D), 30, "x")
    wg, wu = (at((F, D), 31 + i, n, D ** -0.5).t() if layout else at((D, F), 31 + i, n, D ** -0.5) for i, n in enumerate(("w_gate", "w_up")))
    dh = _rand((M, F), BF16, 33)
    h, g, u = (torch.empty((M, F), device="cuda", dtype=BF16) for _ in range(3))
    pd.pd_gated_forward(x, wg, wu, h, gate=g, up=u)
    for got, ref in zip((h, g, u), ob.gated(_np(x), _np(wg), _np(wu), "silu")):
        _same(got, ref, 4e-3, "forward")
    dx, dw = torch.empty((M, D), device="cuda", dtype=BF16), [torch.empty_strided(w.shape, (F, 1) if not layout else (1, D), device="cuda", dtype=BF16) for w in (wg, wu)]
    pd.pd_gated_backward(dh, x, wg, wu, g, u, dx=dx, dw_gate=dw[0], dw_up=dw[1])
    for got, ref in zip((dx, *dw), ob.gated_grad(*(_np(t) for t in (dh, x, wg, wu, g, u)), "silu")):
        _same(got, ref, 4e-3, "backward")


def test_forward_of_aligned_operands_takes_no_memory():
    x, w, h = _rand((4096, 1024), BF16, 40), [_rand((1024, 2736), BF16, 41 + i) for i in range(2)], torch.empty((4096, 2736), device="cuda", dtype=BF16)
    torch.cuda.synchronize()
    torch.cuda.reset_peak_memory_stats()
    before = torch.cuda.memory_allocated()
    pd.pd_gated_forward(x, *w, h)
    assert torch.cuda.max_memory_allocated() == before
