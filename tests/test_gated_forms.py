"""Every form of block that the gated product's kernels have, against the formulas in float64.

A product runs in blocks of one of five forms, with its sum whole or in parts, and with as many blocks as tiles or
blocks that go from tile to tile; sizes decide (`cut` in gated.hip).  `SIZES` reaches all of these in every product,
type and layout: a CPU test asks the library how random sizes are cut and looks whether the list has the same."""
import ctypes
import math
import random

import pytest
import torch

import paper_2305_16317_amd as pd

F32, BF16 = torch.float32, torch.bfloat16
ACTS = {"silu": pd.PD_ACT_SILU, "gelu": pd.PD_ACT_GELU, "gelu_tanh": pd.PD_ACT_GELU_TANH, "sigmoid": pd.PD_ACT_SIGMOID,
        "relu": pd.PD_ACT_RELU}
# rows, width, hidden; multiples of 8 (operands read where they are) and others (laid out first)
SIZES = [(1, 1, 1), (336, 1, 1), (268, 3847, 1090), (68959, 1, 1), (6, 269, 10899), (3017, 2, 6067), (35713, 136, 96), (5700, 2832, 8),
         (11994, 784, 136), (399, 1283, 12931), (422, 788, 9476), (1044, 4360, 1576), (1, 979, 1), (21827, 24, 72), (3312, 3936, 632),
         (10943, 184, 1576), (1, 5421, 8632), (99572, 176, 104), (1063, 2720, 3776), (678, 5088, 2880), (69768, 495, 236), (34476, 144, 1096),
         (1744, 2, 12787), (22640, 1120, 163), (3054, 1657, 2729), (33001, 2807, 2), (429, 2121, 5573), (4118, 2280, 3816), (145, 5344, 6176),
         (2374, 1, 12251), (358, 5472, 5688), (8552, 1016, 4152), (5931, 1474, 5681), (430, 6076, 7426)]


def _cuts(M, D, F, dtype, layout):
    """{(product, type, layout, form, in parts, from tile to tile)} of a forward and a backward call."""
    forms = pd.load()._ZN2pd11gated_formsERK13pd_gated_descbPi
    forms.argtypes, forms.restype = [ctypes.c_void_p, ctypes.c_bool, ctypes.c_void_p], ctypes.c_int
    w = D if layout else F
    d = pd._GatedDesc(rows=M, width=D, hidden=F, dtype=dtype, activation=0, weight_layout=layout, aligned=0, x_stride=D, w_gate_stride=w,
                      w_up_stride=w, gate_stride=F, up_stride=F, h_stride=F, dh_stride=F, dx_stride=D, dw_gate_stride=w, dw_up_stride=w)
    out = (ctypes.c_int * 8)()
    found = set()
    for backward, names in ((False, ["forward"]), (True, ["dx", "dw"])):
        for i in range(forms(ctypes.byref(d), backward, out)):
            form, parts, tiles, blocks = out[4 * i:4 * i + 4]
            found.add((names[i], dtype, layout, form, parts > 1, tiles > blocks))
    return found


def _all_cuts(sizes):
    return set().union(*(_cuts(*s, dtype, layout) for s in sizes for dtype in (pd.PD_F32, pd.PD_BF16) for layout in (0, 1)))


def test_sizes_reach_every_form():
    r = random.Random(3)
    some = lambda a, b: int(math.exp(r.uniform(math.log(a), math.log(b + 1))))  # noqa: E731
    have = _all_cuts(SIZES)
    # each form in parts and whole, in each product, type and layout (dw has no blocks of 32 rows)
    assert {k[:5] for k in have} == {(p, t, w, f, s) for p in ("forward", "dx", "dw") for t in (pd.PD_F32, pd.PD_BF16) for w in (0, 1)
                                     for f in range(4 if p == "dw" else 5) for s in (False, True)}
    assert _all_cuts([(some(1, 1 << 17), some(1, 1 << 13), some(1, 1 << 14)) for _ in range(6000)]) <= have


def _close(got, ref, tol, what, size=None):
    """In the root mean square relative to the size, and every element to the largest of its value and the root mean squares of
    all sizes and its row's.  `size`: of each element (None: itself)."""
    size = ref if size is None else size
    off, rms = got.double() - ref, float(size.pow(2).mean().sqrt())
    assert float(off.pow(2).mean().sqrt()) <= tol * rms, (what, float(off.pow(2).mean().sqrt()) / rms)
    size = torch.maximum(ref.abs(), size.pow(2).mean(-1, keepdim=True).sqrt()).clamp_min(rms)
    assert float((off.abs() / size).max()) <= 12 * tol, (what, float((off.abs() / size).max()))


def _activate(g, kind):
    """(act, slope) in float64."""
    s = torch.sigmoid(g)
    if kind == "silu":
        return g * s, s * (1 + g * (1 - s))
    if kind == "gelu":
        p = 0.5 * torch.erfc(-g / math.sqrt(2))
        return g * p, p + g * torch.exp(-0.5 * g * g) / math.sqrt(2 * math.pi)
    if kind == "gelu_tanh":
        r = math.sqrt(2 / math.pi)
        s = torch.sigmoid(2 * r * (g + 0.044715 * g**3))
        return g * s, s + g * s * (1 - s) * 2 * r * (1 + 3 * 0.044715 * g * g)
    return (s, s * (1 - s)) if kind == "sigmoid" else (g.clamp_min(0), (g > 0).double())


@pytest.mark.gpu
@pytest.mark.parametrize("M,D,F", SIZES)
def test_forms_against_float64(M, D, F):
    """Tolerances: float32 products to 2^-24 in parts, and float32 sums of up to 10^5 terms, each of whose partial sums
    (n / 16 a segment) rounds to 2^-25 in the root mean square: 2^-25 sqrt(6 10^5 / 16) / 2 = 3e-6, with the products'
    2^-24 5e-6.  bfloat16: one rounding, of 2^-8 / sqrt 3 at most: 4e-3.

    The partial sums, and so these errors, are as large as the root of the terms' squares, sqrt(sum a^2 b^2), which is a
    gradient's root mean square too where it has many elements.  That of 68959 x 1 x 1 is one sum of 68959 terms: its value
    happened to be -13.7 with terms whose squares add up to some 150^2, and an error of 1.6e-4, 1.1e-6 of them.  So the
    gradients' errors are relative to that root."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    act = sorted(ACTS)[(M + D + F) % 5]
    for dtype, tol in ((F32, 5e-6), (BF16, 4e-3)):
        for layout in (pd.PD_WEIGHTS_IN_OUT, pd.PD_WEIGHTS_OUT_IN):
            print(f"gated {M} x {D} x {F} {dtype} {layout} {act}", flush=True)
            g = torch.Generator(device="cuda").manual_seed(M + layout)
            rand = lambda *s: torch.randn(s, device="cuda", generator=g).to(dtype)  # noqa: E731
            x, dh, gate, up = rand(M, D), rand(M, F), rand(M, F), rand(M, F)
            w = [(rand(*((F, D) if layout else (D, F))) * D ** -0.5).to(dtype) for _ in range(2)]
            w = [v.t() for v in w] if layout else w
            h, dx, dw = torch.full_like(dh, 9.0), torch.full_like(x, 9.0), [torch.full_like(v, 9.0) for v in w]
            pd.pd_gated_forward(x, *w, h, activation=ACTS[act])
            pd.pd_gated_backward(dh, x, *w, gate, up, dx=dx, dw_gate=dw[0], dw_up=dw[1], activation=ACTS[act])
            xd, dhd, wd = x.double(), dh.double(), [v.double().contiguous() for v in w]
            _close(h, _activate(xd @ wd[0], act)[0] * (xd @ wd[1]), tol, "h")
            a, slope = _activate(gate.double(), act)
            dg, du = dhd * up.double() * slope, dhd * a
            of = lambda *pairs: sum(a.square() @ b.square() for a, b in pairs).sqrt()  # noqa: E731
            _close(dx, dg @ wd[0].t() + du @ wd[1].t(), tol, "dx", of((dg, wd[0].t()), (du, wd[1].t())))
            _close(dw[0], xd.t() @ dg, tol, "dw_gate", of((xd.t(), dg)))
            _close(dw[1], xd.t() @ du, tol, "dw_up", of((xd.t(), du)))
