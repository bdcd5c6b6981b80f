"""The operators of a latent transformer's block on the GPU against the oracle in float64.

Tolerances (relative L2 of a whole tensor, and `PEAK` times that for one element against the
largest of its value, the tensor's root mean square and its row's):
  float32   a norm's sums, a product's parts and its sum are 2^-24 each relative to their terms;
            with the activations' functions under 1e-6: 5e-6.
  bfloat16  a rounding is 2^-9 at most in the root mean square 1.7e-3 of the result: 4e-3; gradients
            of the gated product of more than 32 rows round dgate and dup before their products (a
            sum's error is theirs in the root mean square) and the result: 6e-3.
"""
import numpy as np
import pytest
import torch

import paper_2305_16317_amd as pd
from oracle import block as ob

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
TOL = {F32: 5e-6, BF16: 4e-3}
TOL_GRAD = {F32: 5e-6, BF16: 6e-3}
PEAK = 12
NAN = float("nan")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    pd.load()


def _np(t):
    return t.detach().double().cpu().numpy()


def _close(got, ref, tol, what=""):
    got = _np(got) if isinstance(got, torch.Tensor) else got
    assert got.shape == ref.shape, what
    fine = np.isfinite(ref)
    assert np.array_equal(np.isnan(got), np.isnan(ref)), what
    assert np.array_equal(got[~fine & ~np.isnan(ref)], ref[~fine & ~np.isnan(ref)]), what
    g, r = got[fine], ref[fine]
    if not r.size:
        return
    norm, off = np.linalg.norm(r), np.linalg.norm(g - r)
    if norm == 0:
        assert off == 0, what
        return
    assert off <= tol * norm, (what, off / norm)
    vec = np.sqrt(np.mean(np.where(fine, ref, 0.0) ** 2, axis=-1, keepdims=True))
    size = np.maximum(np.maximum(np.abs(ref), vec), norm / np.sqrt(r.size))[fine]
    big = np.max(np.abs(g - r) / size)
    assert big <= PEAK * tol, (what, big)


def _rand(shape, dtype, seed, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, device="cuda", generator=g) * scale).to(dtype)


def _wide(rows, cols, dtype, seed, left=0, right=0, fill=NAN, scale=1.0):
    """Rows cut from a wider buffer that holds `fill` beside them; (view, buffer)."""
    buf = torch.full((rows, left + cols + right), fill, device="cuda", dtype=dtype)
    buf[:, left:left + cols] = _rand((rows, cols), dtype, seed, scale)
    return buf[:, left:left + cols], buf


def _untouched(buf, left, cols, fill):
    out = torch.cat([buf[:, :left], buf[:, left + cols:]], 1)
    return bool((out == fill).all())


# ------------------------------------------------------------------ layer norm
NORM_SIZES = [(1, 1, 0), (3, 7, 3), (5, 8, 0), (4, 64, 2), (9, 511, 3), (17, 512, 0), (6, 513, 2), (34, 1024, 2), (7, 1001, 7),
              (5, 2048, 0), (4, 2049, 2), (2, 4104, 0), (4, 8192, 2), (4, 8193, 2), (3, 20000, 3), (1, 65536, 0), (2, 40000, 0),
              (700, 320, 70), (1200, 96, 2), (2000, 72, 1)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,width,runs", NORM_SIZES)
def test_layernorm_forward(rows, width, runs, dtype):
    print(f"layernorm {rows} x {width} / {runs} {dtype}", flush=True)
    x, r = _rand((rows, width), dtype, 1), (_rand((rows, width), F32, 2, 3.0) + 5.0).to(dtype)
    shape = (runs, width) if runs else (width,)
    w, b = _rand(shape, F32, 3), _rand(shape, F32, 4)
    y, h = torch.full_like(x, 7), torch.full_like(x, 7)
    mean, rstd = (torch.full((rows,), 7.0, device="cuda") for _ in range(2))
    pd.pd_layernorm_forward(x, y, weight=w, bias=b, residual=r, sum_out=h, mean=mean, rstd=rstd, eps=1e-5)
    s, yr, mr, rr = ob.layernorm(_np(x), _np(r), _np(w), _np(b), 1e-5)
    _close(h, s, TOL[dtype])
    _close(y, yr, TOL[dtype])
    _close(mean, mr, 2e-6)
    if width > 1:
        _close(rstd, rr, 2e-6)
    pd.pd_layernorm_forward(x, y, eps=1e-5)                 # neither residual nor weight nor bias
    _close(y, ob.layernorm(_np(x), None, None, None, 1e-5)[1], TOL[dtype])
    pd.pd_layernorm_forward(x, y, bias=b, eps=1e-5)
    _close(y, ob.layernorm(_np(x), None, None, _np(b), 1e-5)[1], TOL[dtype])


def test_layernorm_of_rows_far_from_zero_and_constant_rows():
    """An offset of 1000 beside differences of 1: the squares are summed around the mean, whose rounding of
    2^-24 1000 shifts the normed values by 6e-5 of them."""
    x = _rand((8, 700), F32, 5) + 1000.0
    y = torch.empty_like(x)
    pd.pd_layernorm_forward(x, y)
    ref = ob.layernorm(_np(x), None, None, None, 1e-6)[1]
    assert np.max(np.abs(_np(y) - ref)) <= 2.0**-24 * 1000 * 2 + 1e-5
    x = torch.full((3, 65), 2.5, device="cuda")
    y = torch.full_like(x, 7)
    pd.pd_layernorm_forward(x, y, bias=_rand((65,), F32, 6))
    assert torch.equal(y, _rand((65,), F32, 6).expand(3, 65))


def test_layernorm_rows_with_nan_keep_to_themselves():
    x, w = _rand((9, 300), BF16, 7), _rand((300,), F32, 8)
    ref = ob.layernorm(_np(x), None, _np(w), None, 1e-6)[1]
    x[4, 7] = NAN
    y = torch.empty_like(x)
    pd.pd_layernorm_forward(x, y, weight=w)
    assert torch.isnan(y[4]).all()
    keep = [i for i in range(9) if i != 4]
    _close(y[keep], ref[keep], TOL[BF16])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,width,runs", [c for c in NORM_SIZES if c[1] > 1] + [(3000, 96, 0), (64, 40, 64), (5000, 24, 1000)])
def test_layernorm_backward(rows, width, runs, dtype):
    print(f"layernorm backward {rows} x {width} / {runs} {dtype}", flush=True)
    dy, ds = _rand((rows, width), dtype, 10), _rand((rows, width), dtype, 11)
    h = (_rand((rows, width), F32, 12, 2.0) + 1.0).to(dtype)
    shape = (runs, width) if runs else (width,)
    w = _rand(shape, F32, 13)
    mean = h.double().mean(1).float()
    rstd = torch.rsqrt(h.double().var(1, unbiased=False) + 1e-6).float()
    dx, dw, db = torch.full_like(dy, 7), torch.full(shape, 7.0, device="cuda"), torch.full(shape, 7.0, device="cuda")
    pd.pd_layernorm_backward(dy, h, mean, rstd, dx, weight=w, dweight=dw, dbias=db, dsum=ds)
    args = (_np(dy), _np(h), _np(w), _np(mean), _np(rstd))
    rx, rw, rb = ob.layernorm_grad(*args, _np(ds), runs)
    _close(dx, rx, TOL[dtype])
    _close(dw, rw, 5e-6)
    _close(db, rb, 5e-6)
    again = torch.empty_like(dw)
    pd.pd_layernorm_backward(dy, h, mean, rstd, dx, weight=w, dweight=again)      # the same bits again, alone
    _close(dx, ob.layernorm_grad(*args, None, runs)[0], TOL[dtype])
    assert torch.equal(again, dw)
    pd.pd_layernorm_backward(dy, h, mean, rstd, dx, dbias=again)                  # without a weight
    assert torch.equal(again, db)
    _close(dx, ob.layernorm_grad(_np(dy), _np(h), None, _np(mean), _np(rstd), None, runs)[0], TOL[dtype])
    pd.pd_layernorm_backward(dy, h, mean, rstd, dy, weight=w)                     # over dy, dx alone
    _close(dy, ob.layernorm_grad(*args, None, runs)[0], TOL[dtype])


def test_layernorm_backward_in_place_with_sums():
    """dx over dy while dweight is summed from dy, also where the sums have a pass of their own."""
    for width in (300, 9000):
        dy, h, w = _rand((12, width), F32, 14), _rand((12, width), F32, 15), _rand((width,), F32, 16)
        mean, rstd = h.mean(1), torch.rsqrt(h.var(1, unbiased=False))
        dw = torch.empty_like(w)
        rx, rw, _ = ob.layernorm_grad(_np(dy), _np(h), _np(w), _np(mean), _np(rstd), None)
        pd.pd_layernorm_backward(dy, h, mean, rstd, dy, weight=w, dweight=dw)
        _close(dy, rx, TOL[F32])
        _close(dw, rw, 5e-6)


def test_layernorm_backward_of_no_rows_and_against_differences():
    z = torch.empty((0, 40), device="cuda")
    none = torch.empty(0, device="cuda")
    dw, db = torch.full((40,), 7.0, device="cuda"), torch.full((40,), 7.0, device="cuda")
    pd.pd_layernorm_backward(z, z, none, none, torch.empty_like(z), dweight=dw, dbias=db)
    assert torch.all(dw == 0) and torch.all(db == 0)
    dw = torch.full((3, 40), 7.0, device="cuda")
    pd.pd_layernorm_backward(z, z, none, none, torch.empty_like(z), dweight=dw)        # runs without rows
    assert torch.all(dw == 0)
    pd.pd_layernorm_forward(z, torch.empty_like(z))
    x, dy, w, d = (_rand(s, F32, 20 + i) for i, s in enumerate([(4, 50), (4, 50), (2, 50), (4, 50)]))
    y, h, mean, rstd, dx = torch.empty_like(x), torch.empty_like(x), *(torch.empty(4, device="cuda") for _ in range(2)), torch.empty_like(x)
    pd.pd_layernorm_forward(x, y, weight=w, sum_out=h, mean=mean, rstd=rstd)
    pd.pd_layernorm_backward(dy, h, mean, rstd, dx, weight=w)
    loss = lambda e: float(np.sum(ob.layernorm(_np(x) + e * _np(d), None, _np(w), None, 1e-6)[1] * _np(dy)))  # noqa: E731
    want = (loss(1e-5) - loss(-1e-5)) / 2e-5
    assert abs(float((dx.double() * d.double()).sum()) - want) <= 1e-5 * float(dx.norm() * d.norm())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("width", [515, 1027, 2049, 4099, 4610, 8195, 16387, 32770])
def test_layernorm_in_place_at_odd_widths(width, dtype):
    """Widths whose last values are read together with a neighbour's, in another wave or step."""
    print(f"layernorm in place {width} {dtype}", flush=True)
    rows = 300
    x, r, w = _rand((rows, width), dtype, 31), _rand((rows, width), dtype, 32), _rand((3, width), F32, 33)
    s, y, mean, rstd = ob.layernorm(_np(x), _np(r), _np(w), None, 1e-6)
    y2, r2 = x.clone(), r.clone()
    pd.pd_layernorm_forward(y2, y2, weight=w, residual=r2, sum_out=r2)
    _close(y2, y, TOL[dtype])
    _close(r2, s, TOL[dtype])
    mean, rstd = (torch.from_numpy(v).float().cuda() for v in (mean, rstd))
    h, dw, db = r2, torch.empty_like(w), torch.empty_like(w)
    rx, rw, rb = ob.layernorm_grad(_np(x), _np(h), _np(w), _np(mean), _np(rstd), _np(r), 3)
    for over in (0, 1):                                     # dx over dy, over dsum; with the sums and alone
        dy, ds = x.clone(), r.clone()
        pd.pd_layernorm_backward(dy, h, mean, rstd, (dy, ds)[over], weight=w, dweight=dw, dbias=db, dsum=ds)
        _close((dy, ds)[over], rx, TOL[dtype])
        _close(dw, rw, 5e-6)
        _close(db, rb, 5e-6)
        dy, ds = x.clone(), r.clone()
        pd.pd_layernorm_backward(dy, h, mean, rstd, (dy, ds)[over], weight=w, dsum=ds)
        _close((dy, ds)[over], rx, TOL[dtype])


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_layernorm_strides_and_in_place(dtype):
    x, bx = _wide(6, 33, dtype, 25, 3, 14, 9.0)             # rows that start at no multiple of 16 bytes
    res, bres = _wide(6, 33, dtype, 26, 5, 2, 9.0)
    m = _rand((2, 80), F32, 27)                             # weight and bias side by side, as one product makes them
    w, b = m[:, 1:34], m[:, 40:73]
    s, y, _, _ = ob.layernorm(_np(x), _np(res), _np(w), _np(b), 1e-6)
    pd.pd_layernorm_forward(x, x, weight=w, bias=b, residual=res, sum_out=res)
    _close(x, y, TOL[dtype])
    _close(res, s, TOL[dtype])
    assert _untouched(bx, 3, 33, 9.0) and _untouched(bres, 5, 33, 9.0)
    x3 = _rand((2, 3, 33), dtype, 28)
    y3 = torch.empty_like(x3)
    pd.pd_layernorm_forward(x3, y3, weight=w)
    _close(y3.view(6, 33), ob.layernorm(_np(x3).reshape(6, 33), None, _np(w), None, 1e-6)[1], TOL[dtype])


def test_layernorm_of_more_rows_than_a_launch_holds():
    rows = (1 << 21) + 6
    x, w = _rand((rows, 8), BF16, 29), _rand((2, 8), F32, 30)
    y, mean = torch.empty_like(x), torch.empty(rows, device="cuda")
    pd.pd_layernorm_forward(x, y, weight=w, mean=mean)
    for part, run in ((slice(0, 5), 0), (slice(rows // 2 - 4, rows // 2), 0), (slice(rows // 2, rows // 2 + 4), 1), (slice(rows - 5, rows), 1)):
        _, yr, mr, _ = ob.layernorm(_np(x[part]), None, _np(w[run]), None, 1e-6)
        _close(y[part], yr, TOL[BF16])
        _close(mean[part], mr, 2e-6)


def test_layernorm_refuses_what_it_cannot_read():
    x, w, r = torch.zeros((4, 8), device="cuda"), torch.ones(8, device="cuda"), torch.empty(4, device="cuda")
    e = torch.empty_like(x)
    for bad in (lambda: pd.pd_layernorm_forward(x.t(), torch.empty((8, 4), device="cuda")),
                lambda: pd.pd_layernorm_forward(x, e, weight=w[:7]), lambda: pd.pd_layernorm_forward(x, e, weight=w.to(BF16)),
                lambda: pd.pd_layernorm_forward(x, e, weight=torch.ones((3, 8), device="cuda")),
                lambda: pd.pd_layernorm_forward(x, e, weight=torch.ones((2, 8), device="cuda"), bias=torch.ones((4, 8), device="cuda")),
                lambda: pd.pd_layernorm_forward(x, e.to(BF16)), lambda: pd.pd_layernorm_forward(x, w.expand(4, 8)),
                lambda: pd.pd_layernorm_forward(x, e, mean=r[:3]), lambda: pd.pd_layernorm_forward(x, e, rstd=r.double()),
                lambda: pd.pd_layernorm_backward(x, x, r, r, e, weight=w.expand(2, 8), dweight=torch.empty(8, device="cuda")),
                lambda: pd.pd_layernorm_backward(x, x, r, r, e, dweight=torch.empty((2, 8), device="cuda"), dbias=torch.empty(8, device="cuda")),
                lambda: pd.pd_layernorm_backward(x, x, r, r[:2], e)):
        with pytest.raises(ValueError):
            bad()
    big, stats = torch.zeros((64, 8), device="cuda"), torch.empty(64, device="cuda")
    with pytest.raises(pd.PdError):
        pd.pd_layernorm_backward(big, big, stats, stats, torch.empty_like(big), dweight=torch.empty(8, device="cuda"),
                                 scratch=torch.empty(4, device="cuda", dtype=torch.uint8))


# ------------------------------------------------------------------ rotary positions over axes
SECTIONS = [[8], [4, 4], [16, 24, 24], [1, 0, 6], [3, 5, 2, 7], [13, 19]]


@pytest.mark.parametrize("sections", SECTIONS)
@pytest.mark.parametrize("order,shared", [(pd.PD_AXES_RUNS, False), (pd.PD_AXES_TURNS, False), (pd.PD_AXES_TURNS, True)])
def test_rotary_axes_table(sections, order, shared):
    """The same double-precision formula: a rounding to float32 apart."""
    n = len(sections)
    base, scale = [100.0 + 50 * a for a in range(n)], [1.0, 0.5, 2.0, -1.25][:n]
    t = torch.empty((9, sum(sections), 2), device="cuda")
    pd.pd_rotary_axes_table(t, sections, base=base, scale=scale, order=order, shared=shared, first=3)
    ref = ob.axes_table(sections, order == pd.PD_AXES_TURNS, range(3, 12), base, scale, shared)
    assert np.max(np.abs(_np(t) - ref)) <= 2.0**-24


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("layout", [pd.PD_ROTARY_HALF, pd.PD_ROTARY_INTERLEAVED])
@pytest.mark.parametrize("order", [pd.PD_AXES_RUNS, pd.PD_AXES_TURNS])
@pytest.mark.parametrize("sections", SECTIONS)
def test_rotary_axes(sections, order, layout, dtype):
    half, n = sum(sections), len(sections)
    B, L, H, K, D = 2, 11, 6, 3, 2 * half + (5 if half % 2 else 0)
    print(f"rotary axes {sections} {order} {layout} {dtype}", flush=True)
    t = torch.empty((13, half, 2), device="cuda")
    pd.pd_rotary_axes_table(t, sections, base=50.0, order=order)
    both = _rand((B, L, H + K, D), dtype, 40)
    q, k = both.split([H, K], 2)
    g = torch.Generator().manual_seed(7)
    pos = torch.randint(-2, 16, (B, L, n), generator=g, dtype=torch.int32).cuda()        # some outside the table
    axis = ob.axis_of_pair(sections, order == pd.PD_AXES_TURNS)
    for back in (False, True):
        qo, ko = torch.full((B, L, H, D), 7.0, device="cuda", dtype=dtype), torch.full((B, L, K, D), 7.0, device="cuda", dtype=dtype)
        pd.pd_rotary_axes_apply(q, k, pos, t, sections, qo, ko, layout=layout, order=order, backward=back)
        for x, got in ((q, qo), (k, ko)):
            _close(got, ob.rotary_axes(_np(x), _np(t), pos.cpu().numpy(), axis, layout == pd.PD_ROTARY_INTERLEAVED, back), TOL[dtype])
    # axes as rows of the positions, shared by the batch; in place; q alone
    rows = pos[0].t().contiguous()
    ref = ob.rotary_axes(_np(q), _np(t), np.repeat(pos[:1].cpu().numpy(), B, 0), axis, layout == pd.PD_ROTARY_INTERLEAVED)
    before = k.clone()
    pd.pd_rotary_axes_apply(q, None, rows.t(), t, sections, q, layout=layout, order=order)
    _close(q, ref, TOL[dtype])
    assert torch.equal(k, before)


def test_rotary_axes_of_one_axis_is_rotary():
    t = torch.empty((20, 16, 2), device="cuda")
    pd.pd_rotary_axes_table(t, [16])
    one = torch.empty_like(t)
    pd.pd_rotary_table(one)
    assert float((t - one).abs().max()) <= 2.0**-23       # the same angles, formed from -i/16 and from -2i/32
    q = _rand((2, 20, 4, 40), BF16, 41)
    pos = torch.arange(20, device="cuda", dtype=torch.int32)
    a, b = torch.empty_like(q), torch.empty_like(q)
    pd.pd_rotary_apply(q, None, pos, t, a)
    pd.pd_rotary_axes_apply(q, None, pos[:, None], t, [16], b)
    assert torch.equal(a, b)


def test_rotary_axes_refuses_what_it_cannot_read():
    q, t = torch.zeros((1, 4, 2, 16), device="cuda"), torch.zeros((4, 8, 2), device="cuda")
    pos = torch.zeros((4, 2), device="cuda", dtype=torch.int32)
    for bad in (lambda: pd.pd_rotary_axes_apply(q, None, pos, t, [8], q), lambda: pd.pd_rotary_axes_apply(q, None, pos.long(), t, [4, 4], q),
                lambda: pd.pd_rotary_axes_apply(q, None, pos, t, [], q), lambda: pd.pd_rotary_axes_apply(q, None, pos, t, [2, 2, 2, 1, 1], q),
                lambda: pd.pd_rotary_axes_table(t, [4, 4], base=[1e4]), lambda: pd.pd_rotary_axes_table(t[:, ::2], [4])):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: pd.pd_rotary_axes_apply(q, None, pos, t, [4, 5], q), lambda: pd.pd_rotary_axes_apply(q, None, pos, t, [9, -1], q),
                lambda: pd.pd_rotary_axes_apply(q, None, pos, t, [4, 4], q, order=2)):
        with pytest.raises(pd.PdError):
            bad()


# ------------------------------------------------------------------ dropout
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,width,p", [(1, 1, 0.5), (3, 7, 0.3), (5, 8, 0.1), (16, 1024, 0.1), (33, 100, 0.25), (257, 1001, 0.5),
                                          (2, 40000, 0.9), (1000, 16, 1e-4), (40, 64, 0.0), (40, 64, 1.0)])
def test_dropout(rows, width, p, dtype):
    print(f"dropout {rows} x {width} {p} {dtype}", flush=True)
    x, r = _rand((rows, width), dtype, 50), _rand((rows, width), dtype, 51)
    seed, stream, step = 0xFEDCBA9876543210, 5, 77
    keep = ob.kept(rows, width, p, seed, stream, step)
    y = torch.full_like(x, 7)
    pd.pd_dropout_apply(x, y, p, seed, rng_stream=stream, step=step)
    assert np.array_equal(_np(y) != 0, keep & (_np(x) != 0))
    _close(y, ob.dropout(_np(x), None, p, keep), TOL[dtype])
    pd.pd_dropout_apply(x, y, p, seed, rng_stream=stream, step=step, residual=r)
    _close(y, ob.dropout(_np(x), _np(r), p, keep), TOL[dtype])
    half = rows // 2                                       # a call on part of the rows, and the step from the device
    more = torch.tensor([70], device="cuda", dtype=torch.int32)
    part = y[half:].clone()
    pd.pd_dropout_apply(x[half:], part, p, seed, rng_stream=stream, step=step - 70, step_more=more, residual=r[half:], first_row=half)
    assert torch.equal(part, y[half:])


def test_dropout_strides_in_place_and_numbers_that_are_none():
    x, buf = _wide(20, 61, BF16, 52, 3, 6, 9.0)
    keep = ob.kept(20, 61, 0.4, 3, 0, 0)
    ref = ob.dropout(_np(x), None, 0.4, keep)
    pd.pd_dropout_apply(x, x, 0.4, 3)
    _close(x, ref, TOL[BF16])
    assert _untouched(buf, 3, 61, 9.0)
    bad = torch.tensor([NAN, float("inf")], device="cuda").repeat(20, 16)
    y = torch.empty_like(bad)
    pd.pd_dropout_apply(bad, y, 0.4, 3)
    keep = torch.from_numpy(ob.kept(20, 32, 0.4, 3, 0, 0)).cuda()
    assert torch.all(y[~keep] == 0) and torch.equal(torch.isfinite(y), ~keep)
    x, r = _rand((6, 40), F32, 53), _rand((6, 40), F32, 54)
    ref = ob.dropout(_np(x), _np(r), 0.2, ob.kept(6, 40, 0.2, 2**63 + 1, 2**32 - 1, 2**32 - 2))
    pd.pd_dropout_apply(x, r, 0.2, 2**63 + 1, rng_stream=2**32 - 1, step=2**32 - 2, residual=r)      # over the residual
    _close(r, ref, TOL[F32])


def test_dropout_shares_and_streams_differ():
    """The kept share of 2^20 values is within 5 standard deviations of 1 - p; another seed, stream or step gives
    another mask, half of whose values agree where p is 1/2."""
    x = torch.ones((1024, 1024), device="cuda")
    y = torch.empty_like(x)
    masks = []
    for kw in (dict(seed=1), dict(seed=2), dict(seed=1, rng_stream=1), dict(seed=1, step=1), dict(seed=1, first_row=1024)):
        pd.pd_dropout_apply(x, y, 0.5, **kw)
        masks.append(y != 0)
        assert abs(float(masks[-1].double().mean()) - 0.5) < 5 * 0.5 / 1024
    for i in range(len(masks)):
        for j in range(i):
            assert abs(float((masks[i] == masks[j]).double().mean()) - 0.5) < 5 * 0.5 / 1024


def test_dropout_far_rows_use_the_counters_high_word():
    x = torch.ones((4, 64), device="cuda")
    y = torch.empty_like(x)
    first = 2**29 + 12345                                  # 8 blocks a row: past 2^32
    pd.pd_dropout_apply(x, y, 0.5, 9, first_row=first)
    assert np.array_equal(_np(y) != 0, ob.kept(4, 64, 0.5, 9, 0, 0, first))


def test_dropout_backward_is_the_same_mask():
    x, dy = _rand((50, 70), F32, 55), _rand((50, 70), F32, 56)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    pd.pd_dropout_apply(x, y, 0.3, 4, step=2)
    pd.pd_dropout_apply(dy, dx, 0.3, 4, step=2)
    d = _rand((50, 70), F32, 57)
    more = torch.empty_like(x)
    pd.pd_dropout_apply(x + d, more, 0.3, 4, step=2)
    want = float(((more.double() - y.double()) * dy.double()).sum())          # (linear in x)
    assert abs(float((dx.double() * d.double()).sum()) - want) <= 1e-5 * float(dx.norm() * d.norm())


def test_dropout_refuses():
    x = torch.zeros((4, 8), device="cuda")
    y = torch.empty_like(x)
    for kw in (dict(p=-0.1), dict(p=1.1), dict(p=NAN), dict(p=0.1, step=2**32 - 1), dict(p=0.1, first_row=-1)):
        with pytest.raises(pd.PdError):
            pd.pd_dropout_apply(x, y, seed=1, **kw)
    for bad in (lambda: pd.pd_dropout_apply(x, y, 0.1, -1), lambda: pd.pd_dropout_apply(x, y, 0.1, 2**64),
                lambda: pd.pd_dropout_apply(x, y[:1].expand(4, 8), 0.1, 1), lambda: pd.pd_dropout_apply(x, y.to(BF16), 0.1, 1),
                lambda: pd.pd_dropout_apply(x, y, 0.1, 1, step_more=torch.zeros(1, device="cuda"))):
        with pytest.raises(ValueError):
            bad()


# ------------------------------------------------------------------ gated product
ACTS = {"silu": pd.PD_ACT_SILU, "gelu": pd.PD_ACT_GELU, "gelu_tanh": pd.PD_ACT_GELU_TANH, "sigmoid": pd.PD_ACT_SIGMOID,
        "relu": pd.PD_ACT_RELU}
GATED = [(1, 1, 1), (1, 8, 8), (2, 7, 5), (1, 1024, 264), (3, 64, 100), (4, 333, 65), (5, 40, 24), (8, 512, 72), (9, 130, 250),
         (16, 256, 128), (17, 128, 520), (24, 1000, 96), (31, 72, 33), (32, 64, 256), (33, 100, 64), (64, 320, 136), (100, 63, 129),
         (128, 128, 64), (129, 200, 333), (300, 96, 200), (257, 584, 8), (515, 1, 130)]


def _weights(D, F, dtype, seed, layout, pad=0):
    """Weights as (width, hidden), whose rows or columns are contiguous; pad: cut from buffers that are wider and hold
    NaN there."""
    out = []
    for i in range(2):
        shape = (D, F) if layout == pd.PD_WEIGHTS_IN_OUT else (F, D)
        w, _ = _wide(*shape, dtype, seed + i, 0, pad, NAN, D ** -0.5)
        out.append(w if layout == pd.PD_WEIGHTS_IN_OUT else w.t())
    return out


def _forward(x, wg, wu, act, dtype, keep=True, guard=3):
    """h (and gate, up) into wider buffers, of which nothing else is written."""
    M, F = x.shape[0], wg.shape[1]
    bufs = [torch.full((M, F + guard), 9.0, device="cuda", dtype=dtype) for _ in range(3)]
    h, g, u = (b[:, 1:F + 1] for b in bufs)
    pd.pd_gated_forward(x, wg, wu, h, gate=g if keep else None, up=u if keep else None, activation=ACTS[act])
    for b in bufs[:3 if keep else 1]:
        assert _untouched(b, 1, F, 9.0)
    return h, g, u


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("layout", [pd.PD_WEIGHTS_IN_OUT, pd.PD_WEIGHTS_OUT_IN])
@pytest.mark.parametrize("M,D,F", GATED)
def test_gated_forward(M, D, F, layout, dtype):
    act = sorted(ACTS)[(M + D + F) % 5]
    print(f"gated {M} x {D} x {F} {layout} {dtype} {act}", flush=True)
    for pad in (0, 8, 3):                                   # as it lies, whole units apart, no alignment
        x, _ = _wide(M, D, dtype, 60, 0, pad)
        wg, wu = _weights(D, F, dtype, 61, layout, pad)
        h, g, u = _forward(x, wg, wu, act, dtype, keep=pad != 8)
        rh, rg, ru = ob.gated(_np(x), _np(wg), _np(wu), act)
        _close(h, rh, TOL[dtype], "h")
        if pad != 8:
            _close(g, rg, TOL[dtype], "gate")
            _close(u, ru, TOL[dtype], "up")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("layout", [pd.PD_WEIGHTS_IN_OUT, pd.PD_WEIGHTS_OUT_IN])
@pytest.mark.parametrize("M,D,F", GATED)
def test_gated_backward(M, D, F, layout, dtype):
    act = sorted(ACTS)[(M + 2 * D + F) % 5]
    print(f"gated backward {M} x {D} x {F} {layout} {dtype} {act}", flush=True)
    for pad in (0, 8, 3):
        x, _ = _wide(M, D, dtype, 70, 0, pad)
        wg, wu = _weights(D, F, dtype, 71, layout, pad)
        g, _ = _wide(M, F, dtype, 73, 0, pad)
        u, _ = _wide(M, F, dtype, 74, pad, 0)
        dh, _ = _wide(M, F, dtype, 75, 1, pad)
        dxb, hb = torch.full((M, D + 3), 9.0, device="cuda", dtype=dtype), torch.full((M, F + 3), 9.0, device="cuda", dtype=dtype)
        dw = [torch.full(w.t().shape if layout else w.shape, 9.0, device="cuda", dtype=dtype) for w in (wg, wu)]
        dw = [w.t() for w in dw] if layout else dw
        pd.pd_gated_backward(dh, x, wg, wu, g, u, dx=dxb[:, 2:D + 2], dw_gate=dw[0], dw_up=dw[1], h=hb[:, :F], activation=ACTS[act])
        rx, rg, ru, rh = ob.gated_grad(*(_np(t) for t in (dh, x, wg, wu, g, u)), act)
        assert _untouched(dxb, 2, D, 9.0) and _untouched(hb, 0, F, 9.0)
        tol = TOL_GRAD[dtype] if M > 32 else TOL[dtype]     # (few rows keep dgate and dup in two parts)
        _close(dxb[:, 2:D + 2], rx, tol, "dx")
        _close(dw[0], rg, tol, "dw_gate")
        _close(dw[1], ru, tol, "dw_up")
        _close(hb[:, :F], rh, TOL[dtype], "h")
    again = [torch.empty_like(t) for t in (x, *dw)]          # each alone: the same bits
    pd.pd_gated_backward(dh, x, wg, wu, g, u, dx=again[0], activation=ACTS[act])
    pd.pd_gated_backward(dh, x, wg, wu, g, u, dw_gate=again[1], dw_up=again[2], activation=ACTS[act])
    assert torch.equal(again[0], dxb[:, 2:D + 2]) and torch.equal(again[1], dw[0]) and torch.equal(again[2], dw[1])


@pytest.mark.parametrize("layout", [pd.PD_WEIGHTS_IN_OUT, pd.PD_WEIGHTS_OUT_IN])
@pytest.mark.parametrize("M,D,F", [(4100, 136, 2056), (2304, 320, 1336), (8200, 72, 1000), (6200, 264, 1544), (1700, 200, 2731)])
def test_gated_of_many_tiles(M, D, F, layout):
    """Enough tiles for the large blocks; the sums over many rows in parts."""
    x, dh = _rand((M, D), BF16, 80), _rand((M, F), BF16, 81)
    wg, wu = _weights(D, F, BF16, 82, layout)
    h, g, u = _forward(x, wg, wu, "silu", BF16, guard=8)
    rh, rg, ru = ob.gated(_np(x), _np(wg), _np(wu), "silu")
    for got, ref in ((h, rh), (g, rg), (u, ru)):
        _close(got, ref, TOL[BF16])
    dx, dw = torch.empty_like(x), [torch.empty_like(w) for w in (wg, wu)]
    pd.pd_gated_backward(dh, x, wg, wu, g, u, dx=dx, dw_gate=dw[0], dw_up=dw[1])
    rx, rg, ru, _ = ob.gated_grad(*(_np(t) for t in (dh, x, wg, wu, g, u)), "silu")
    for got, ref in ((dx, rx), (dw[0], rg), (dw[1], ru)):
        _close(got, ref, TOL_GRAD[BF16])


def test_gated_activations_of_infinite_gates():
    """Through few rows, many rows and bfloat16: act(inf) = inf (the sigmoid: 1), and NaN stays."""
    for dtype, rows in ((BF16, 4), (BF16, 300)):            # (float32 products give NaN for an infinity)
        g = torch.tensor([float("inf"), NAN, 3.0], device="cuda").repeat(rows, 1).to(dtype)
        x = torch.cat([g[:, :1], torch.ones_like(g[:, :1])], 1)
        for act in ACTS:
            for value, want in ((float("inf"), 1.0 if act == "sigmoid" else float("inf")), (NAN, NAN), (-200.0, 0.0)):
                x[:, 0] = value
                wg, wu = torch.tensor([[1.0], [0.0]], device="cuda", dtype=dtype), torch.tensor([[0.0], [1.0]], device="cuda", dtype=dtype)
                x2 = x.clone()
                h = torch.empty((rows, 1), device="cuda", dtype=dtype)
                up = torch.empty_like(h)
                pd.pd_gated_forward(x2, wg, wu, h, up=up, activation=ACTS[act])
                if value == value and abs(value) != float("inf"):
                    assert torch.all(h == want), (act, value)
                else:                                       # 0 times the value is NaN in up, and so in h
                    assert torch.isnan(up).all() and torch.isnan(h).all()
        # the slopes' kernel alone: h from gate and up as stored
        for act in ACTS:
            gate = torch.tensor([[float("inf"), NAN, -200.0, 200.0]], device="cuda", dtype=dtype).repeat(rows, 2)
            one, h = torch.ones_like(gate), torch.empty_like(gate)
            w = torch.zeros((8, 8), device="cuda", dtype=dtype)
            pd.pd_gated_backward(one, torch.zeros((rows, 8), device="cuda", dtype=dtype), w, w, gate, one, h=h, activation=ACTS[act])
            top = 1.0 if act == "sigmoid" else float("inf")
            assert torch.all(h[:, 0] == top) and torch.isnan(h[:, 1]).all() and torch.all(h[:, 2] == 0), act
            assert torch.all(h[:, 3] == (1.0 if act == "sigmoid" else 200.0)), act


@pytest.mark.parametrize("act", sorted(ACTS))
def test_gated_activations_far_out(act):
    """Gates from -200 to 200: exponentials that overflow; x is the gate and up is 1."""
    g = torch.linspace(-200, 200, 4001, device="cuda")[:, None].contiguous()
    x = torch.cat([g, torch.ones_like(g)], 1)
    wg, wu = torch.tensor([[1.0], [0.0]], device="cuda"), torch.tensor([[0.0], [1.0]], device="cuda")
    h = torch.empty_like(g)
    pd.pd_gated_forward(x, wg, wu, h, activation=ACTS[act])
    a, slope = ob.activate(_np(g), act)
    # the functions' own errors near 1, relative to what they are added to: a few 2^-24 of max(1, |g|)
    lim = 1e-6 * np.maximum(1, np.abs(_np(g)))
    assert np.all(np.abs(_np(h) - a) <= lim)
    dx = torch.empty_like(x)
    pd.pd_gated_backward(torch.ones_like(g), x, wg, wu, g, torch.ones_like(g), dx=dx, activation=ACTS[act])
    assert np.all(np.abs(_np(dx)[:, :1] - slope) <= 1e-5) and np.all(np.abs(_np(dx)[:, 1:] - a) <= lim)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("layout", [pd.PD_WEIGHTS_IN_OUT, pd.PD_WEIGHTS_OUT_IN])
@pytest.mark.parametrize("M", [3, 40, 200])
def test_gated_nan_reaches_its_row_and_column_alone(M, layout, dtype):
    D, F = 72, 100
    x = _rand((M, D), dtype, 90)
    wg, wu = _weights(D, F, dtype, 91, layout)
    rh, rg, ru = ob.gated(_np(x), _np(wg), _np(wu), "silu")
    x[M - 1, D - 1], wg[5, F - 1] = NAN, NAN
    h, g, u = _forward(x, wg, wu, "silu", dtype)
    for got, ref, col in ((h, rh, True), (g, rg, True), (u, ru, False)):
        ref = ref.copy()
        ref[M - 1] = NAN
        if col:
            ref[:, F - 1] = NAN
        _close(got, ref, TOL[dtype])
    dh = _rand((M, F), dtype, 93)
    x, (wg, wu) = _rand((M, D), dtype, 90), _weights(D, F, dtype, 91, layout)
    g, u = _rand((M, F), dtype, 94), _rand((M, F), dtype, 95)
    rx, rg, ru, _ = ob.gated_grad(*(_np(t) for t in (dh, x, wg, wu, g, u)), "silu")
    dh[M - 1, F - 1] = NAN
    dx, dw = torch.empty_like(x), [torch.empty_like(w) for w in (wg, wu)]
    pd.pd_gated_backward(dh, x, wg, wu, g, u, dx=dx, dw_gate=dw[0], dw_up=dw[1])
    rx[M - 1], rg[:, F - 1], ru[:, F - 1] = NAN, NAN, NAN
    for got, ref in ((dx, rx), (dw[0], rg), (dw[1], ru)):
        _close(got, ref, TOL_GRAD[dtype])


def test_gated_float32_of_large_and_small_values():
    """Values over the whole range of float32: relative to the sum of the terms' sizes."""
    M, D, F = 40, 90, 70
    x = _rand((M, D), F32, 100) * torch.exp2(_rand((M, D), F32, 101, 20.0))
    wg, wu = (_rand((D, F), F32, 102 + i) * torch.exp2(_rand((D, F), F32, 104 + i, 15.0)) for i in range(2))
    x[0, 0], wu[0, 0] = 3.4e38, 2.0**-100                     # (past the largest bfloat16)
    h, g, u = _forward(x, wg, wu, "relu", F32)
    for got, w in ((g, wg), (u, wu)):
        ref, size = _np(x) @ _np(w), np.abs(_np(x)) @ np.abs(_np(w))
        fine = size < 3e38
        assert fine.mean() > 0.9
        assert np.all(np.abs(_np(got) - ref)[fine] <= 5e-6 * size[fine])


def test_gated_backward_against_differences():
    M, D, F = 6, 20, 14
    x, dh, d = _rand((M, D), F32, 110), _rand((M, F), F32, 111), _rand((M, D), F32, 112)
    wg, wu = _weights(D, F, F32, 113, pd.PD_WEIGHTS_OUT_IN)
    for act in ACTS:
        h, g, u = _forward(x, wg, wu, act, F32)
        dx, dw = torch.empty_like(x), [torch.empty_like(w) for w in (wg, wu)]
        pd.pd_gated_backward(dh, x, wg, wu, g, u, dx=dx, dw_gate=dw[0], dw_up=dw[1], activation=ACTS[act])
        args = [_np(t) for t in (x, wg, wu)]
        for which, (got, e) in enumerate(((dx, _np(d)), (dw[0], _np(_rand((D, F), F32, 114))), (dw[1], _np(_rand((D, F), F32, 115))))):
            def loss(t):
                a = list(args)
                a[which] = a[which] + t * e
                return float(np.sum(ob.gated(*a, act)[0] * _np(dh)))
            want = (loss(1e-6) - loss(-1e-6)) / 2e-6
            # (relu: no gate lies within the step of 0)
            assert abs(float(np.sum(_np(got) * e)) - want) <= 2e-5 * float(got.norm()) * np.linalg.norm(e), act


def test_gated_no_rows():
    wg, wu = _weights(24, 40, F32, 120, pd.PD_WEIGHTS_IN_OUT)
    x, h = torch.empty((0, 24), device="cuda"), torch.empty((0, 40), device="cuda")
    pd.pd_gated_forward(x, wg, wu, h)
    for layout in (0, 1):
        dw = [torch.full((24, 40), 7.0, device="cuda") if not layout else torch.full((40, 24), 7.0, device="cuda").t() for _ in range(2)]
        a, b = (wg, wu) if not layout else (wg.t().contiguous().t(), wu.t().contiguous().t())
        pd.pd_gated_backward(h, x, a, b, h, h, dx=x, dw_gate=dw[0], dw_up=dw[1])
        assert all(torch.all(w == 0) for w in dw)


def test_gated_refuses_what_it_cannot_read():
    x, w, h = torch.zeros((4, 8), device="cuda"), torch.zeros((8, 16), device="cuda"), torch.zeros((4, 16), device="cuda")
    for bad in (lambda: pd.pd_gated_forward(x, w, w[:, :8], h), lambda: pd.pd_gated_forward(x, w.t(), w.t(), h),
                lambda: pd.pd_gated_forward(x, w.to(BF16), w, h), lambda: pd.pd_gated_forward(x, w, w, h[:, :8]),
                lambda: pd.pd_gated_forward(x, w, w.t().contiguous().t(), h), lambda: pd.pd_gated_forward(x.half(), w, w, h),
                lambda: pd.pd_gated_forward(x, w, w, h[:1].expand(4, 16)), lambda: pd.pd_gated_forward(x, w, w, h, gate=h.to(BF16)),
                lambda: pd.pd_gated_backward(h, x, w, w, h, h, dx=x, dw_gate=w),
                lambda: pd.pd_gated_backward(h, x, w, w, h, h, dw_gate=torch.zeros((16, 8), device="cuda").t(), dw_up=w)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(pd.PdError):
        pd.pd_gated_forward(x, w, w, h, activation=5)
    none = torch.empty(0, device="cuda", dtype=torch.uint8)
    pd.pd_gated_forward(x, w, w, h, scratch=none)            # (few rows need none)
    big = torch.zeros((1000, 8), device="cuda")
    for bad in (lambda: pd.pd_gated_forward(big, w, w, torch.zeros((1000, 16), device="cuda"), scratch=none),
                lambda: pd.pd_gated_backward(h, x, w, w, h, h, dx=x, scratch=none)):
        with pytest.raises(pd.PdError):
            bad()


# ------------------------------------------------------------------ streams and graphs
def _block(x, res, w, mod, table, pos, step, stream=None):
    """A latent block's run of calls, from buffers made beforehand."""
    B, n, H, D = x.shape
    width, F = H * D, w[0].shape[1]
    rows = lambda t: t.view(B * n, -1)      # noqa: E731
    s, y, rq, out, h, back = (torch.empty_like(x) for _ in range(6))
    g, u, f, df = (torch.empty((B * n, F), device="cuda", dtype=x.dtype) for _ in range(4))
    mean, rstd = (torch.empty(B * n, device="cuda") for _ in range(2))
    dw = [torch.empty_like(t) for t in w]
    dmod = [torch.empty((B, width), device="cuda") for _ in range(2)]
    dx = torch.empty_like(x)

    def go(stream=stream):
        kw = dict(stream=stream)
        pd.pd_dropout_apply(rows(x), rows(h), 0.2, 5, rng_stream=1, step_more=step, residual=rows(res), **kw)
        pd.pd_layernorm_forward(rows(h), rows(y), weight=mod[0], bias=mod[1], sum_out=rows(s), mean=mean, rstd=rstd, **kw)
        pd.pd_rotary_axes_apply(y, None, pos, table, [D // 4, D // 4], rq, **kw)
        pd.pd_attention_forward(rq, rq, y, out, causal=False, **kw)
        pd.pd_gated_forward(rows(out), *w, f, gate=g, up=u, **kw)
        pd.pd_gated_backward(f, rows(out), *w, g, u, dx=rows(back), dw_gate=dw[0], dw_up=dw[1], **kw)
        pd.pd_layernorm_backward(rows(back), rows(s), mean, rstd, rows(dx), weight=mod[0], dweight=dmod[0], dbias=dmod[1], **kw)
    return go, [h, s, y, rq, out, g, u, f, back, *dw, dx, *dmod]


@pytest.mark.parametrize("n,dtype", [(50, BF16), (50, F32), (1, BF16), (200, BF16)])
def test_block_on_another_stream_and_in_graphs(n, dtype):
    """The calls together: on a side stream, and two graphs of them (with scratch of their own) replayed in turn, each
    replay against the eager run; the mask changes with the step on the device."""
    D = 32
    x, res = _rand((2, n, 4, D), dtype, 130), _rand((2, n, 4, D), dtype, 131)
    w = [_rand((4 * D, 264), dtype, 132 + i, 0.1) for i in range(2)]
    mod = [_rand((2, 4 * D), F32, 134 + i) for i in range(2)]
    table = torch.empty((n + 1, D // 2, 2), device="cuda")
    pd.pd_rotary_axes_table(table, [D // 4, D // 4])
    pos = torch.stack([torch.arange(n, device="cuda"), torch.arange(n, device="cuda") // 3], 1).int()
    step = torch.zeros(1, device="cuda", dtype=torch.int32)
    go, outs = _block(x, res, w, mod, table, pos, step)
    go()
    want = [t.clone() for t in outs]
    side = torch.cuda.Stream()
    for t in outs:
        t.zero_()
    side.wait_stream(torch.cuda.current_stream())
    go(side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for graph in graphs:
        with torch.cuda.graph(graph):
            go()
    seen = []
    for i in range(4):
        x.copy_(_rand(x.shape, dtype, 140 + i))
        step += 1
        go()
        want = [t.clone() for t in outs]
        for t in outs:
            t.zero_()
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want)), i
        seen.append((outs[0] == res).flatten())
    assert not torch.equal(seen[0], seen[1])


# ------------------------------------------------------------------ a few rows of any alignment
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("layout", [pd.PD_WEIGHTS_IN_OUT, pd.PD_WEIGHTS_OUT_IN])
@pytest.mark.parametrize("M,D,F", [(1, 8, 8), (2, 9, 15), (33, 8, 687), (5, 133, 41), (64, 7, 40), (64, 300, 17), (65, 264, 520), (31, 1001, 303),
                                   (128, 67, 1031), (100, 129, 1100), (3, 45, 4201), (17, 72, 4136), (129, 40, 72), (40, 8, 8)])
def test_gated_few_rows_of_any_alignment(M, D, F, layout, dtype):
    """The ends of rows inside a unit of 16 bytes, blocks of 32 and of 16 columns, several blocks of rows."""
    print(f"gated few {M} x {D} x {F} {layout} {dtype}", flush=True)
    for pad in (0, 5):
        x, _ = _wide(M, D, dtype, 160, 0, pad)
        wg, wu = _weights(D, F, dtype, 161, layout, pad)
        h, g, u = _forward(x, wg, wu, "silu", dtype)
        rh, rg, ru = ob.gated(_np(x), _np(wg), _np(wu), "silu")
        for got, ref in ((h, rh), (g, rg), (u, ru)):
            _close(got, ref, TOL[dtype])


# ------------------------------------------------------------------ offsets past 32 bits
def test_offsets_past_32_bits():
    """Tensors of more than 2^31 values, of which the last rows hold numbers."""
    rows, width = (1 << 21) + 40, 1032
    x = torch.zeros((rows, width), device="cuda", dtype=BF16)
    y = torch.empty_like(x)
    x[-3:] = _rand((3, width), BF16, 150)
    w = _rand((2, width), F32, 151)
    pd.pd_layernorm_forward(x, y, weight=w, eps=1.0)
    _close(y[-3:], ob.layernorm(_np(x[-3:]), None, _np(w[1]), None, 1.0)[1], TOL[BF16])
    assert not y[:-3].any()
    mean, rstd = torch.zeros(rows, device="cuda"), torch.ones(rows, device="cuda")
    dw = torch.empty_like(w)
    pd.pd_layernorm_backward(x, x, mean, rstd, y, weight=w, dweight=dw)
    rx, rw, _ = ob.layernorm_grad(_np(x[-3:]), _np(x[-3:]), _np(w[1]), np.zeros(3), np.ones(3), None)
    _close(y[-3:], rx, TOL[BF16])
    _close(dw[1], rw, 5e-6)
    assert not dw[0].any() and not y[:-3].any()
    pd.pd_dropout_apply(x, y, 0.5, 7)
    _close(y[-3:], ob.dropout(_np(x[-3:]), None, 0.5, ob.kept(3, width, 0.5, 7, 0, 0, rows - 3)), TOL[BF16])
    del x, y
    rows, F = 270000, 8192
    x = torch.zeros((rows, 40), device="cuda", dtype=BF16)
    x[-3:] = _rand((3, 40), BF16, 152)
    wg, wu = _weights(40, F, BF16, 153, pd.PD_WEIGHTS_IN_OUT)
    h, g, u = (torch.full((rows, F), 9.0, device="cuda", dtype=BF16) for _ in range(3))
    pd.pd_gated_forward(x, wg, wu, h, gate=g, up=u)
    rh, rg, ru = ob.gated(_np(x[-3:]), _np(wg), _np(wu), "silu")
    for got, ref in ((h, rh), (g, rg), (u, ru)):
        _close(got[-3:], ref, TOL[BF16])
        assert not got[:-3].any()
    dx, dw = torch.full_like(x, 9.0), [torch.empty_like(t) for t in (wg, wu)]
    pd.pd_gated_backward(h, x, wg, wu, g, u, dx=dx, dw_gate=dw[0], dw_up=dw[1])
    rx, rg, ru, _ = ob.gated_grad(*(_np(t) for t in (h[-3:], x[-3:], wg, wu, g[-3:], u[-3:])), "silu")
    _close(dx[-3:], rx, TOL_GRAD[BF16])
    assert not dx[:-3].any()
    _close(dw[0], rg, TOL_GRAD[BF16])
    _close(dw[1], ru, TOL_GRAD[BF16])
