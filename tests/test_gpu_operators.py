"""The transformer operators on the GPU against the oracle in float64.

Tolerances (relative L2 of a whole tensor, and `PEAK` times that for one element
against the largest of its value, the tensor's root mean square and its vector's: a
vector of the last dimension is a sum of vectors, whose roundings go by their size):
  float32   2^-24 for each of the products' terms and for the scores, whose error the
            exponential multiplies by |score| <= about 10: under 1e-6 each; 5e-6.
  bfloat16  a rounding is 2^-9 at most and 1.1e-3 in the root mean square; forward the
            probabilities and the result (1.6e-3): 4e-3; backward the forward's result,
            probabilities, scores' gradients and the result (2.2e-3): 8e-3.
"""
import numpy as np
import pytest
import torch

import paper_2305_16317_amd as pd
from oracle import transformer as ot

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
TOL = {F32: 5e-6, BF16: 4e-3}
TOL_GRAD = {F32: 5e-6, BF16: 8e-3}
PEAK = 12


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    pd.load()


def _np(t):
    return t.detach().double().cpu().numpy()


def _close(got, ref, tol, what=""):
    got = _np(got) if isinstance(got, torch.Tensor) else got
    assert got.shape == ref.shape
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


# ------------------------------------------------------------------ norm
NORM_SIZES = [(1, 1), (3, 7), (5, 8), (4, 64), (9, 511), (17, 512), (6, 513), (33, 1024), (7, 1001), (5, 2048), (3, 2049),
              (2, 4104), (3, 8192), (2, 8193), (2, 20000), (1, 65536), (700, 320)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,width", NORM_SIZES)
def test_norm_forward(rows, width, dtype):
    print(f"norm {rows} x {width} {dtype}", flush=True)
    x, r = _rand((rows, width), dtype, 1), _rand((rows, width), dtype, 2, 3.0)
    w = _rand((width,), F32, 3)
    y, h, rstd = torch.full_like(x, 7), torch.full_like(x, 7), torch.full((rows,), 7.0, device="cuda")
    pd.pd_rmsnorm_forward(x, w, y, residual=r, sum_out=h, rstd=rstd, eps=1e-5)
    s, yr, rr = ot.rmsnorm(_np(x), _np(r), _np(w), 1e-5)
    _close(h, s, TOL[dtype])
    _close(y, yr, TOL[dtype])
    _close(rstd, rr, 2e-6)
    pd.pd_rmsnorm_forward(x, w, y, eps=1e-5)                # without a residual
    _close(y, ot.rmsnorm(_np(x), None, _np(w), 1e-5)[1], TOL[dtype])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,width,group", [(1, 1, 0), (5, 100, 0), (4, 100, 16), (9, 1024, 128), (3, 1000, 64), (2, 4100, 512),
                                              (3, 9000, 0), (2, 9000, 256), (64, 320, 32)])
def test_norm_eight_bits(rows, width, group, dtype):
    print(f"norm f8 {rows} x {width} / {group} {dtype}", flush=True)
    x, w = _rand((rows, width), dtype, 4), _rand((width,), F32, 5)
    per = -(-width // group) if group else 1
    y = torch.empty((rows, width), device="cuda", dtype=torch.float8_e4m3fn)
    scale = torch.full((rows, per), 7.0, device="cuda")
    pd.pd_rmsnorm_forward(x, w, y, scale=scale, group=group)
    q, sc = ot.quantise(ot.rmsnorm(_np(x), None, _np(w), 1e-6)[1], group)
    _close(scale, sc, 2e-6)
    # each value is one of the format's nearest to q, up to float32's error of q itself
    v = ot.e4m3_values()
    grid = np.concatenate([-v[:0:-1], v])
    at = np.clip(np.searchsorted(grid, q), 1, grid.size - 1)
    nearest = np.minimum(np.abs(grid[at] - q), np.abs(grid[at - 1] - q))
    assert np.all(np.abs(_np(y.float()) - q) <= nearest + 4e-6 * np.abs(q) + 1e-12)


def test_norm_eight_bits_of_zeros_tiny_and_infinite_rows():
    x = torch.zeros((4, 128), device="cuda")
    x[1, 5], x[2, 9], x[3, 7] = 1e-30, float("inf"), float("nan")
    w = torch.full((128,), 1e-12, device="cuda")
    y = torch.empty((4, 128), device="cuda", dtype=torch.float8_e4m3fn)
    scale = torch.empty((4, 2), device="cuda")
    pd.pd_rmsnorm_forward(x, w, y, scale=scale, group=64, eps=1.0)
    s, q = _np(scale), _np(y.float())
    assert np.all(s[0] == 0) and np.all(s[1] == 0) and np.all(q[:2] == 0)
    assert not np.isfinite(s[2, 0]) and not np.isfinite(s[3]).all()
    for i in (2, 3):
        assert not np.isfinite(q[i, :64] * s[i, 0]).any()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,width", NORM_SIZES[1:] + [(3000, 96)])     # (one value: a difference of equal numbers)
def test_norm_backward(rows, width, dtype):
    print(f"norm backward {rows} x {width} {dtype}", flush=True)
    dy, h, ds = _rand((rows, width), dtype, 6), _rand((rows, width), dtype, 7, 2.0), _rand((rows, width), dtype, 8)
    w = _rand((width,), F32, 9)
    rstd = torch.rsqrt(h.float().square().mean(1) + 1e-6)
    dx, dw = torch.full_like(dy, 7), torch.full((width,), 7.0, device="cuda")
    pd.pd_rmsnorm_backward(dy, h, w, rstd, dx, dw, dsum=ds)
    rx, rw = ot.rmsnorm_grad(_np(dy), _np(h), _np(w), _np(rstd), _np(ds))
    _close(dx, rx, TOL[dtype])
    _close(dw, rw, 5e-6)
    again = torch.empty_like(dw)
    pd.pd_rmsnorm_backward(dy, h, w, rstd, dx, again)       # without the other gradient; the same bits again
    _close(dx, ot.rmsnorm_grad(_np(dy), _np(h), _np(w), _np(rstd), None)[0], TOL[dtype])
    assert torch.equal(again, dw)
    pd.pd_rmsnorm_backward(dy, h, w, rstd, dx)              # without the weight's
    _close(dx, ot.rmsnorm_grad(_np(dy), _np(h), _np(w), _np(rstd), None)[0], TOL[dtype])


def test_norm_backward_of_no_rows_and_against_differences():
    z, w = torch.empty((0, 40), device="cuda"), torch.ones(40, device="cuda")
    dw = torch.full((40,), 7.0, device="cuda")
    pd.pd_rmsnorm_backward(z, z, w, torch.empty(0, device="cuda"), torch.empty_like(z), dw)
    assert torch.all(dw == 0)
    x, dy, w, d = (_rand(s, F32, 10 + i) for i, s in enumerate([(4, 50), (4, 50), (50,), (4, 50)]))
    y, h, rstd, dx = torch.empty_like(x), torch.empty_like(x), torch.empty(4, device="cuda"), torch.empty_like(x)
    pd.pd_rmsnorm_forward(x, w, y, sum_out=h, rstd=rstd)
    pd.pd_rmsnorm_backward(dy, h, w, rstd, dx)
    loss = lambda e: float(np.sum(ot.rmsnorm(_np(x) + e * _np(d), None, _np(w), 1e-6)[1] * _np(dy)))  # noqa: E731
    want = (loss(1e-5) - loss(-1e-5)) / 2e-5
    assert abs(float((dx.double() * d.double()).sum()) - want) <= 1e-5 * float(dx.norm() * d.norm())


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_norm_strides_and_in_place(dtype):
    wide, w = _rand((6, 50), dtype, 20), _rand((33,), F32, 21)
    res = _rand((6, 47), dtype, 22)[:, 5:38]
    x = wide[:, 3:36]                                       # rows that start at no multiple of 16 bytes
    before = wide.clone()
    s, y, _ = ot.rmsnorm(_np(x), _np(res), _np(w), 1e-6)
    keep = res.clone()
    pd.pd_rmsnorm_forward(x, w, x, residual=res, sum_out=res)   # y over x, sum over residual
    _close(x, y, TOL[dtype])
    _close(res, s, TOL[dtype])
    assert torch.equal(wide[:, :3], before[:, :3]) and torch.equal(wide[:, 36:], before[:, 36:])
    dy, rstd = _rand((2, 3, 33), dtype, 23), torch.rsqrt(keep.float().square().mean(1) + 1e-6)
    rx, _ = ot.rmsnorm_grad(_np(dy).reshape(6, 33), _np(keep), _np(w), _np(rstd), None)
    pd.pd_rmsnorm_backward(dy, keep.view(2, 3, 33), w, rstd, dy)
    _close(dy.view(6, 33), rx, TOL[dtype])


def test_norm_of_more_rows_than_a_launch_holds():
    rows = (1 << 21) + 3
    x, w = _rand((rows, 8), BF16, 25), _rand((8,), F32, 26)
    y = torch.empty((rows, 8), device="cuda", dtype=torch.float8_e4m3fn)
    scale, rstd, h = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), torch.empty_like(x)
    pd.pd_rmsnorm_forward(x, w, y, residual=x, sum_out=h, scale=scale, rstd=rstd)
    for part in (slice(0, 5), slice(rows - 5, rows)):
        s, yr, rr = ot.rmsnorm(_np(x[part]), _np(x[part]), _np(w), 1e-6)
        _close(h[part], s, TOL[BF16])
        _close(rstd[part], rr, 2e-6)
        _close(scale[part, None], ot.quantise(yr, 0)[1], 2e-6)


def test_norm_refuses_what_it_cannot_read():
    x, w = torch.zeros((4, 8), device="cuda"), torch.ones(8, device="cuda")
    for bad in (lambda: pd.pd_rmsnorm_forward(x.t(), torch.ones(4, device="cuda"), torch.empty((8, 4), device="cuda")),
                lambda: pd.pd_rmsnorm_forward(x, w[:7], torch.empty_like(x)),
                lambda: pd.pd_rmsnorm_forward(x, w, torch.empty((4, 8), device="cuda", dtype=BF16)),
                lambda: pd.pd_rmsnorm_forward(x, w, w.expand(4, 8)),
                lambda: pd.pd_rmsnorm_forward(x, w, torch.empty((4, 8), device="cuda", dtype=torch.float8_e4m3fn)),
                lambda: pd.pd_rmsnorm_forward(x, w, torch.empty_like(x), rstd=torch.empty(3, device="cuda")),
                lambda: pd.pd_rmsnorm_backward(x, x, w, torch.empty(4, device="cuda"), torch.empty_like(x),
                                               torch.empty(8, device="cuda", dtype=BF16))):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(pd.PdError):
        pd.pd_rmsnorm_backward(x, x, w, torch.empty(4, device="cuda"), torch.empty_like(x), torch.empty(8, device="cuda"),
                               scratch=torch.empty(4, device="cuda", dtype=torch.uint8))


# ------------------------------------------------------------------ rotary
SCALINGS = [("plain", pd.PD_ROTARY_PLAIN), ("linear", pd.PD_ROTARY_LINEAR), ("base", pd.PD_ROTARY_BASE),
            ("by_parts", pd.PD_ROTARY_BY_PARTS)]


@pytest.mark.parametrize("name,kind", SCALINGS)
@pytest.mark.parametrize("R,first,rows", [(2, 0, 5), (6, 3, 7), (64, 1000, 33), (128, 1 << 20, 9)])
def test_rotary_table(name, kind, R, first, rows):
    t = torch.empty((rows, R // 2, 2), device="cuda")
    pd.pd_rotary_table(t, base=5e5, scaling=kind, factor=4.0, original_length=2048.0, turns_low=1.0, turns_high=16.0,
                       magnitude=1.1, first=first)
    f = ot.rotary_freqs(R, 5e5, name, 4.0, 2048.0, 1.0, 16.0)
    ref = ot.rotary_table(f, range(first, first + rows), 1.1)
    # a double's angle of up to 1e6 is off by 1e-10, a float of 1.1 by 6.6e-8
    assert np.max(np.abs(_np(t) - ref)) <= 1e-7


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("B,n,H,K,D,R", [(1, 1, 1, 1, 2, 2), (2, 5, 3, 1, 20, 6), (1, 16, 16, 16, 64, 64), (3, 33, 8, 2, 80, 48),
                                         (2, 70, 7, 1, 33, 18), (1, 300, 32, 8, 128, 96), (2, 9, 2, 2, 300, 300)])
def test_rotary(B, n, H, K, D, R, interleaved, backward, dtype):
    print(f"rotary {B, n, H, K, D, R, interleaved, backward, dtype}", flush=True)
    q, k = _rand((B, n, H, D), dtype, 1), _rand((B, n, K, D), dtype, 2)
    table = torch.empty((400, R // 2, 2), device="cuda")
    pd.pd_rotary_table(table, base=1e4)
    pos = torch.randint(-3, 410, (B, n), device="cuda", dtype=torch.int32)      # some outside the table: clamped
    qo, ko = torch.full_like(q, 7), torch.full_like(k, 7)
    lay = pd.PD_ROTARY_INTERLEAVED if interleaved else pd.PD_ROTARY_HALF
    pd.pd_rotary_apply(q, k, pos, table, qo, ko, layout=lay, backward=backward)
    t, p = _np(table), pos.cpu().numpy()
    _close(qo, ot.rotary(_np(q), t, p, interleaved, backward), TOL[dtype])
    _close(ko, ot.rotary(_np(k), t, p, interleaved, backward), TOL[dtype])
    assert torch.equal(qo[..., R:], q[..., R:])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rotary_in_place_in_a_fused_buffer_and_into_a_cache(interleaved, dtype):
    B, n, H, K, D = 2, 11, 4, 2, 40
    buf = _rand((B, n, (H + 2 * K) * D + 3), dtype, 3)
    qkv = buf[:, :, 3:].unflatten(2, (H + 2 * K, D))          # starts at no multiple of 16 bytes
    q, k, v = qkv[:, :, :H], qkv[:, :, H:H + K], qkv[:, :, H + K:].clone()
    table = torch.empty((64, 8, 2), device="cuda")
    pd.pd_rotary_table(table)
    pos = torch.arange(20, 20 + n, device="cuda", dtype=torch.int32)
    lay = pd.PD_ROTARY_INTERLEAVED if interleaved else pd.PD_ROTARY_HALF
    p = pos.cpu().numpy()[None].repeat(B, 0)
    rq, rk = (ot.rotary(_np(x), _np(table), p, interleaved) for x in (q, k))
    cache = torch.full((B, K, 50, D), 7.0, device="cuda", dtype=dtype)
    pd.pd_rotary_apply(q, k, pos, table, q, cache[:, :, 20:20 + n].transpose(1, 2), layout=lay)
    _close(q, rq, TOL[dtype])
    _close(cache[:, :, 20:20 + n].transpose(1, 2), rk, TOL[dtype])
    assert torch.all(cache[:, :, :20] == 7) and torch.all(cache[:, :, 20 + n:] == 7)
    assert torch.equal(qkv[:, :, H + K:], v)
    pd.pd_rotary_apply(k, None, pos, table, k, layout=lay)    # k alone, in place
    _close(k, rk, TOL[dtype])


def test_rotary_refuses_what_it_cannot_read():
    q, t = torch.zeros((1, 4, 2, 8), device="cuda"), torch.zeros((4, 4, 2), device="cuda")
    pos = torch.zeros(4, device="cuda", dtype=torch.int32)
    for bad in (lambda: pd.pd_rotary_apply(q, q, pos.long(), t, q, q), lambda: pd.pd_rotary_apply(q, q, pos[:3], t, q, q),
                lambda: pd.pd_rotary_apply(q, q, pos, t, q), lambda: pd.pd_rotary_apply(q, None, pos, t[:, :, 0], q),
                lambda: pd.pd_rotary_apply(q, None, pos, t, q[:, :1].expand(1, 4, 2, 8)),
                lambda: pd.pd_rotary_apply(q.to(BF16), None, pos, t, q)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(pd.PdError):
        pd.pd_rotary_apply(q, None, pos, torch.zeros((4, 5, 2), device="cuda"), torch.empty_like(q))


# ------------------------------------------------------------------ attention
def _att_inputs(B, n, m, H, K, D, dtype, seed=0, layout="token"):
    def make(L, h, s):
        if layout == "head":                                  # [batch, head, token, dim]
            return _rand((B, h, L, D), dtype, s, 1.25).transpose(1, 2)
        if layout == "odd":                                   # rows that start at no multiple of 16 bytes
            return _rand((B, L, h * D + 3), dtype, s, 1.25)[:, :, 1:1 + h * D].unflatten(2, (h, D))
        return _rand((B, L, h, D), dtype, s, 1.25)
    return make(n, H, seed + 1), make(m, K, seed + 2), make(m, K, seed + 3), make(n, H, seed + 4)


def _lens(v):
    return None if v is None else torch.tensor(v, device="cuda", dtype=torch.int32)


def _forward(q, k, v, causal, window, sinks, q_lens, kv_lens, scale, tol, what=""):
    print("attention", tuple(q.shape), tuple(k.shape), q.dtype, causal, window, sinks, q_lens, kv_lens, what, flush=True)
    out = torch.full(q.shape, 7.0, device="cuda", dtype=q.dtype)
    lse = torch.full((q.shape[0], q.shape[2], q.shape[1]), 7.0, device="cuda")
    pd.pd_attention_forward(q, k, v, out, lse=lse, causal=causal, window=window, sinks=sinks, scale=scale,
                            q_lens=_lens(q_lens), kv_lens=_lens(kv_lens))
    ro, rl = ot.attention(_np(q), _np(k), _np(v), q.shape[3] ** -0.5 if scale is None else scale, causal, window, sinks,
                          q_lens, kv_lens)
    _close(out, ro, tol, "out")
    _close(lse, rl, 5e-6, "lse")
    return out, lse


#            B   n    m    H  K  D    causal window sinks q_lens kv_lens
ATTENTION = [
    (1, 1, 1, 1, 1, 1, True, 0, 0, None, None),
    (1, 1, 7, 2, 1, 8, True, 0, 0, None, None),
    (2, 16, 16, 4, 4, 64, False, 0, 0, None, None),
    (2, 31, 33, 3, 1, 32, True, 0, 0, None, None),
    (1, 65, 65, 2, 2, 33, True, 0, 0, None, None),
    (1, 129, 129, 2, 1, 128, True, 40, 3, None, None),
    (1, 100, 260, 4, 2, 80, True, 64, 70, None, None),
    (2, 70, 70, 2, 2, 96, False, 9, 5, None, None),
    (1, 150, 150, 1, 1, 64, False, 1, 0, None, None),
    (1, 40, 40, 7, 1, 20, True, 1, 1, None, None),
    (3, 33, 90, 2, 1, 72, True, 16, 2, None, [90, 40, 10]),       # a sequence shorter than its queries: empty rows
    (4, 5, 64, 8, 2, 64, True, 0, 0, [5, 0, 3, 1], [64, 64, 0, 1]),
    (2, 20, 50, 2, 2, 100, False, 4, 0, [20, 30], [-3, 400]),     # lengths out of range are clamped
    (2, 30, 12, 2, 1, 48, False, 0, 0, None, [12, 5]),            # more queries than keys, two-sided
    (2, 30, 12, 2, 1, 48, True, 5, 2, None, None),
    (2, 30, 12, 2, 1, 48, False, 6, 2, None, None),
    (1, 1, 700, 8, 1, 128, True, 300, 4, None, None),             # a single token
    (3, 1, 513, 4, 4, 64, True, 0, 0, None, [513, 100, 0]),
    (2, 1, 1000, 32, 4, 80, True, 128, 16, None, [1000, 7]),
    (1, 3, 900, 14, 2, 128, True, 200, 130, None, None),
    (1, 4, 600, 4, 2, 64, False, 50, 10, None, None),
    (1, 300, 300, 2, 1, 64, True, 100000, 4, None, None),         # a window longer than the sequence
    (1, 64, 128, 2, 1, 64, True, 2**31 - 1, 2**31 - 1, None, None),
    (1, 64, 128, 2, 1, 64, True, 8, 2**31 - 1, None, None),
    (1, 6, 0, 2, 1, 64, True, 0, 0, None, None),                  # no keys at all
    (9, 2, 260, 16, 2, 64, True, 0, 0, None, [260, 200, 129, 128, 127, 65, 64, 2, 1]),
]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("case", ATTENTION)
def test_attention_forward(case, dtype):
    B, n, m, H, K, D, causal, window, sinks, ql, kl = case
    q, k, v, _ = _att_inputs(B, n, m, H, K, D, dtype)
    _forward(q, k, v, causal, window, sinks, ql, kl, None, TOL[dtype])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("layout", ["head", "odd"])
@pytest.mark.parametrize("n,m,D", [(70, 70, 64), (1, 300, 128), (50, 130, 36), (5, 200, 80)])
def test_attention_layouts(n, m, D, layout, dtype):
    q, k, v, _ = _att_inputs(2, n, m, 4, 2, D, dtype, 5, layout)
    _forward(q, k, v, True, 60, 4, None, None, None, TOL[dtype], layout)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_attention_strides_over_single_elements(dtype):
    """One sequence, one key head: their strides may be anything (here odd)."""
    q, k, v, g = _att_inputs(1, 40, 90, 4, 1, 64, dtype, 6)
    k, v = (x.contiguous().as_strided(x.shape, (13, 64, 7, 1)) for x in (k, v))
    _forward(q, k, v, True, 30, 2, None, None, None, TOL[dtype])
    _backward(q, k, v, g, True, 30, 2, None, None, None, TOL_GRAD[dtype])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("scale", [-0.3, 0.0, 2.0])
@pytest.mark.parametrize("n,m", [(40, 90), (1, 200)])
def test_attention_scales(n, m, scale, dtype):
    q, k, v, _ = _att_inputs(1, n, m, 2, 1, 64, dtype, 7)
    # scores of up to about 100: their float32 error is 100 2^-23 and so is the probabilities'
    _forward(q, k, v, True, 0, 0, None, None, scale, max(TOL[dtype], 4e-5), scale)


def test_attention_long_two_sided_and_windowed():
    q, k, v, _ = _att_inputs(1, 700, 700, 2, 1, 64, BF16, 9)
    _forward(q, k, v, False, 0, 0, None, None, None, TOL[BF16])
    _forward(q, k, v, True, 129, 33, None, None, None, TOL[BF16])
    q, k, v, _ = _att_inputs(1, 2, 5000, 4, 2, 64, F32, 9)
    _forward(q, k, v, True, 0, 0, None, None, None, TOL[F32])
    _forward(q, k, v, True, 3000, 100, None, [4900], None, TOL[F32])


#                     B   n    m    H   K  D  causal window sinks ragged layout
MANY_BLOCKS = [
    (64, 257, 257, 8, 8, 64, False, 0, 0, False, "token"),        # 1024 tiles of 256 rows, the second with one row
    (64, 257, 300, 8, 8, 64, True, 40, 3, True, "token"),
    (32, 150, 150, 16, 8, 64, True, 0, 0, True, "head"),          # two query heads to a key head: 300 rows
    (64, 257, 257, 8, 8, 36, False, 30, 5, True, "odd"),          # through the registers
    (64, 513, 513, 4, 4, 24, True, 100, 70, False, "token"),
    (171, 200, 90, 3, 3, 50, True, 0, 0, False, "odd"),           # rows before the first key
]


@pytest.mark.parametrize("case", MANY_BLOCKS)
def test_attention_of_many_blocks(case):
    """From 512 tiles of 256 rows on, heads of up to 64 bfloat16 values go two tiles of 32 rows a wave.  The first,
    two middle and the last sequences are compared, of the others that the rows past their queries are 0."""
    B, n, m, H, K, D, causal, window, sinks, ragged, layout = case
    print("many blocks", case, flush=True)
    assert -(-n * (H // K) // 256) * K * B >= 512 and D <= 64
    q, k, v, _ = _att_inputs(B, n, m, H, K, D, BF16, 41, layout)
    ql, kl = ([n - 5 * b % n for b in range(B)], [(m * (B - b)) // B for b in range(B)]) if ragged else ([n] * B, [m] * B)
    out, lse = torch.full(q.shape, 7.0, device="cuda", dtype=BF16), torch.full((B, H, n), 7.0, device="cuda")
    pd.pd_attention_forward(q, k, v, out, lse=lse, causal=causal, window=window, sinks=sinks, q_lens=_lens(ql), kv_lens=_lens(kl))
    for b in (0, B // 2, B // 2 + 1, B - 1):
        one = slice(b, b + 1)
        ro, rl = ot.attention(_np(q[one]), _np(k[one]), _np(v[one]), D ** -0.5, causal, window, sinks, ql[one], kl[one])
        _close(out[one], ro, TOL[BF16], ("out", b))
        _close(lse[one], rl, 5e-6, ("lse", b))
    for b in range(B):
        assert torch.all(out[b, ql[b]:] == 0) and torch.all(lse[b, :, ql[b]:] == -float("inf")), b


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("layout", ["head", "odd"])
@pytest.mark.parametrize("B,n,H,K,D,window,sinks,lens", [
    (3, 1, 8, 2, 128, 0, 0, [5000, 37, 0]), (3, 1, 8, 2, 64, 0, 0, [4999, 1, 2500]), (2, 1, 8, 8, 64, 3000, 100, [5000, 4200]),
    (2, 1, 32, 4, 128, 2100, 7, [5000, 3000]), (1, 4, 16, 2, 80, 0, 0, [5000]), (2, 2, 6, 3, 40, 4000, 40, [5000, 4001])])
def test_attention_of_few_rows_over_long_caches(B, n, H, K, D, window, sinks, lens, layout, dtype):
    """A cache in parts, whose results are joined: parts that a window leaves without keys, sequences shorter than a part."""
    q, k, v, _ = _att_inputs(B, n, 5000, H, K, D, dtype, 43, layout)
    _forward(q, k, v, True, window, sinks, None, lens, None, TOL[dtype], layout)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("n,m", [(96, 200), (1, 200), (3, 400)])
def test_attention_out_of_sight_values_do_not_reach_a_row(n, m, bad, dtype):
    """Keys past a sequence's length, keys that left the window, and, for the rows before it, a key to come."""
    q, k, v, _ = _att_inputs(2, n, m, 4, 2, 64, dtype, 11)
    for x in (k, v):
        x[0, m - 30:] = bad                                  # past the length of sequence 0
        x[1, 5:20] = bad                                     # behind the window, after the sinks
        if n > 1:
            x[1, m - 2] = bad                                # seen by the last two rows alone
    out, lse = (torch.empty(s, device="cuda", dtype=d) for s, d in ((q.shape, dtype), ((2, 4, n), F32)))
    lens = [m - 30, m]
    pd.pd_attention_forward(q, k, v, out, lse=lse, window=70, sinks=5, kv_lens=_lens(lens))
    with np.errstate(invalid="ignore", over="ignore"):
        ro, rl = ot.attention(_np(q), _np(k), _np(v), 0.125, True, 70, 5, None, lens)
    got, gl = _np(out), _np(lse)
    sees = np.array([[np.isfinite(_np(k[b, ot.visible(i, n, lens[b], True, 70, 5)])).all() for i in range(n)] for b in range(2)])
    assert sees.sum() >= 2 * n - 75
    _close(got[sees], ro[sees], TOL[dtype])
    _close(gl.transpose(0, 2, 1)[sees], rl.transpose(0, 2, 1)[sees], 5e-6)
    assert not np.isfinite(got[~sees]).any()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_attention_values_of_the_types_ends(dtype):
    """Scores near the ends of float32, and a value that is infinite for those who see it."""
    q, k, v, _ = _att_inputs(1, 40, 40, 1, 1, 64, dtype, 13)
    k[0, 3] = -1e30
    k[0, 4] = 1e30
    q[0, :, 0] = q[0, :, 0].abs()
    out = torch.empty_like(q)
    pd.pd_attention_forward(q, k, v, out, causal=True)
    ro, _ = ot.attention(_np(q), _np(k), _np(v), 0.125, True)
    _close(out, ro, TOL[dtype])                              # each row takes the one key with the largest score
    q, k, v, _ = _att_inputs(1, 40, 40, 1, 1, 64, dtype, 14)
    v[0, 7, 0, 5] = float("inf")
    pd.pd_attention_forward(q, k, v, out, causal=True)
    ro, _ = ot.attention(_np(q), _np(k), _np(v), 0.125, True)
    _close(out, ro, TOL[dtype])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,m", [(1, 50), (1, 700), (3, 40), (40, 70), (70, 600)])
def test_attention_of_scores_that_are_all_minus_infinity(n, m, dtype):
    """Keys of -inf under queries above 0 weigh nothing, alone as beside others: then there is no sum, as
    for a row that sees nothing, whatever the type and the way the rows go."""
    q, k, v, _ = _att_inputs(1, n, m, 2, 1, 64, dtype, 33)
    q = q.abs() + 0.1
    k.fill_(-float("inf"))
    out, lse = torch.full_like(q, 7), torch.full((1, 2, n), 7.0, device="cuda")
    pd.pd_attention_forward(q, k, v, out, lse=lse, causal=False)
    assert torch.all(out == 0) and torch.all(lse == -float("inf"))
    k[0, m // 2] = 0.5                                       # one key with a score: its value alone
    pd.pd_attention_forward(q, k, v, out, lse=lse, causal=False)
    _close(out, np.broadcast_to(_np(v[0, m // 2]), out.shape), TOL[dtype])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("scale", [0.0, 1e-39, -1e-30, 1e-10])
def test_attention_backward_of_scales_near_zero(scale, dtype):
    """All keys weigh the same, so dv is a mean; dq and dk go with the scale."""
    q, k, v, g = _att_inputs(1, 40, 60, 4, 2, 64, dtype, 29)
    out, lse = torch.empty_like(q), torch.empty((1, 4, 40), device="cuda")
    pd.pd_attention_forward(q, k, v, out, lse=lse, causal=False, scale=scale)
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    pd.pd_attention_backward(q, k, v, out, lse, g, dq, dk, dv, causal=False, scale=scale)
    refs = ot.attention_grad(_np(q), _np(k), _np(v), _np(g), scale, False)
    _close(dv, refs[2], TOL_GRAD[dtype])
    if abs(scale) > 1e-35:
        _close(dq, refs[0], TOL_GRAD[dtype])
        _close(dk, refs[1], TOL_GRAD[dtype])
    else:                                      # (gradients below the normal numbers)
        assert float(dq.abs().max()) <= 1e-36 and float(dk.abs().max()) <= 1e-36


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n,m", [(40, 40), (1, 40)])
def test_attention_backward_of_scores_near_the_types_end(n, m, dtype):
    """One key takes each row whole (as in the test above): dv is the sum of its rows' dout."""
    q, k, v, g = _att_inputs(1, n, m, 1, 1, 64, dtype, 13)
    k[0, 3], k[0, 4] = -1e30, 1e30
    out, lse = torch.empty_like(q), torch.empty((1, 1, n), device="cuda")
    pd.pd_attention_forward(q, k, v, out, lse=lse)
    _close(lse, ot.attention(_np(q), _np(k), _np(v), 0.125, True)[1], 5e-6)
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    pd.pd_attention_backward(q, k, v, out, lse, g, dq, dk, dv)
    _close(dv, ot.attention_grad(_np(q), _np(k), _np(v), _np(g), 0.125, True)[2], TOL_GRAD[dtype])


def _grad_bounds(q, k, v, g, out, scale, causal, u, window=0, sinks=0, q_lens=None, kv_lens=None):
    """What roundings can add to dq, dk and dv when each of a pair's terms (p, dout v, dout out and their
    product) is off by u of the sizes that it is summed from."""
    q, k, v, g, out = (np.abs(_np(x)) if x is not q and x is not k else _np(x) for x in (q, k, v, g, out))
    dq, dk, dv = np.zeros(q.shape), np.zeros(k.shape), np.zeros(v.shape)
    for b, i, h, e, j in ot._each(q, k, q_lens, kv_lens, causal, window, sinks):
        x = scale * (k[b, j, e] @ q[b, i, h])
        p = np.exp(x - np.max(x))
        p /= p.sum()
        ds = u * p * (v[b, j, e] @ g[b, i, h] + out[b, i, h] @ g[b, i, h])
        dq[b, i, h] = abs(scale) * (ds @ np.abs(k[b, j, e]))
        dk[b, j, e] += abs(scale) * ds[:, None] * np.abs(q[b, i, h])
        dv[b, j, e] += u * p[:, None] * g[b, i, h]
    return dq, dk, dv


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("size", [2.0**12, 2.0**21, -2.0**21])
@pytest.mark.parametrize("n,m,causal", [(40, 70, False), (1, 40, True), (150, 150, True)])
def test_attention_backward_of_keys_beside_the_largest(n, m, causal, size, dtype):
    """Scores of `size` less 0 to 3, whole numbers that every sum forms exactly: equal ones share a row, and
    keys that lie 1 to 3 lower keep their weight, though the row's lse is no number of float32 there.
    bfloat16: out, p or ds, and the result are rounded, 2^-9 each; float32: fewer than 512 roundings of 2^-24."""
    print("near the largest", n, m, causal, size, dtype, flush=True)
    q, k, v, g = _att_inputs(1, n, m, 2, 1, 64, dtype, 31)
    q.zero_(), k.zero_()
    q[..., 0], q[..., 1], k[..., 0] = size, 1.0, 1.0
    k[..., 1] = -(torch.arange(m, device="cuda") % 4)[None, :, None].to(dtype)
    refs = ot.attention_grad(_np(q), _np(k), _np(v), _np(g), 1.0, causal)
    kw = dict(causal=causal, scale=1.0)
    out, lse = torch.empty_like(q), torch.empty((1, 2, n), device="cuda")
    grads = [torch.empty_like(x) for x in (q, k, v)]
    pd.pd_attention_forward(q, k, v, out, lse=lse, **kw)
    pd.pd_attention_backward(q, k, v, out, lse, g, *grads, **kw)
    u = 2.0**-8 if dtype == BF16 else 2.0**-15
    bounds = [b + u * np.abs(r) for b, r in zip(_grad_bounds(q, k, v, g, out, 1.0, causal, u), refs)]

    def check(which, part=slice(None)):
        off = np.abs(_np(grads[which])[:, part] - refs[which][:, part])
        assert np.all(off <= bounds[which][:, part]), (("dq", "dk", "dv")[which], np.nanmax(off / (bounds[which][:, part] + 1e-300)))
    for which in range(3):
        check(which)
    if n != m:
        return
    # the same beside a NaN: rows that do not see the last key, keys that the first row does not see
    for x, at, which, clean in ((k, n - 1, 0, slice(0, n - 1)), (q, 0, 1, slice(1, n)), (q, 0, 2, slice(1, n))):
        kept = x[0, at].clone()
        x[0, at] = float("nan")
        pd.pd_attention_backward(q, k, v, out, lse, g, *grads, **kw)
        x[0, at] = kept
        check(which, clean)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("size", [2.0**11, 2.0**20])
@pytest.mark.parametrize("B,n,m,H,K,D,causal,window,sinks,ql,kl,layout", [
    (2, 70, 90, 6, 2, 128, True, 30, 4, None, [90, 40], "head"), (1, 130, 130, 4, 4, 96, False, 20, 3, None, None, "token"),
    (3, 33, 65, 2, 1, 20, True, 0, 0, [33, 5, 0], None, "token"), (1, 300, 300, 8, 2, 32, True, 0, 0, None, None, "token"),
    (2, 40, 200, 4, 1, 36, True, 0, 0, None, [200, 0], "odd"), (1, 1, 400, 8, 1, 128, True, 100, 7, None, None, "head")])
def test_attention_backward_of_large_scores(B, n, m, H, K, D, causal, window, sinks, ql, kl, layout, size, dtype):
    """Two rows of three have scores of `size` and a small whole number each, which every sum forms exactly; the third's
    are small.  Bounds as in the test of keys beside the largest."""
    print("large scores", B, n, m, H, K, D, causal, window, sinks, size, dtype, flush=True)
    q, k, v, g = _att_inputs(B, n, m, H, K, D, dtype, 47, layout)
    r = torch.Generator(device="cuda").manual_seed(48)
    for x in (q, k):
        x.copy_(torch.randint(-1, 2, x.shape, device="cuda", generator=r))
    q[..., 0] = (size * (torch.arange(n, device="cuda") % 3 > 0))[None, :, None].to(dtype)
    k[..., 0] = 1.0
    refs = ot.attention_grad(_np(q), _np(k), _np(v), _np(g), 1.0, causal, window, sinks, ql, kl)
    kw = dict(causal=causal, scale=1.0, window=window, sinks=sinks, q_lens=_lens(ql), kv_lens=_lens(kl))
    out, lse = torch.empty(q.shape, device="cuda", dtype=dtype), torch.empty((B, H, n), device="cuda")
    grads = [torch.full(x.shape, 7.0, device="cuda", dtype=dtype) for x in (q, k, v)]
    pd.pd_attention_forward(q, k, v, out, lse=lse, **kw)
    pd.pd_attention_backward(q, k, v, out, lse, g, *grads, **kw)
    u = 2.0**-8 if dtype == BF16 else 2.0**-15
    bounds = _grad_bounds(q, k, v, g, out, 1.0, causal, u, window, sinks, ql, kl)
    for name, got, ref, bound in zip(("dq", "dk", "dv"), grads, refs, bounds):
        off = np.abs(_np(got) - ref)
        assert np.all(off <= bound + u * np.abs(ref)), (name, np.max(off / (bound + u * np.abs(ref) + 1e-300)))


def test_attention_cache_offsets_past_32_bits():
    """A cache whose tokens lie 80 MB apart: the last of 60 is 2.4e9 elements from the first."""
    D, m, step = 64, 60, 40_000_000
    buf = torch.empty(m * step, device="cuda", dtype=BF16)
    view = buf.as_strided((1, m, 2, D), (m * step, step, D, 1))
    more = buf[4 * D:].as_strided((1, m, 2, D), (m * step - 4 * D, step, D, 1))
    q, k, v, g = _att_inputs(1, 20, m, 4, 2, D, BF16, 15)
    view.copy_(k)
    more.copy_(v)
    out, lse = _forward(q, view, more, True, 0, 0, None, None, None, TOL[BF16])
    o1, _ = _forward(q[:, :1], view, more, True, 0, 0, None, None, None, TOL[BF16])
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    pd.pd_attention_backward(q, view, more, out, lse, g, dq, dk, dv)
    for got, ref in zip((dq, dk, dv), ot.attention_grad(_np(q), _np(k), _np(v), _np(g), 0.125, True)):
        _close(got, ref, TOL_GRAD[BF16])


GRAD = [c for c in ATTENTION if c[2] > 0] + [
    (1, 200, 200, 4, 2, 64, True, 0, 0, None, None),
    (1, 257, 257, 2, 1, 128, False, 100, 7, None, None),
    (2, 90, 300, 6, 2, 80, True, 70, 20, [90, 50], [300, 20]),
]


def _backward(q, k, v, g, causal, window, sinks, q_lens, kv_lens, scale, tol, refs=None):
    print("attention backward", tuple(q.shape), tuple(k.shape), q.dtype, causal, window, sinks, q_lens, kv_lens, flush=True)
    kw = dict(causal=causal, window=window, sinks=sinks, scale=scale, q_lens=_lens(q_lens), kv_lens=_lens(kv_lens))
    out, lse = torch.empty_like(q), torch.empty((q.shape[0], q.shape[2], q.shape[1]), device="cuda")
    pd.pd_attention_forward(q, k, v, out, lse=lse, **kw)
    grads = [torch.full(x.shape, 7.0, device="cuda", dtype=x.dtype) for x in (q, k, v)]
    pd.pd_attention_backward(q, k, v, out, lse, g, *grads, **kw)
    refs = refs or ot.attention_grad(_np(q), _np(k), _np(v), _np(g), q.shape[3] ** -0.5 if scale is None else scale, causal,
                                     window, sinks, q_lens, kv_lens)
    for name, got, ref in zip(("dq", "dk", "dv"), grads, refs):
        _close(got, ref, tol, name)
    return grads




@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("case", [c for c in GRAD if c[7] != 1 and c[2] > 1])
def test_attention_backward(case, dtype):
    B, n, m, H, K, D, causal, window, sinks, ql, kl = case
    q, k, v, g = _att_inputs(B, n, m, H, K, D, dtype, 17)
    _backward(q, k, v, g, causal, window, sinks, ql, kl, None, TOL_GRAD[dtype])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("case", [c for c in GRAD if c[7] == 1 or c[2] == 1])
def test_attention_backward_of_rows_with_one_key(case, dtype):
    """p = 1, so dv is dout's sum and the scores' gradient is 0, formed as dout v - dout out: what is left
    of it is the rounding of out (2^-9 or 2^-24) times the sizes of dout, v and q."""
    B, n, m, H, K, D, causal, window, sinks, ql, kl = case
    q, k, v, g = _att_inputs(B, n, m, H, K, D, dtype, 17)
    out, lse = torch.empty_like(q), torch.empty((B, H, n), device="cuda")
    kw = dict(causal=causal, window=window, sinks=sinks)
    pd.pd_attention_forward(q, k, v, out, lse=lse, **kw)
    dq, dk, dv = (torch.full(x.shape, 7.0, device="cuda", dtype=dtype) for x in (q, k, v))
    pd.pd_attention_backward(q, k, v, out, lse, g, dq, dk, dv, **kw)
    rq, rk, rv = ot.attention_grad(_np(q), _np(k), _np(v), _np(g), D ** -0.5, causal, window, sinks)
    _close(dv, rv, TOL_GRAD[dtype], "dv")
    size = float(g.double().abs().max() * v.double().abs().max() * max(q.double().abs().max(), k.double().abs().max())) * D
    for got, ref in ((dq, rq), (dk, rk)):
        assert np.max(np.abs(_np(got) - ref)) <= (2**-9 if dtype == BF16 else 2**-20) * size * H / K


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("case", [c for c in GRAD if c[7] == 1 or c[2] == 1])
def test_attention_backward_of_rows_with_a_key_or_two_to_their_rounding(case, dtype):
    """The same rows element by element: where a key has its row alone dq and dk are what the rounding of out
    leaves of dout v - dout out, far under dout v itself (as in the test of keys beside the largest)."""
    B, n, m, H, K, D, causal, window, sinks, ql, kl = case
    q, k, v, g = _att_inputs(B, n, m, H, K, D, dtype, 37)
    out, lse = torch.empty_like(q), torch.empty((B, H, n), device="cuda")
    kw = dict(causal=causal, window=window, sinks=sinks)
    pd.pd_attention_forward(q, k, v, out, lse=lse, **kw)
    grads = [torch.full(x.shape, 7.0, device="cuda", dtype=dtype) for x in (q, k, v)]
    pd.pd_attention_backward(q, k, v, out, lse, g, *grads, **kw)
    u = 2.0**-8 if dtype == BF16 else 2.0**-15
    refs = ot.attention_grad(_np(q), _np(k), _np(v), _np(g), D ** -0.5, causal, window, sinks)
    bounds = _grad_bounds(q, k, v, g, out, D ** -0.5, causal, u, window, sinks)
    for name, got, ref, bound in zip(("dq", "dk", "dv"), grads, refs, bounds):
        assert np.all(np.abs(_np(got) - ref) <= bound + u * np.abs(ref)), name


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("layout", ["head", "odd"])
@pytest.mark.parametrize("D", [64, 36, 128])
def test_attention_backward_layouts(D, layout, dtype):
    q, k, v, g = _att_inputs(2, 70, 100, 4, 2, D, dtype, 19, layout)
    _backward(q, k, v, g, True, 60, 4, None, None, -0.2, TOL_GRAD[dtype])


def test_attention_backward_against_differences():
    q, k, v, g = _att_inputs(1, 20, 30, 4, 2, 24, F32, 21)
    grads = _backward(q, k, v, g, True, 9, 2, None, None, None, TOL_GRAD[F32])
    args = [_np(x) for x in (q, k, v)]
    for which in range(3):
        d = _np(_rand(args[which].shape, F32, 30 + which))

        def loss(e):
            a = list(args)
            a[which] = a[which] + e * d
            return float(np.sum(ot.attention(*a, 24 ** -0.5, True, 9, 2)[0] * _np(g)))
        want = (loss(1e-5) - loss(-1e-5)) / 2e-5
        assert abs(float(np.sum(_np(grads[which]) * d)) - want) <= 1e-5 * float(grads[which].norm()) * np.linalg.norm(d)


def test_attention_backward_same_bits_again():
    q, k, v, g = _att_inputs(2, 200, 200, 8, 2, 64, BF16, 23)
    a = _backward(q, k, v, g, True, 100, 4, None, None, None, TOL_GRAD[BF16])
    b = _backward(q, k, v, g, True, 100, 4, None, None, None, TOL_GRAD[BF16])
    assert all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_attention_backward_out_of_sight_values(dtype):
    """NaN past a sequence's keys, in queries past its queries, and in a row that sees only some keys."""
    n, m = 60, 90
    q, k, v, g = _att_inputs(2, n, m, 4, 2, 64, dtype, 25)
    ql, kl = [n, 40], [m, 70]
    args = [_np(x) for x in (q, k, v, g)]
    refs = ot.attention_grad(*args, 0.125, True, 30, 3, ql, kl)
    bad = float("nan")
    k[1, 70:], v[1, 70:], q[1, 40:], g[1, 40:] = bad, bad, bad, bad
    _backward(q, k, v, g, True, 30, 3, ql, kl, None, TOL_GRAD[dtype], refs)
    # a live NaN reaches what sees it and nothing else
    q[0, 59] = bad
    out, lse = torch.empty_like(q), torch.empty((2, 4, n), device="cuda")
    kw = dict(causal=True, window=30, sinks=3, q_lens=_lens(ql), kv_lens=_lens(kl))
    pd.pd_attention_forward(q, k, v, out, lse=lse, **kw)
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    pd.pd_attention_backward(q, k, v, out, lse, g, dq, dk, dv, **kw)
    seen = ot.visible(59, n, m, True, 30, 3)
    other = np.setdiff1d(np.arange(m), seen)
    # sight runs both ways: the rows whose keys are clean, the keys that the row does not see
    _close(dq[:, :59], refs[0][:, :59], TOL_GRAD[dtype])
    _close(dk[0, other], refs[1][0, other], TOL_GRAD[dtype])
    _close(dv[0, other], refs[2][0, other], TOL_GRAD[dtype])
    assert torch.isnan(dq[0, 59]).all() and torch.isnan(dk[0, seen]).all() and torch.isnan(dv[0, seen]).all()


def test_attention_refuses_what_it_cannot_read():
    q = torch.zeros((2, 4, 4, 16), device="cuda")
    k = torch.zeros((2, 6, 2, 16), device="cuda")
    o = torch.empty_like(q)
    for bad in (lambda: pd.pd_attention_forward(q, k, k[:, :5], o), lambda: pd.pd_attention_forward(q, k[:1], k[:1], o),
                lambda: pd.pd_attention_forward(q, k.to(BF16), k, o), lambda: pd.pd_attention_forward(q, k, k, o[:, :3]),
                lambda: pd.pd_attention_forward(q, k, k, o, lse=torch.empty((2, 4, 5), device="cuda")),
                lambda: pd.pd_attention_forward(q, k, k, o, kv_lens=torch.zeros(2, device="cuda", dtype=torch.int64)),
                lambda: pd.pd_attention_forward(q, k, k, o[:, :1].expand(2, 4, 4, 16)),
                lambda: pd.pd_attention_forward(q.transpose(2, 3), k, k, o)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(ValueError):
        pd.pd_attention_forward(q, k, k, o, window=-2**40)
    for kw in (dict(window=-1), dict(sinks=-2), dict(scale=float("nan")), dict(scale=1e60)):
        with pytest.raises(pd.PdError):
            pd.pd_attention_forward(q, k, k, o, **kw)
    big = torch.zeros((1, 1, 1, 256), device="cuda")
    with pytest.raises(pd.PdError) as e:
        pd.pd_attention_forward(big, big, big, torch.empty_like(big))
    assert e.value.code == pd.PD_ERR_UNSUPPORTED
    lse = torch.empty((2, 4, 4), device="cuda")
    with pytest.raises(pd.PdError):
        pd.pd_attention_backward(q, k, k, o, lse, q, o, k.clone(), k.clone(), scratch=torch.empty(0, device="cuda"))


# ------------------------------------------------------------------ streams and graphs
def _block(x, w, table, pos, stream=None):
    """Norm, turn and attend, from buffers made beforehand; returns a function that runs it and its output."""
    B, n, H, D = x.shape
    h, rq, rk, out = (torch.empty_like(x) for _ in range(4))
    lse = torch.empty((B, H, n), device="cuda")

    def go(stream=stream):
        pd.pd_rmsnorm_forward(x.view(B * n, H * D), w, h.view(B * n, H * D), stream=stream)
        pd.pd_rotary_apply(h, h, pos, table, rq, rk, stream=stream)
        pd.pd_attention_forward(rq, rk, h, out, lse=lse, window=20, sinks=2, stream=stream)
    return go, out


@pytest.mark.parametrize("n,dtype", [(50, BF16), (50, F32), (1, BF16)])
def test_operators_on_another_stream_and_in_a_graph(n, dtype):
    x, w = _rand((2, n, 4, 64), dtype, 40), _rand((256,), F32, 41)
    table = torch.empty((64, 32, 2), device="cuda")
    pd.pd_rotary_table(table)
    pos = torch.arange(n, device="cuda", dtype=torch.int32)
    go, out = _block(x, w, table, pos)
    go()
    want = out.clone()
    side = torch.cuda.Stream()
    out.zero_()
    side.wait_stream(torch.cuda.current_stream())
    go(side)
    side.synchronize()
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go()
    for i in range(4):
        x.copy_(_rand(x.shape, dtype, 50 + i))
        go()
        want = out.clone()
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want), i


@pytest.mark.parametrize("D,dtype", [(64, BF16), (128, BF16), (128, F32)])
def test_gradients_in_a_graph(D, dtype):
    """The backward calls captured and replayed with other gradients, among them rows with large scores."""
    q, k, v, g = _att_inputs(2, 150, 150, 4, 2, D, dtype, 60)
    q[:, 100:] *= 4096
    out, lse = torch.empty_like(q), torch.empty((2, 4, 150), device="cuda")
    grads = [torch.empty_like(x) for x in (q, k, v)]
    kw = dict(window=90, sinks=3)
    pd.pd_attention_forward(q, k, v, out, lse=lse, **kw)
    assert float(lse.abs().max()) > 2048
    w, dw, rstd = _rand((4 * D,), F32, 61), torch.empty(4 * D, device="cuda"), _rand((300,), F32, 62).abs()
    dx = torch.empty((300, 4 * D), device="cuda", dtype=dtype)

    def go():
        pd.pd_attention_backward(q, k, v, out, lse, g, *grads, **kw)
        pd.pd_rmsnorm_backward(grads[0].view(300, -1), q.view(300, -1), w, rstd, dx, dw)
    go()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go()
    for i in range(4):
        g.copy_(_rand(g.shape, dtype, 70 + i))
        go()
        want = [x.clone() for x in (*grads, dx, dw)]
        for x in (*grads, dx, dw):
            x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip((*grads, dx, dw), want)), i
