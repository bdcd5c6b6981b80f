"""CPU checks of the transformer operators: the oracle's own gradients against
differences, and the refusals of the C entry points and of the binding, which
need no GPU."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2305_16317_amd as pd
from oracle import transformer as ot


# ------------------------------------------------------------------ the oracle
def _difference(f, x, direction, eps=1e-5):
    return (f(x + eps * direction) - f(x - eps * direction)) / (2 * eps)


@pytest.mark.parametrize("causal,window,sinks,lens", [
    (True, 0, 0, None), (False, 0, 0, None), (True, 3, 2, [9, 4]), (False, 2, 1, [7, 0])])
def test_oracle_attention_gradient_matches_differences(causal, window, sinks, lens):
    r = np.random.default_rng(1)
    q, do = r.standard_normal((2, 2, 6, 4, 5))
    k, v = r.standard_normal((2, 2, 9, 2, 5))
    kw = dict(scale=0.4, causal=causal, window=window, sinks=sinks, kv_lens=lens)
    grads = ot.attention_grad(q, k, v, do, **kw)
    for which in range(3):
        def loss(x):
            a = [q, k, v]
            a[which] = x
            return float(np.sum(ot.attention(*a, **kw)[0] * do))
        x = (q, k, v)[which]
        d = r.standard_normal(x.shape)
        # central differences in float64: error ~ eps^2 f''' + 1e-16 |f| / eps ~ 1e-9
        assert abs(_difference(loss, x, d) - np.sum(grads[which] * d)) < 1e-7


def test_oracle_norm_gradient_matches_differences():
    r = np.random.default_rng(2)
    x, dy, ds = r.standard_normal((3, 5, 7))
    w = r.standard_normal(7)
    s, _, rstd = ot.rmsnorm(x, None, w, 1e-3)
    dx, dw = ot.rmsnorm_grad(dy, s, w, rstd, ds)
    loss = lambda x, w: float(np.sum(ot.rmsnorm(x, None, w, 1e-3)[1] * dy) + np.sum(x * ds))  # noqa: E731
    d, e = r.standard_normal(x.shape), r.standard_normal(7)
    assert abs(_difference(lambda y: loss(y, w), x, d) - np.sum(dx * d)) < 1e-7
    assert abs(_difference(lambda y: loss(x, y), w, e) - np.sum(dw * e)) < 1e-7


def test_oracle_rotary_backward_is_the_transpose():
    r = np.random.default_rng(3)
    x, g = r.standard_normal((2, 1, 4, 2, 10))
    table = ot.rotary_table(ot.rotary_freqs(6, 100.0, "by_parts", 2.0, 50.0), range(9), 1.2)
    pos = np.array([[0, 3, 8, 50]])
    for inter in (False, True):
        a = np.sum(ot.rotary(x, table, pos, inter) * g)
        b = np.sum(x * ot.rotary(g, table, pos, inter, backward=True))
        assert abs(a - b) < 1e-12


def test_e4m3_values():
    v = ot.e4m3_values()
    assert v.size == 127 and v[-1] == 448 and np.all(np.diff(v) > 0)
    t = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(t, v)


# ------------------------------------------------------------------ refusals of the C entry points
def _status(name, *args):
    L = pd.load()
    return getattr(L, name)(*args), L.pd_last_error().decode()


def _norm(**kw):
    d = dict(rows=4, width=8, x_stride=8, residual_stride=8, sum_stride=8, y_stride=8, dtype=pd.PD_F32,
             out_dtype=pd.PD_F32, group=0, eps=1e-6)
    d.update(kw)
    return pd._RmsnormDesc(**d)


P = ctypes.c_void_p(16)      # a pointer that no refused call may follow


@pytest.mark.parametrize("kw,msg", [
    (dict(rows=-1), "rows"), (dict(width=0), "width"), (dict(width=65537), "width"), (dict(dtype=2), "dtype"),
    (dict(out_dtype=pd.PD_BF16), "out_dtype"), (dict(eps=-1.0), "eps"), (dict(eps=float("nan")), "eps"),
    (dict(x_stride=-8), "stride"), (dict(y_stride=7), "y_stride"), (dict(sum_stride=0), "sum_stride"),
    (dict(out_dtype=pd.PD_F8E4M3, group=24), "group"), (dict(out_dtype=pd.PD_F8E4M3, group=8), "group"),
    (dict(out_dtype=pd.PD_F8E4M3, group=1024), "group"), (dict(group=-16), "group"),
])
def test_norm_refusals(kw, msg):
    code, m = _status("pd_rmsnorm_forward", ctypes.byref(_norm(**kw)), P, P, P, P, P, P, P, None)
    assert code == pd.PD_ERR_INVALID_ARG and msg in m


def test_norm_null_arguments():
    d = _norm()
    for i in (0, 2, 4):                                    # x, weight, y
        args = [P, P, P, P, P, P, P]
        args[i] = None
        assert _status("pd_rmsnorm_forward", ctypes.byref(d), *args, None)[0] == pd.PD_ERR_INVALID_ARG
    assert _status("pd_rmsnorm_forward", None, P, P, P, P, P, P, P, None)[0] == pd.PD_ERR_INVALID_ARG
    code, m = _status("pd_rmsnorm_forward", ctypes.byref(_norm(out_dtype=pd.PD_F8E4M3)), P, P, P, P, P, None, P, None)
    assert code == pd.PD_ERR_INVALID_ARG and "scale" in m
    assert _status("pd_rmsnorm_forward", ctypes.byref(_norm(rows=0)), *[None] * 7, None)[0] == pd.PD_OK
    bad = _norm(out_dtype=pd.PD_F8E4M3)
    assert _status("pd_rmsnorm_backward", ctypes.byref(bad), *[P] * 8, 0, None)[0] == pd.PD_ERR_INVALID_ARG


def _table(**kw):
    d = dict(rotary_dim=8, scaling=pd.PD_ROTARY_PLAIN, base=1e4, factor=1.0, original_length=0.0, turns_low=1.0,
             turns_high=32.0, magnitude=1.0)
    d.update(kw)
    return pd._RotaryTableDesc(**d)


@pytest.mark.parametrize("kw,msg", [
    (dict(rotary_dim=7), "rotary_dim"), (dict(rotary_dim=0), "rotary_dim"), (dict(scaling=4), "scaling"),
    (dict(base=1.0), "base"), (dict(scaling=pd.PD_ROTARY_LINEAR, factor=0.5), "factor"),
    (dict(scaling=pd.PD_ROTARY_BY_PARTS, original_length=0.0), "original_length"),
    (dict(scaling=pd.PD_ROTARY_BY_PARTS, original_length=9.0, turns_low=32.0), "turns"),
    (dict(magnitude=float("inf")), "magnitude")])
def test_rotary_table_refusals(kw, msg):
    code, m = _status("pd_rotary_table", ctypes.byref(_table(**kw)), 0, 4, P, None)
    assert code == pd.PD_ERR_INVALID_ARG and msg in m
    for first, rows in ((-1, 4), (0, -1)):
        assert _status("pd_rotary_table", ctypes.byref(_table()), first, rows, P, None)[0] == pd.PD_ERR_INVALID_ARG
    assert _status("pd_rotary_table", ctypes.byref(_table()), 0, 0, None, None)[0] == pd.PD_OK


def test_launches_past_2_32_threads_are_refused():
    code, _ = _status("pd_rotary_table", ctypes.byref(_table(rotary_dim=128)), 0, 2**27, P, None)
    assert code == pd.PD_ERR_UNSUPPORTED
    for kw in (dict(batch=2**31, length=2**20), dict(batch=2**20, length=2**12, heads_q=64, head_dim=128, rotary_dim=64)):
        assert _status("pd_rotary_apply", ctypes.byref(_rotary(**kw)), *[P] * 6, None)[0] == pd.PD_ERR_UNSUPPORTED


def _rotary(**kw):
    st = pd._I64x3(64, 32, 8)
    d = dict(batch=2, length=3, heads_q=4, heads_k=2, head_dim=8, rotary_dim=8, layout=0, dtype=pd.PD_F32, backward=0,
             table_rows=5, position_stride=0, q_stride=st, k_stride=st, q_out_stride=st, k_out_stride=st)
    d.update(kw)
    return pd._RotaryDesc(**d)


@pytest.mark.parametrize("kw,msg", [
    (dict(batch=-1), "batch"), (dict(heads_q=0), "heads"), (dict(rotary_dim=10), "rotary_dim"),
    (dict(rotary_dim=3), "rotary_dim"), (dict(head_dim=2048), "head_dim"), (dict(layout=2), "layout"),
    (dict(dtype=3), "dtype"), (dict(table_rows=0), "table_rows"), (dict(position_stride=-1), "position_stride"),
    (dict(q_stride=pd._I64x3(-1, 0, 0)), "stride")])
def test_rotary_refusals(kw, msg):
    code, m = _status("pd_rotary_apply", ctypes.byref(_rotary(**kw)), P, P, P, P, P, P, None)
    assert code == pd.PD_ERR_INVALID_ARG and msg in m


def test_rotary_null_arguments():
    for i in (0, 2, 3, 4, 5):                              # q, positions, table, q_out, k_out
        args = [P] * 6
        args[i] = None
        assert _status("pd_rotary_apply", ctypes.byref(_rotary()), *args, None)[0] == pd.PD_ERR_INVALID_ARG
    assert _status("pd_rotary_apply", ctypes.byref(_rotary(length=0)), *[None] * 6, None)[0] == pd.PD_OK


def _att(**kw):
    st = pd._I64x3(640, 64, 16)
    d = dict(batch=2, heads_q=4, heads_kv=2, head_dim=16, q_len=3, kv_len=5, dtype=pd.PD_BF16, causal=1, window=0, sinks=0,
             scale=0.25)
    d.update({n + "_stride": st for n in ("q", "k", "v", "out", "dq", "dk", "dv", "dout")})
    d.update(kw)
    return pd._AttentionDesc(**d)


@pytest.mark.parametrize("kw,code,msg", [
    (dict(batch=-1), 1, "batch"), (dict(heads_kv=3), 1, "multiple"), (dict(heads_kv=0), 1, "heads"),
    (dict(head_dim=0), 1, "head_dim"), (dict(head_dim=129), 5, "head_dim"), (dict(q_len=-1), 1, "q_len"),
    (dict(window=-1), 1, "window"), (dict(sinks=-1), 1, "sinks"), (dict(scale=float("inf")), 1, "scale"),
    (dict(dtype=2), 1, "dtype"), (dict(k_stride=pd._I64x3(0, -1, 0)), 1, "stride"),
    (dict(kv_len=2**30), 5, "keys"), (dict(q_len=2**30), 5, "keys"),
    (dict(batch=2**30, heads_kv=1, heads_q=1, q_len=64), 5, "tiles")])
def test_attention_refusals(kw, code, msg):
    d = _att(**kw)
    n = ctypes.c_int64()
    for got in (_status("pd_attention_forward", ctypes.byref(d), *[P] * 8, 0, None),
                _status("pd_attention_backward", ctypes.byref(d), *[P] * 12, 0, None),
                _status("pd_attention_forward_scratch", ctypes.byref(d), ctypes.byref(n)),
                _status("pd_attention_backward_scratch", ctypes.byref(d), ctypes.byref(n))):
        assert got[0] == code and msg in got[1]


def test_attention_null_arguments():
    d = _att()
    for i in (0, 1, 2, 5):                                 # q, k, v, out
        args = [P] * 8
        args[i] = None
        assert _status("pd_attention_forward", ctypes.byref(d), *args, 1 << 30, None)[0] == pd.PD_ERR_INVALID_ARG
    for i in (0, 1, 2, 3, 4, 5, 8, 9, 10):
        args = [P] * 12
        args[i] = None
        assert _status("pd_attention_backward", ctypes.byref(d), *args, 1 << 30, None)[0] == pd.PD_ERR_INVALID_ARG
    assert _status("pd_attention_forward", ctypes.byref(_att(batch=0)), *[None] * 8, 0, None)[0] == pd.PD_OK
    assert _status("pd_attention_forward", None, *[P] * 8, 0, None)[0] == pd.PD_ERR_INVALID_ARG


def _share(stride, counts, row):
    """Whether rows at the strides share an element, by going through them all."""
    at = sorted(sum(i * s for i, s in zip(ix, stride)) for ix in np.ndindex(*counts))
    return any(b - a < row for a, b in zip(at, at[1:]))


def test_outputs_whose_rows_share_elements_are_refused():
    """What passes the check is refused by the next: scratch is missing (many keys or a gradient need some)."""
    r = np.random.default_rng(4)
    cases = [(640, 64, 16), (64, 128, 16), (16, 32, 160), (0, 64, 16), (640, 0, 16), (640, 64, 15), (640, 60, 16), (100, 64, 16),
             (48, 32, 16), (40, 64, 24), (2**39, 2**39, 2**39), (2**39, 2**20, 16)]
    cases += [tuple(8 * r.integers(0, 40, 3)) for _ in range(400)]
    seen = {True: 0, False: 0}
    for stride in cases:
        st = pd._I64x3(*[int(x) for x in stride])
        for name, counts in (("out", (2, 3, 4)), ("dq", (2, 3, 4)), ("dk", (2, 5, 2)), ("dv", (2, 5, 2))):
            want = _share(stride, counts, 16)
            seen[want] += 1
            d = _att(**{name + "_stride": st}, kv_len=2**20 if name == "out" else 5)
            if name == "out":
                code, m = _status("pd_attention_forward", ctypes.byref(d), *[P] * 7, None, 0, None)
            else:
                code, m = _status("pd_attention_backward", ctypes.byref(d), *[P] * 11, None, 0, None)
            assert code == pd.PD_ERR_INVALID_ARG
            assert ("share elements" in m and name in m) == want and ("scratch" in m) != want, (name, stride, m)
        counts = (2, 3, 4)
        d = _rotary(q_out_stride=st, k_out_stride=pd._I64x3(96, 32, 8), table_rows=1)
        code, m = _status("pd_rotary_apply", ctypes.byref(d), *[P] * 6, None) if _share(stride, counts, 8) else (None, "")
        assert code in (None, pd.PD_ERR_INVALID_ARG) and (code is None or "q_out" in m)
    assert min(seen.values()) > 100
    # single elements of an axis have no stride; what is only read may be shared
    for kw in (dict(batch=1, out_stride=pd._I64x3(0, 64, 16)), dict(q_len=1, out_stride=pd._I64x3(64, 3, 16)),
               dict(q_stride=pd._I64x3(0, 0, 0), k_stride=pd._I64x3(0, 0, 16))):
        code, m = _status("pd_attention_forward", ctypes.byref(_att(kv_len=2**20, **kw)), *[P] * 7, None, 0, None)
        assert code == pd.PD_ERR_INVALID_ARG and "scratch" in m


def test_packed_descriptions_are_laid_out_as_the_structures():
    for packed, struct in ((pd._RMSNORM_BYTES, pd._RmsnormDesc), (pd._ROTARY_BYTES, pd._RotaryDesc),
                           (pd._ATTENTION_BYTES, pd._AttentionDesc)):
        assert packed.size == ctypes.sizeof(struct)
        n = len(packed.unpack(bytes(packed.size)))
        d = struct.from_buffer_copy(packed.pack(*range(1, n + 1)))
        flat = []
        for name, kind in struct._fields_:
            v = getattr(d, name)
            flat += list(v) if hasattr(v, "__len__") else [v]
        assert flat == list(range(1, n + 1))


# ------------------------------------------------------------------ refusals of the binding
def test_binding_refuses_cpu_tensors_and_wrong_types():
    x = torch.zeros(2, 8)
    with pytest.raises(ValueError):
        pd.pd_rmsnorm_forward(x, torch.ones(8), torch.zeros(2, 8))
    with pytest.raises(ValueError):
        pd.pd_rmsnorm_forward(x.half(), torch.ones(8), x.half())
    q = torch.zeros(1, 2, 1, 8)
    with pytest.raises(ValueError):
        pd.pd_attention_forward(q, q, q, q)
    with pytest.raises(ValueError):
        pd.pd_rotary_apply(q, q, torch.zeros(2, dtype=torch.int32), torch.zeros(2, 4, 2), q, q)
    with pytest.raises(ValueError):
        pd.pd_rotary_table(torch.zeros(2, 4, 2))
