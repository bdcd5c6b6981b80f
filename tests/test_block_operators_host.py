"""CPU checks of the block's operators: the oracle's own gradients against differences, and the refusals of
the C entry points and of the binding, which need no GPU."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2305_16317_amd as pd
from oracle import block as ob


# ------------------------------------------------------------------ the oracle
def _difference(f, x, direction, eps=1e-5):
    return (f(x + eps * direction) - f(x - eps * direction)) / (2 * eps)


@pytest.mark.parametrize("runs", [0, 3])
def test_oracle_layernorm_gradient_matches_differences(runs):
    r = np.random.default_rng(1)
    x, dy, ds = r.standard_normal((3, 6, 7))
    w, b = r.standard_normal((2, *((runs, 7) if runs else (7,))))
    s, _, mean, rstd = ob.layernorm(x, None, w, b, 1e-3)
    grads = ob.layernorm_grad(dy, s, w, mean, rstd, ds, runs)
    loss = lambda x, w, b: float(np.sum(ob.layernorm(x, None, w, b, 1e-3)[1] * dy) + np.sum(x * ds))  # noqa: E731
    for which, v in enumerate((x, w, b)):
        def one(t):
            a = [x, w, b]
            a[which] = t
            return loss(*a)
        d = r.standard_normal(v.shape)
        # central differences in float64: error ~ eps^2 f''' + 1e-16 |f| / eps ~ 1e-9
        assert abs(_difference(one, v, d) - np.sum(grads[which] * d)) < 1e-7


@pytest.mark.parametrize("kind", ["silu", "gelu", "gelu_tanh", "sigmoid", "relu"])
def test_oracle_gated_gradient_matches_differences(kind):
    r = np.random.default_rng(2)
    x, wg, wu, dh = (r.standard_normal(s) for s in ((4, 5), (5, 6), (5, 6), (4, 6)))
    h, g, u = ob.gated(x, wg, wu, kind)
    grads = ob.gated_grad(dh, x, wg, wu, g, u, kind)
    assert np.allclose(grads[3], h, rtol=1e-12, atol=1e-12)
    for which in range(3):
        def loss(t):
            a = [x, wg, wu]
            a[which] = t
            return float(np.sum(ob.gated(*a, kind)[0] * dh))
        v = (x, wg, wu)[which]
        d = r.standard_normal(v.shape)
        assert abs(_difference(loss, v, d, 1e-6) - np.sum(grads[which] * d)) < 1e-6


def test_oracle_rotary_axes_backward_is_the_transpose():
    r = np.random.default_rng(3)
    x, g = r.standard_normal((2, 1, 4, 2, 18))
    sections = [3, 1, 4]
    pos = r.integers(-1, 12, (1, 4, 3))
    for turns in (False, True):
        axis = ob.axis_of_pair(sections, turns)
        assert sorted(axis) == [0] * 3 + [1] + [2] * 4
        table = ob.axes_table(sections, turns, range(9), [10.0] * 3, [1.0, 2.0, 0.5], False)
        for inter in (False, True):
            a = np.sum(ob.rotary_axes(x, table, pos, axis, inter) * g)
            b = np.sum(x * ob.rotary_axes(g, table, pos, axis, inter, backward=True))
            assert abs(a - b) < 1e-12
    assert ob.axis_of_pair([3, 1, 4], True) == [0, 1, 2, 0, 2, 0, 2, 2]


def test_oracle_dropout_mask():
    a = ob.kept(64, 500, 0.25, 2**63 + 7, 3, 11)
    assert abs(a.mean() - 0.75) < 5 * np.sqrt(0.25 * 0.75 / a.size)
    assert np.array_equal(ob.kept(10, 500, 0.25, 2**63 + 7, 3, 11, first_row=54), a[54:])
    assert np.array_equal(ob.kept(64, 496, 0.25, 2**63 + 7, 3, 11)[0], a[0, :496])
    assert ob.kept(4, 9, 0.0, 1, 0, 0).all() and not ob.kept(4, 9, 1.0, 1, 0, 0).any()


# ------------------------------------------------------------------ refusals of the C entry points
def _status(name, *args):
    L = pd.load()
    return getattr(L, name)(*args), L.pd_last_error().decode()


P = ctypes.c_void_p(16)      # a pointer that no refused call may follow
REF = ctypes.byref


def _norm(**kw):
    d = dict(rows=4, width=8, span=2, x_stride=8, residual_stride=8, sum_stride=8, y_stride=8, weight_stride=8, bias_stride=8,
             dtype=pd.PD_F32, eps=1e-6)
    d.update(kw)
    return pd._LayernormDesc(**d)


@pytest.mark.parametrize("kw,msg", [
    (dict(rows=-1), "rows"), (dict(rows=2**31 + 2), "rows"), (dict(width=0), "width"), (dict(width=65537), "width"),
    (dict(dtype=2), "dtype"), (dict(eps=-1.0), "eps"), (dict(eps=float("nan")), "eps"), (dict(span=3), "span"),
    (dict(span=-2), "span"), (dict(x_stride=-8), "stride"), (dict(weight_stride=-1), "stride"), (dict(bias_stride=2**40), "stride"),
    (dict(y_stride=7), "y_stride"), (dict(sum_stride=0), "sum_stride")])
def test_layernorm_refusals(kw, msg):
    code, m = _status("pd_layernorm_forward", REF(_norm(**kw)), *[P] * 8, None)
    assert code == pd.PD_ERR_INVALID_ARG and msg in m


def test_layernorm_null_arguments():
    d = _norm()
    for i in (0, 5):                                       # x, y
        args = [P] * 8
        args[i] = None
        assert _status("pd_layernorm_forward", REF(d), *args, None)[0] == pd.PD_ERR_INVALID_ARG
    assert _status("pd_layernorm_forward", None, *[P] * 8, None)[0] == pd.PD_ERR_INVALID_ARG
    assert _status("pd_layernorm_forward", REF(_norm(rows=0)), *[None] * 8, None)[0] == pd.PD_OK
    for i in (0, 1, 3, 4, 6):                              # dy, sum, mean, rstd, dx
        args = [P] * 9
        args[i] = None
        assert _status("pd_layernorm_backward", REF(d), *args, P, 1 << 30, None)[0] == pd.PD_ERR_INVALID_ARG
    code, m = _status("pd_layernorm_backward", REF(_norm(x_stride=4)), *[P] * 9, P, 1 << 30, None)
    assert code == pd.PD_ERR_INVALID_ARG and "dx" in m
    code, m = _status("pd_layernorm_backward", REF(_norm(rows=4096, span=0)), *[P] * 9, None, 0, None)
    assert code == pd.PD_ERR_INVALID_ARG and "scratch" in m
    n = ctypes.c_int64()
    assert _status("pd_layernorm_backward_scratch", REF(_norm(rows=4096, span=1)), REF(n))[0] == pd.PD_OK and n.value == 0
    assert _status("pd_layernorm_backward_scratch", REF(_norm(rows=4096, span=0)), REF(n))[0] == pd.PD_OK and n.value > 0
    assert _status("pd_layernorm_backward_scratch", REF(d), None)[0] == pd.PD_ERR_INVALID_ARG
    # a span without rows has no runs, and so no gradients to write
    assert _status("pd_layernorm_backward", REF(_norm(rows=0)), *[None] * 9, None, 0, None)[0] == pd.PD_OK


def _rotary(axes=2, order=0, sections=(2, 2, 0, 0), position_stride=(0, 2, 1), **kw):
    st = pd._I64x3(64, 32, 8)
    d = dict(batch=2, length=3, heads_q=4, heads_k=2, head_dim=8, rotary_dim=8, layout=0, dtype=pd.PD_F32, backward=0,
             table_rows=5, position_stride=0, q_stride=st, k_stride=st, q_out_stride=st, k_out_stride=st)
    d.update(kw)
    return pd._RotaryAxesDesc(pd._RotaryDesc(**d), axes, order, (ctypes.c_int32 * 4)(*sections), pd._I64x3(*position_stride))


@pytest.mark.parametrize("kw,msg", [
    (dict(axes=0), "axes"), (dict(axes=5), "axes"), (dict(order=2), "order"), (dict(sections=(2, 3, 0, 0)), "sections"),
    (dict(sections=(5, -1, 0, 0)), "sections"), (dict(axes=1), "sections"), (dict(position_stride=(0, -1, 1)), "stride"),
    (dict(batch=-1), "batch"), (dict(rotary_dim=10), "rotary_dim"), (dict(layout=2), "layout"), (dict(dtype=3), "dtype"),
    (dict(table_rows=0), "table_rows"), (dict(q_out_stride=pd._I64x3(0, 32, 8)), "q_out")])
def test_rotary_axes_refusals(kw, msg):
    code, m = _status("pd_rotary_axes_apply", REF(_rotary(**kw)), *[P] * 6, None)
    assert code == pd.PD_ERR_INVALID_ARG and msg in m


def test_rotary_axes_null_arguments():
    for i in (0, 2, 3, 4, 5):                              # q, positions, table, q_out, k_out
        args = [P] * 6
        args[i] = None
        assert _status("pd_rotary_axes_apply", REF(_rotary()), *args, None)[0] == pd.PD_ERR_INVALID_ARG
    assert _status("pd_rotary_axes_apply", REF(_rotary(length=0)), *[None] * 6, None)[0] == pd.PD_OK
    code, _ = _status("pd_rotary_axes_apply", REF(_rotary(batch=2**31, length=2**20)), *[P] * 6, None)
    assert code == pd.PD_ERR_UNSUPPORTED


@pytest.mark.parametrize("kw,msg", [
    (dict(rotary_dim=7), "rotary_dim"), (dict(rotary_dim=2048), "rotary_dim"), (dict(axes=0), "axes"), (dict(order=-1), "order"),
    (dict(sections=(1, 2, 0, 0)), "sections"), (dict(base=(1.0, 2.0, 0, 0)), "base"), (dict(scale=(float("inf"), 1, 0, 0)), "scale")])
def test_rotary_axes_table_refusals(kw, msg):
    d = dict(rotary_dim=8, axes=2, order=0, shared=0, sections=(2, 2, 0, 0), base=(1e4, 1e4, 0, 0), scale=(1, 1, 0, 0))
    d.update(kw)
    for name, kind in (("sections", ctypes.c_int32), ("base", ctypes.c_double), ("scale", ctypes.c_double)):
        d[name] = (kind * 4)(*d[name])
    code, m = _status("pd_rotary_axes_table", REF(pd._RotaryAxesTableDesc(**d)), 0, 4, P, None)
    assert code == pd.PD_ERR_INVALID_ARG and msg in m


def test_rotary_axes_table_ranges():
    d = pd._RotaryAxesTableDesc(8, 1, 0, 0, (ctypes.c_int32 * 4)(4, 0, 0, 0), (ctypes.c_double * 4)(1e4), (ctypes.c_double * 4)(1))
    for first, rows in ((-1, 4), (0, -1)):
        assert _status("pd_rotary_axes_table", REF(d), first, rows, P, None)[0] == pd.PD_ERR_INVALID_ARG
    assert _status("pd_rotary_axes_table", REF(d), 0, 0, None, None)[0] == pd.PD_OK
    d.rotary_dim, d.sections[0] = 128, 64
    assert _status("pd_rotary_axes_table", REF(d), 0, 2**27, P, None)[0] == pd.PD_ERR_UNSUPPORTED


def _drop(**kw):
    d = dict(rows=4, width=8, first_row=0, x_stride=8, residual_stride=8, y_stride=8, seed=1, p=0.5, rng_stream=0, step=0, dtype=0)
    d.update(kw)
    return pd._DropoutDesc(**d)


@pytest.mark.parametrize("kw,msg", [
    (dict(rows=-1), "rows"), (dict(width=0), "width"), (dict(width=2**31), "width"), (dict(rows=2**40, width=2**10), "rows"),
    (dict(first_row=-1), "rows"), (dict(first_row=2**40, width=2**30, rows=1, y_stride=2**30), "first_row"), (dict(p=-0.1), "p must"),
    (dict(p=1.5), "p must"), (dict(p=float("nan")), "p must"), (dict(dtype=2), "dtype"), (dict(x_stride=-1), "stride"),
    (dict(y_stride=7), "y_stride")])
def test_dropout_refusals(kw, msg):
    code, m = _status("pd_dropout_apply", REF(_drop(**kw)), P, P, P, P, None)
    assert code == pd.PD_ERR_INVALID_ARG and msg in m


def test_dropout_null_arguments():
    assert _status("pd_dropout_apply", REF(_drop(step=2**32 - 1)), P, None, None, P, None)[0] == pd.PD_ERR_INVALID_ARG
    for args in ((None, None, None, P), (P, None, None, None)):
        assert _status("pd_dropout_apply", REF(_drop()), *args, None)[0] == pd.PD_ERR_INVALID_ARG
    assert _status("pd_dropout_apply", None, P, None, None, P, None)[0] == pd.PD_ERR_INVALID_ARG
    assert _status("pd_dropout_apply", REF(_drop(rows=0)), None, None, None, None, None)[0] == pd.PD_OK


def _gated(**kw):
    d = dict(rows=4, width=8, hidden=16, dtype=pd.PD_BF16, activation=0, weight_layout=0, x_stride=8, w_gate_stride=16,
             w_up_stride=16, gate_stride=16, up_stride=16, h_stride=16, dh_stride=16, dx_stride=8, dw_gate_stride=16, dw_up_stride=16)
    d.update(kw)
    return pd._GatedDesc(**d)


@pytest.mark.parametrize("kw,code,msg", [
    (dict(rows=-1), 1, "rows"), (dict(width=0), 1, "width"), (dict(hidden=0), 1, "hidden"), (dict(hidden=2**20 + 1), 1, "hidden"),
    (dict(dtype=2), 1, "dtype"), (dict(activation=5), 1, "activation"), (dict(activation=-1), 1, "activation"),
    (dict(weight_layout=2), 1, "weight_layout"), (dict(x_stride=-1), 1, "stride"), (dict(dw_up_stride=2**40), 1, "stride"),
    (dict(rows=2**24 + 1), 5, "rows"), (dict(rows=2**24, hidden=2**20), 5, "tiles"), (dict(width=2**20, hidden=2**20), 5, "tiles")])
def test_gated_refusals(kw, code, msg):
    d = _gated(**kw)
    n = ctypes.c_int64()
    for got in (_status("pd_gated_forward", REF(d), *[P] * 7, 1 << 40, None),
                _status("pd_gated_backward", REF(d), *[P] * 11, 1 << 40, None),
                _status("pd_gated_forward_scratch", REF(d), REF(n)), _status("pd_gated_backward_scratch", REF(d), REF(n))):
        assert got[0] == code and msg in got[1]


def test_gated_null_arguments():
    d = _gated()
    for i in (0, 1, 2, 5):                                 # x, w_gate, w_up, h
        args = [P] * 7
        args[i] = None
        assert _status("pd_gated_forward", REF(d), *args, 1 << 30, None)[0] == pd.PD_ERR_INVALID_ARG
    for i in (0, 1, 2, 3, 4, 5, 8, 9):                     # x, weights, gate, up, dh, one of dw_gate and dw_up
        args = [P] * 11
        args[i] = None
        assert _status("pd_gated_backward", REF(d), *args, 1 << 30, None)[0] == pd.PD_ERR_INVALID_ARG, i
    assert _status("pd_gated_forward", REF(_gated(rows=0)), *[None] * 7, 0, None)[0] == pd.PD_OK
    assert _status("pd_gated_backward", REF(_gated(rows=0)), *[None] * 11, 0, None)[0] == pd.PD_OK
    assert _status("pd_gated_backward", REF(d), *[P] * 6, None, None, None, None, None, 0, None)[0] == pd.PD_OK     # nothing asked for
    assert _status("pd_gated_forward", None, *[P] * 7, 0, None)[0] == pd.PD_ERR_INVALID_ARG
    big = _gated(rows=4096, width=72, x_stride=72)
    for name, count in (("pd_gated_forward", 6), ("pd_gated_backward", 10)):
        code, m = _status(name, REF(big), *[P] * count, None, 0, None)
        assert code == pd.PD_ERR_INVALID_ARG and ("scratch" in m or "share" in m)
    for kw, what in ((dict(h_stride=15), "h"), (dict(gate_stride=4), "gate"), (dict(up_stride=0), "up")):
        code, m = _status("pd_gated_forward", REF(_gated(**kw)), *[P] * 7, 1 << 30, None)
        assert code == pd.PD_ERR_INVALID_ARG and m.startswith(what)
    for kw, what in ((dict(dx_stride=7), "dx"), (dict(dw_gate_stride=8), "dw_gate"), (dict(dw_up_stride=8), "dw_up")):
        code, m = _status("pd_gated_backward", REF(_gated(**kw)), *[P] * 11, 1 << 30, None)
        assert code == pd.PD_ERR_INVALID_ARG and m.startswith(what)


def test_packed_descriptions_are_laid_out_as_the_structures():
    def flat(d):
        out = []
        for name, _ in d._fields_:
            v = getattr(d, name)
            out += flat(v) if isinstance(v, ctypes.Structure) else list(v) if hasattr(v, "__len__") else [v]
        return out
    for packed, struct in ((pd._LAYERNORM_BYTES, pd._LayernormDesc), (pd._ROTARY_AXES_BYTES, pd._RotaryAxesDesc),
                           (pd._DROPOUT_BYTES, pd._DropoutDesc), (pd._GATED_BYTES, pd._GatedDesc)):
        assert packed.size == ctypes.sizeof(struct)
        n = len(packed.unpack(bytes(packed.size)))
        assert flat(struct.from_buffer_copy(packed.pack(*range(1, n + 1)))) == list(range(1, n + 1))


# ------------------------------------------------------------------ refusals of the binding
def test_binding_refuses_cpu_tensors():
    x, w, q = torch.zeros(2, 8), torch.zeros(8, 8), torch.zeros(1, 2, 1, 8)
    for bad in (lambda: pd.pd_layernorm_forward(x, x), lambda: pd.pd_layernorm_backward(x, x, x[:, 0], x[:, 0], x),
                lambda: pd.pd_rotary_axes_apply(q, q, torch.zeros(2, 1, dtype=torch.int32), torch.zeros(2, 4, 2), [4], q, q),
                lambda: pd.pd_rotary_axes_table(torch.zeros(2, 4, 2), [4]), lambda: pd.pd_dropout_apply(x, x, 0.1, 1),
                lambda: pd.pd_gated_forward(x, w, w, x), lambda: pd.pd_gated_backward(x, x, w, w, x, x, dx=x),
                lambda: pd.pd_layernorm_forward(x.half(), x.half())):
        with pytest.raises(ValueError):
            bad()
