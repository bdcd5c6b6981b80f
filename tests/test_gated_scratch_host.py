"""CPU checks of the scratch of the gated product."""
import ctypes

import pytest

import paper_2305_16317_amd as pd

REF = ctypes.byref


def _gated(rows, width, hidden, dtype=pd.PD_BF16, layout=0, aligned=1, **kw):
    rest = width if layout else hidden
    d = dict(rows=rows, width=width, hidden=hidden, dtype=dtype, activation=0, weight_layout=layout, aligned=aligned, x_stride=width,
             w_gate_stride=rest, w_up_stride=rest, gate_stride=hidden, up_stride=hidden, h_stride=hidden, dh_stride=hidden, dx_stride=width,
             dw_gate_stride=rest, dw_up_stride=rest)
    d.update(kw)
    return pd._GatedDesc(**d)


def _bytes(d, backward=False):
    n = ctypes.c_int64(-1)
    L = pd.load()
    assert (L.pd_gated_backward_scratch if backward else L.pd_gated_forward_scratch)(REF(d), REF(n)) == pd.PD_OK
    return n.value


@pytest.mark.parametrize("layout", [0, 1])
def test_scratch_has_no_room_for_operands_that_are_read_where_they_are(layout):
    """A sum in one part: none forward, and dgate and dup (two parts of 2 bytes a value each) backward, but for sums in parts."""
    M, D, F = 36864, 1024, 4096
    laid = M * D * 2, 2 * D * F * 2
    assert _bytes(_gated(M, D, F, layout=layout)) == 0
    assert _bytes(_gated(M, D, F, layout=layout, aligned=0)) == sum(laid)
    slopes = 2 * 2 * 2 * M * F
    with_room = _bytes(_gated(M, D, F, layout=layout, aligned=0), True)
    assert with_room - _bytes(_gated(M, D, F, layout=layout), True) == sum(laid) and with_room >= sum(laid) + slopes
    # rows that no copy of 16 bytes reads, weights at two distances, float32: these are laid out as before
    for kw, part in ((dict(x_stride=D + 4), laid[0]), (dict(w_up_stride=8192), laid[1])):
        assert _bytes(_gated(M, D, F, layout=layout, **kw)) == part
    assert _bytes(_gated(1600, 1024, 2736, pd.PD_F32, layout)) == _bytes(_gated(1600, 1024, 2736, pd.PD_F32, layout, aligned=0)) > 0


def test_operands_that_are_not_aligned_as_said_are_refused():
    L, P = pd.load(), ctypes.c_void_p(1 << 20)
    odd = ctypes.c_void_p((1 << 20) + 8)
    d = _gated(300, 64, 64)
    for which in range(3):                                   # x, w_gate, w_up
        args = [P] * 7
        args[which] = odd
        assert L.pd_gated_forward(REF(d), *args, 1 << 30, None) == pd.PD_ERR_INVALID_ARG and b"16 bytes" in L.pd_last_error()
        args = [P] * 11
        args[which] = odd
        assert L.pd_gated_backward(REF(d), *args, 1 << 30, None) == pd.PD_ERR_INVALID_ARG and b"16 bytes" in L.pd_last_error()
