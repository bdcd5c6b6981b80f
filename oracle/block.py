"""Plain float64 forms of the operators of a latent transformer's block, from their definitions:
layer norm modulated by runs of rows, rotary positions over several axes, dropout and the gated
feed-forward product."""
from __future__ import annotations

import math

import numpy as np

from .philox import philox4x32_10

__all__ = ["layernorm", "layernorm_grad", "axis_of_pair", "axes_table", "rotary_axes", "kept", "dropout", "activate",
           "gated", "gated_grad"]


# ------------------------------------------------------------------ layer norm
def _by_run(w, rows, width, default):
    """Weight or bias [width] or [runs, width] as [rows, width]."""
    if w is None:
        return np.full((rows, width), default)
    w = np.atleast_2d(w.astype(np.float64))
    return np.repeat(w, rows // w.shape[0], axis=0) if rows else np.empty((0, width))


def layernorm(x, residual, weight, bias, eps):
    """(sum, y, mean, rstd) of rows [n, d]."""
    s = x.astype(np.float64) + (0.0 if residual is None else residual.astype(np.float64))
    mean = np.mean(s, axis=1)
    off = s - mean[:, None]
    rstd = 1.0 / np.sqrt(np.mean(off * off, axis=1) + eps)
    n, d = s.shape
    return s, off * rstd[:, None] * _by_run(weight, n, d, 1.0) + _by_run(bias, n, d, 0.0), mean, rstd


def layernorm_grad(dy, s, weight, mean, rstd, dsum, runs=0):
    """(dx, dweight, dbias) of rows [n, d]; the gradients of `runs` runs (0: [d])."""
    dy, s, r = dy.astype(np.float64), s.astype(np.float64), rstd.astype(np.float64)[:, None]
    rows, d = dy.shape
    n = (s - mean.astype(np.float64)[:, None]) * r
    a = dy * _by_run(weight, rows, d, 1.0)
    dx = (0.0 if dsum is None else dsum.astype(np.float64)) + r * (
        a - np.mean(a, axis=1, keepdims=True) - n * np.mean(a * n, axis=1, keepdims=True))
    shape = (max(runs, 1), -1, d)
    dw, db = (np.sum(v.reshape(shape), axis=1) for v in (dy * n, dy))
    return (dx, dw, db) if runs else (dx, dw[0], db[0])


# ------------------------------------------------------------------ rotary positions over axes
def axis_of_pair(sections, turns):
    """The axis of each pair, in runs or in turn."""
    if not turns:
        return [a for a, n in enumerate(sections) for _ in range(n)]
    left, out = list(sections), []
    while any(left):
        for a, n in enumerate(left):
            if n:
                out.append(a)
                left[a] -= 1
    return out


def axes_table(sections, turns, positions, base, scale, shared):
    """cos and sin [position, pair, 2]."""
    axis = axis_of_pair(sections, turns)
    f = []
    for k, a in enumerate(axis):
        part = k / len(axis) if shared else axis[:k].count(a) / sections[a]
        f.append(scale[a] * base[a] ** -part)
    t = np.asarray(positions, np.float64)[:, None] * np.array(f)
    return np.stack([np.cos(t), np.sin(t)], axis=2)


def rotary_axes(x, table, positions, axis, interleaved, backward=False):
    """x [batch, token, head, dim]; positions [batch, token, axis] (clamped to the table)."""
    y = x.astype(np.float64).copy()
    half = table.shape[1]
    for k in range(half):
        p = np.clip(positions[..., axis[k]], 0, table.shape[0] - 1)
        c, s = table[p, k, 0][..., None], table[p, k, 1][..., None] * (-1.0 if backward else 1.0)
        i, j = (2 * k, 2 * k + 1) if interleaved else (k, k + half)
        a, b = x[..., i].astype(np.float64), x[..., j].astype(np.float64)
        y[..., i], y[..., j] = a * c - b * s, a * s + b * c
    return y


# ------------------------------------------------------------------ dropout
def kept(rows, width, p, seed, stream, step, first_row=0):
    """The mask [rows, width]."""
    per = -(-width // 8)
    q = np.arange(first_row * per, (first_row + rows) * per, dtype=np.uint64)
    c = np.empty((q.size, 4), np.uint32)
    c[:, 0], c[:, 1] = q & np.uint64(0xFFFFFFFF), q >> np.uint64(32)
    c[:, 2], c[:, 3] = stream, (step + 1) % 2**32
    w = philox4x32_10(c, (seed & 0xFFFFFFFF, seed >> 32))
    u = np.empty((q.size, 8), np.int64)
    for e in range(8):
        u[:, e] = (w[:, e // 2] >> np.uint32(16 * (e % 2))) & np.uint32(0xFFFF)
    return u.reshape(rows, 8 * per)[:, :width] >= math.floor(65536 * p + 0.5)


def dropout(x, residual, p, keep):
    under = math.floor(65536 * p + 0.5)
    with np.errstate(divide="ignore", invalid="ignore"):
        y = np.where(keep, x.astype(np.float64) * np.float64(65536) / (65536 - under), 0.0)
    return y if residual is None else y + residual.astype(np.float64)


# ------------------------------------------------------------------ gated product
def activate(g, kind):
    """(act, slope)."""
    with np.errstate(over="ignore"):
        s = 1.0 / (1.0 + np.exp(-g))
    if kind == "silu":
        return g * s, s * (1 + g * (1 - s))
    if kind == "gelu":
        e = 0.5 * (1 + np.vectorize(math.erf, otypes=[float])(g / math.sqrt(2)))
        return g * e, e + g * np.exp(-0.5 * g * g) / math.sqrt(2 * math.pi)
    if kind == "gelu_tanh":
        r = math.sqrt(2 / math.pi)
        t = np.tanh(r * (g + 0.044715 * g**3))
        return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * r * (1 + 3 * 0.044715 * g * g)
    if kind == "sigmoid":
        return s, s * (1 - s)
    return np.maximum(g, 0), (g > 0) * 1.0


def gated(x, w_gate, w_up, kind):
    """(h, gate, up)."""
    x = x.astype(np.float64)
    g, u = x @ w_gate.astype(np.float64), x @ w_up.astype(np.float64)
    return activate(g, kind)[0] * u, g, u


def gated_grad(dh, x, w_gate, w_up, gate, up, kind):
    """(dx, dw_gate, dw_up, h) from gate and up as stored."""
    dh, x, wg, wu, up = (v.astype(np.float64) for v in (dh, x, w_gate, w_up, up))
    a, slope = activate(gate.astype(np.float64), kind)
    dg, du = dh * up * slope, dh * a
    return dg @ wg.T + du @ wu.T, x.T @ dg, x.T @ du, a * up
