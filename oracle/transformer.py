"""Plain float64 forms of the transformer operators, row by row from their definitions.

A query's row is formed from the keys that it sees alone, so nothing that lies in
the others (infinities and NaN among it) can reach the result.
"""
from __future__ import annotations

import math

import numpy as np

__all__ = ["rmsnorm", "rmsnorm_grad", "e4m3_values", "quantise", "rotary_freqs", "rotary_table", "rotary",
           "visible", "attention", "attention_grad"]


# ------------------------------------------------------------------ norm
def rmsnorm(x, residual, weight, eps):
    """(sum, y, rstd) over the last dimension."""
    s = x.astype(np.float64) + (0.0 if residual is None else residual.astype(np.float64))
    rstd = 1.0 / np.sqrt(np.mean(s * s, axis=-1) + eps)
    return s, s * rstd[..., None] * weight.astype(np.float64), rstd


def rmsnorm_grad(dy, s, weight, rstd, dsum):
    """(dx, dweight) of rows [n, d]."""
    dy, s, r = dy.astype(np.float64), s.astype(np.float64), rstd.astype(np.float64)[:, None]
    n = s * r
    a = dy * weight.astype(np.float64)
    dx = (0.0 if dsum is None else dsum.astype(np.float64)) + r * (a - n * np.mean(a * n, axis=1, keepdims=True))
    return dx, np.sum(dy * n, axis=0)


def e4m3_values():
    """The values >= 0 of e4m3, in order: 2^-9 steps up to 2^-6, then eight a power of two up to 448."""
    v = [m * 2.0**-9 for m in range(8)]
    v += [(8 + m) * 2.0**(e - 3) for e in range(-6, 9) for m in range(8)]
    return np.array(v[:-1])


def quantise(y, group):
    """(values / scale before rounding, scale) of rows [n, d] in groups (0: the row)."""
    n, d = y.shape
    g = group or d
    q, scale = np.empty_like(y), np.empty((n, -(-d // g)))
    for i in range(scale.shape[1]):
        part = y[:, i * g:(i + 1) * g]
        scale[:, i] = np.max(np.abs(part), axis=1) / 448.0
        with np.errstate(divide="ignore", invalid="ignore"):
            q[:, i * g:(i + 1) * g] = np.where(scale[:, i:i + 1] > 0, part / scale[:, i:i + 1], 0.0)
    return q, scale


# ------------------------------------------------------------------ rotary
def rotary_freqs(R, base, scaling="plain", factor=1.0, original_length=0.0, low=1.0, high=32.0):
    if scaling == "base" and R > 2:
        base = base * factor ** (R / (R - 2))
    f = np.array([base ** (-2.0 * k / R) for k in range(R // 2)])
    if scaling == "linear":
        f = f / factor
    if scaling == "by_parts":
        g = np.clip((original_length * f / (2 * math.pi) - low) / (high - low), 0.0, 1.0)
        f = g * f + (1 - g) * f / factor
    return f


def rotary_table(freqs, positions, magnitude=1.0):
    a = np.asarray(positions, np.float64)[:, None] * freqs
    return magnitude * np.stack([np.cos(a), np.sin(a)], axis=2)


def rotary(x, table, positions, interleaved, backward=False):
    """x [batch, token, head, dim]; positions [batch, token] (clamped to the table)."""
    y = x.astype(np.float64).copy()
    half = table.shape[1]
    t = table[np.clip(positions, 0, table.shape[0] - 1)][:, :, None]
    c, s = t[..., 0], t[..., 1] * (-1.0 if backward else 1.0)
    for k in range(half):
        i, j = (2 * k, 2 * k + 1) if interleaved else (k, k + half)
        a, b = x[..., i].astype(np.float64), x[..., j].astype(np.float64)
        y[..., i] = a * c[..., k] - b * s[..., k]
        y[..., j] = a * s[..., k] + b * c[..., k]
    return y


# ------------------------------------------------------------------ attention
def visible(i, n, m, causal, window, sinks):
    """Keys that query i of n sees among m."""
    if i >= n:
        return np.zeros(0, np.int64)
    t, j = m - n + i, np.arange(m)
    see = np.ones(m, bool)
    if window:
        see = (np.abs(t - j) < window) | (j < sinks)
    if causal:
        see &= j <= t
    return j[see]


def _each(q, k, q_lens, kv_lens, causal, window, sinks):
    B, n, H, _ = q.shape
    m, K = k.shape[1], k.shape[2]
    for b in range(B):
        nb = n if q_lens is None else min(max(int(q_lens[b]), 0), n)
        mb = m if kv_lens is None else min(max(int(kv_lens[b]), 0), m)
        for i in range(nb):
            j = visible(i, nb, mb, causal, window, sinks)
            if j.size:
                for h in range(H):
                    yield b, i, h, h // (H // K), j


def attention(q, k, v, scale, causal, window=0, sinks=0, q_lens=None, kv_lens=None):
    """(out, lse) of [batch, token, head, dim] tensors."""
    q, k, v = (x.astype(np.float64) for x in (q, k, v))
    out = np.zeros(q.shape)
    lse = np.full((q.shape[0], q.shape[2], q.shape[1]), -np.inf)
    for b, i, h, g, j in _each(q, k, q_lens, kv_lens, causal, window, sinks):
        x = scale * (k[b, j, g] @ q[b, i, h])
        top = np.max(x)
        p = np.exp(x - top)
        out[b, i, h] = p @ v[b, j, g] / p.sum()
        lse[b, h, i] = top + np.log(p.sum())
    return out, lse


def attention_grad(q, k, v, dout, scale, causal, window=0, sinks=0, q_lens=None, kv_lens=None):
    """(dq, dk, dv)."""
    q, k, v, dout = (x.astype(np.float64) for x in (q, k, v, dout))
    dq, dk, dv = np.zeros(q.shape), np.zeros(k.shape), np.zeros(v.shape)
    for b, i, h, g, j in _each(q, k, q_lens, kv_lens, causal, window, sinks):
        x = scale * (k[b, j, g] @ q[b, i, h])
        p = np.exp(x - np.max(x))
        p /= p.sum()
        dp = v[b, j, g] @ dout[b, i, h]
        ds = p * (dp - p @ dp)
        dq[b, i, h] = scale * (ds @ k[b, j, g])
        dk[b, j, g] += scale * ds[:, None] * q[b, i, h]
        dv[b, j, g] += p[:, None] * dout[b, i, h]
    return dq, dk, dv
