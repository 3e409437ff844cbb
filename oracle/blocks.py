"""Oracle of the state-space block's operators: their definitions in fp64, on the CPU, one
sequence and one token at a time, next to the sum of the magnitudes of what was added up (for
error bounds).  Shares nothing with the library."""
from __future__ import annotations

import numpy as np


def unpack(codes, k):
    """Codes [n, (k + 1) // 2] -> integers in -8..7 [n, k]."""
    q = np.stack((codes & 15, codes >> 4), axis=2).reshape(codes.shape[0], -1)[:, :k].astype(np.int64)
    return np.where(q > 7, q - 16, q)


def dense(x, codes, scales, k, group, bias=None):
    """(y before the activation, sum of magnitudes), both [m, n]."""
    w = unpack(codes, k) * np.repeat(scales.astype(np.float64), group, axis=1)[:, :k]
    b = np.zeros(w.shape[0]) if bias is None else bias.astype(np.float64)
    return x @ w.T + b, np.abs(x) @ np.abs(w).T + np.abs(b)


def act(v, kind):
    if kind == "relu":
        return np.maximum(v, 0)
    if kind == "relu6":
        return np.clip(v, 0, 6)
    if kind in ("hswish", "hsigmoid"):
        s = np.clip(v + 3, 0, 6) / 6
        return v * s if kind == "hswish" else s
    if kind in ("silu", "sigmoid"):
        with np.errstate(over="ignore"):
            s = 1 / (1 + np.exp(-v))
        return v * s if kind == "silu" else s
    return v


def row_norm(v, kind, eps, weight, bias):
    if kind == "layer":
        v = v - v.mean(axis=1, keepdims=True)
    v = v / np.sqrt((v * v).mean(axis=1, keepdims=True) + eps) * weight
    return v if bias is None else v + bias


def block_norm(y, residual=None, gate=None, per=1, kind="rms", eps=1e-5, post=None, post_bias=None, pre=None,
               pre_bias=None, scale=None, gate_act="none", at="after"):
    """(total, normed or None)."""
    t = 0.0
    if y is not None:
        g = None if gate is None else act(gate, gate_act)[np.arange(y.shape[0]) // per]
        t = y * g if g is not None and at == "before" else y
        if post is not None:
            t = row_norm(t, kind, eps, post, post_bias)
        if g is not None and at == "after":
            t = t * g
        if scale is not None:
            t = t * scale
    total = t if residual is None else residual + t
    return total, None if pre is None else row_norm(total, kind, eps, pre, pre_bias)


def conv(x, weight, bias, silu, kept=None, pos=0):
    """One sequence [len, c]: (y, sum of magnitudes, kept after)."""
    n, c = x.shape
    w = weight.shape[1]
    y, mag = np.zeros((n, c)), np.zeros((n, c))
    for t in range(n):
        a = np.zeros(c) if bias is None else bias.astype(np.float64).copy()
        m = np.abs(a)
        for back in range(w):
            if t - back >= 0:
                v = x[t - back]
            elif kept is not None and pos + t - back >= 0:
                v = kept[(pos + t - back) % w]
            else:
                continue
            a += weight[:, w - 1 - back] * v
            m += np.abs(weight[:, w - 1 - back] * v)
        y[t], mag[t] = (act(a, "silu") if silu else a), m
    if kept is not None:
        kept = kept.copy()
        for t in range(max(0, n - w), n):
            kept[(pos + t) % w] = x[t]
    return y, mag, kept


def softplus(v):
    return np.maximum(v, 0) + np.log1p(np.exp(-np.abs(v)))


def scan(xbc, dt, sizes, a, d, dt_bias, state):
    """One sequence: (y [len, heads * head_dim], its magnitudes, state, its magnitudes)."""
    h, p, g, n = sizes
    head = np.arange(h) // (h // g)
    s, ms = state.astype(np.float64).copy(), np.abs(state).astype(np.float64)
    y, my = np.zeros((len(xbc), h * p)), np.zeros((len(xbc), h * p))
    for t in range(len(xbc)):
        x = xbc[t, : h * p].reshape(h, p)
        b = xbc[t, h * p: h * p + g * n].reshape(g, n)[head]
        c = xbc[t, h * p + g * n:].reshape(g, n)[head]
        dd = softplus(dt[t] + (0 if dt_bias is None else dt_bias))
        e = np.exp(dd * a)[:, None, None]
        add = (dd[:, None] * x)[:, :, None] * b[:, None, :]
        s, ms = e * s + add, e * ms + np.abs(add)
        skip = 0 if d is None else d[:, None] * x
        y[t] = ((s * c[:, None, :]).sum(2) + skip).reshape(-1)
        my[t] = ((ms * np.abs(c)[:, None, :]).sum(2) + np.abs(skip)).reshape(-1)
    return y, my, s, ms
