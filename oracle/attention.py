"""Oracle of the attention layer's operators: their definitions in fp64 on the CPU, one sequence and one
token at a time, next to the magnitudes that error bounds need.  Shares nothing with the library."""
from __future__ import annotations

import math
from fractions import Fraction

import numpy as np

TWO_PI = Fraction("6.28318530717958647692528676655900576839433879875021164194988918461563281")


def angle(pos, f):
    """pos * f modulo one turn, exactly but for 2 pi's 70 digits."""
    return float((Fraction(int(pos)) * Fraction(float(f))) % TWO_PI)


def head_rope(x, pos, freq, axes=None, norm="rms", eps=1e-6, weight=None, interleaved=False):
    """x [tokens, heads, dim], pos [tokens, axes] -> (y, the same without rotation)."""
    x = x.astype(np.float64)
    if norm == "layer":
        x = x - x.mean(axis=2, keepdims=True)
    if norm != "none":
        x = x / np.sqrt((x * x).mean(axis=2, keepdims=True) + eps)
        if weight is not None:
            x = x * weight.astype(np.float64)
    y = x.copy()
    n = len(freq)
    for t in range(x.shape[0]):
        for i in range(n):
            a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + n)
            th = angle(pos[t, axes[i] if axes is not None else 0], freq[i])
            c, s = math.cos(th), math.sin(th)
            y[t, :, a], y[t, :, b] = x[t, :, a] * c - x[t, :, b] * s, x[t, :, a] * s + x[t, :, b] * c
    return y, x


def codes(v):
    """(codes, scales) of fp32 rows [..., dim], as the library defines them: divisions in fp32."""
    v = v.astype(np.float32)
    top = np.abs(v).max(axis=-1)
    with np.errstate(all="ignore"):
        s = np.where(top > 0, np.maximum(top / np.float32(127), np.float32(2.0 ** -149)), np.float32(1)).astype(np.float32)
        bad = ~np.isfinite(v).all(axis=-1)
        c = np.where(bad[..., None], 0, np.clip(np.rint(v / s[..., None]), -127, 127)).astype(np.int8)
    return c, np.where(bad, np.float32(np.nan), s)


def place(table, slot, at, page, pages):
    """(page, place) of a position, or None."""
    if slot < 0 or slot >= table.shape[0] or at // page >= table.shape[1]:
        return None
    n = int(table[slot, at // page])
    return (n, at % page) if 0 <= n < pages else None


def attend(q, k, v, table, offsets, pos, scale, max_context=None, slots=None, dims=None):
    """q [tokens, q_heads, dim], k and v [pages, heads, page, dim] fp64 (codes times scales).

    (y, magnitude of the values averaged, error of a score of m roundings divided by m 2^-24, keys seen)"""
    pages, heads, page, dim = k.shape
    group = q.shape[1] // heads
    y, mag = np.zeros(q.shape), np.zeros(q.shape)
    es, seen = np.zeros(q.shape[:2]), np.zeros(q.shape[:2], dtype=np.int64)
    for b in range(len(offsets) - 1):
        slot = b if slots is None else slots[b]
        for t in range(offsets[b], offsets[b + 1]):
            at = pos[b] + t - offsets[b]
            keys = [place(table, slot, j, page, pages) for j in range(at + 1) if max_context is None or j < max_context]
            keys = [p for p in keys if p is not None]
            if not keys:
                continue
            ids, at_ = np.array([p[0] for p in keys]), np.array([p[1] for p in keys])
            for h in range(q.shape[1]):
                kk, vv = k[ids, h // group, at_], v[ids, h // group, at_]
                s = kk @ q[t, h] * scale
                m = s.max()
                if m == -np.inf:
                    continue
                w = np.exp(s - m)
                y[t, h], mag[t, h] = w @ vv / w.sum(), w @ np.abs(vv) / w.sum()
                es[t, h] = (np.abs(kk) @ np.abs(q[t, h])).max() * abs(scale)
                seen[t, h] = len(keys)
    return y, mag, es, seen


def verify(target, draft, tokens, accept, sample, offsets, width):
    """(out [batch, width], count) by exact arithmetic on probabilities in units of 2^-60."""
    unit = 1 << 60

    def fixed(row):
        row = np.where(np.isnan(row), 0.0, np.clip(row, 0.0, 1.0))
        return [round(Fraction(float(x)) * unit) for x in row]

    batch = len(offsets) - 1
    out, count = np.full((batch, width), -1, dtype=np.int32), np.zeros(batch, dtype=np.int32)
    for b in range(batch):
        first, n = offsets[b], offsets[b + 1] - offsets[b]
        for i in range(n + 1):
            p, w = target[first + b + i], None
            if i < n:
                x = tokens[first + i]
                if 0 <= x < p.shape[0]:
                    clean = [float(np.clip(np.nan_to_num(r[x]), 0, 1)) for r in (draft[first + i], p)]
                    if Fraction(float(accept[first + i])) * Fraction(clean[0]) < Fraction(clean[1]):
                        out[b, i] = x
                        continue
                w = [max(a - c, 0) for a, c in zip(fixed(p), fixed(draft[first + i]))]
            if w is None or not any(w):
                w = fixed(p)
            bar, c, at = Fraction(float(sample[b])) * sum(w), 0, len(w) - 1
            for j, x in enumerate(w):
                c += x
                if c > bar:
                    at = j
                    break
            out[b, i], count[b] = at, i
            break
    return out, count
