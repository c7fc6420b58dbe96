"""Float64 definitions of the serving operators: frequencies and rotation by position, the plan of a paged cache, the store of
keys and values in pages, attention over a shared prefix and a request's own pages.  Test infrastructure: plain numpy and loops, written
from the formulas, sharing no code with the kernels.

    frequencies  f[i] = base^(-2i/R); f / factor; base factor^(R/(R-2)) for base; g f + (1 - g) f / factor by parts
    rotation     (a, b) -> m (a cos t - b sin t, b cos t + a sin t), t = position f[i]; backward with -t
    plan         request by request, token by token, page by page, in order
    attention    o = sum of softmax(scale q.k) v over the keys a row sees, lse = log sum exp(scale q.k)
"""

from __future__ import annotations

import math

import numpy as np


def frequencies(R, base, scaling="none", factor=1.0, trained=0.0, fast=0.0, slow=0.0):
    found = []
    for i in range(R // 2):
        f = base ** (-2.0 * i / R)
        if scaling == "positions":
            f = f / factor
        elif scaling == "base" and R > 2:
            f = (base * factor ** (R / (R - 2.0))) ** (-2.0 * i / R)
        elif scaling == "parts":
            turns = trained * f / (2.0 * math.pi)
            g = min(max((turns - slow) / (fast - slow), 0.0), 1.0)
            f = g * f + (1.0 - g) * f / factor
        found.append(f)
    return np.array(found, np.float64)


def rotate(x, heads, D, R, style, positions, freq, magnitude, back=False):
    """x [T, heads * D]"""
    x = np.asarray(x, np.float64).reshape(-1, heads, D)
    y = x.copy()
    t = np.asarray(positions, np.float64)[:, None] * np.asarray(freq)[None]
    c, s = magnitude * np.cos(t)[:, None], magnitude * np.sin(-t if back else t)[:, None]
    first = np.arange(R // 2) if style == "halves" else np.arange(0, R, 2)
    second = first + (R // 2 if style == "halves" else 1)
    a, b = x[..., first], x[..., second]
    y[..., first], y[..., second] = a * c - b * s, b * c + a * s
    return y.reshape(x.shape[0], -1)


def plan(have, fresh, before, free_pages, taken, table, max_pages, pages, page, T):
    """-> rows, lengths, table, slots, positions, counts"""
    table = np.array(table, np.int64)
    rows, lengths, slots, positions = [0], [], [-1] * T, [0] * T
    taken = min(max(int(taken), 0), len(free_pages))
    left_out = 0
    for b, (had, more) in enumerate(zip(have, fresh)):
        had, more = min(max(int(had), 0), max_pages * page), max(int(more), 0)
        held = -(-had // page)
        for j in range(more):
            key, row = had + j, rows[-1] + j
            at = key // page
            if row >= T:
                left_out += more - j
                more = j
                break
            positions[row] = before + key
            if at >= held and at < max_pages and key % page == 0:
                table[b, at] = -1
                if taken < len(free_pages):
                    table[b, at] = free_pages[taken] if 0 <= free_pages[taken] < pages else -1
                    taken += 1
            if at < max_pages and 0 <= table[b, at] < pages:
                slots[row] = int(table[b, at]) * page + key % page
            else:
                left_out += 1
        rows.append(rows[-1] + more)
        lengths.append(had + more)
    return rows, lengths, table, slots, positions, [taken, min(left_out, 2 ** 31 - 1)]


def store(x, heads, D, slots, pool):
    """x [T, heads * D], pool [pages, heads, page, D]"""
    pool = np.array(pool)
    page = pool.shape[2]
    for row, slot in zip(np.asarray(x).reshape(-1, heads, D), slots):
        if 0 <= slot < pool.shape[0] * page:
            pool[slot // page, :, slot % page] = row
    return pool


def attention(q, k, v, scale):
    """One row: q [D], k and v [n, D] of the keys it sees -> o, lse, weights"""
    if len(k) == 0:
        return np.zeros(q.shape), -np.inf, np.zeros(0)
    s = (k @ q) * scale
    top = s.max()
    p = np.exp(s - top)
    return (p / p.sum()) @ v, top + np.log(p.sum()), p / p.sum()
