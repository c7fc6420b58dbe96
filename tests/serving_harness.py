"""Shared plumbing of the GPU tests of the serving operators: inputs, calls through the binding, and how far a correct result may be
from the oracle's.  Units and `near` are those of layers_harness.py."""

from __future__ import annotations

import numpy as np
import torch

from layers_harness import DEV, F, TORCH, UNIT, check_guard, f64, near, workspace
from oracle import serving_oracle as V
from paper_1711_07240_amd import cgbn as L


def ints(values):
    return torch.tensor(np.asarray(values, np.int32), device=DEV)


class Attention:
    """`fresh`: new tokens of each request, `lengths`: its tokens in all.  Places that nobody may look at hold NaN; tables name
    pages that are not there where they are not read."""

    def __init__(self, dtype, fresh, lengths, prefix, page, Hq, Hk, D, seed=0, spread=1.0, pad=0, stride=0, extra=2):
        rng = np.random.default_rng(seed + 7 * sum(lengths) + 31 * prefix + D)
        self.dtype, self.fresh, self.lengths, self.prefix, self.page = dtype, list(fresh), list(lengths), prefix, page
        self.Hq, self.Hk, self.D, self.B, self.pad, self.ld = Hq, Hk, D, len(fresh), pad, Hq * D + stride
        self.T = sum(fresh) + pad
        self.rows = np.concatenate([[0], np.cumsum(fresh)]).astype(np.int32)
        shared = -(-prefix // page)
        need = [-(-n // page) for n in lengths]
        self.pages = shared + sum(need) + 1
        order = rng.permutation(self.pages)
        self.prefix_table = order[:shared].astype(np.int32)
        self.most = max(need + [0]) + extra
        self.table = rng.choice([-1, self.pages, -5, 1 << 30], (self.B, self.most)).astype(np.int32)
        at = shared
        k, v = (np.full((self.pages, Hk, page, D), np.nan, np.float32) for _ in range(2))
        self.keys, self.values = [], []

        def fill(ids, n):
            kk, vv = (torch.from_numpy(rng.standard_normal((Hk, n, D)).astype(np.float32)).to(TORCH[dtype]).float().numpy() for _ in range(2))
            for i, p in enumerate(ids):
                part = slice(i * page, min(n, (i + 1) * page))
                k[p, :, :part.stop - part.start], v[p, :, :part.stop - part.start] = kk[:, part], vv[:, part]
            return kk.astype(np.float64), vv.astype(np.float64)

        self.shared = fill(self.prefix_table, prefix)
        self.own = []
        for b, n in enumerate(need):
            self.table[b, :n] = order[at:at + n]
            self.own.append(fill(order[at:at + n], self.lengths[b]))
            at += n
        q = rng.standard_normal((self.T, self.ld)).astype(np.float32) * spread
        self.q = torch.from_numpy(q).to(TORCH[dtype]).to(DEV)
        self.k, self.v = (torch.from_numpy(t).to(TORCH[dtype]).to(DEV) for t in (k, v))
        self.scale = D ** -0.5

    def place(self, b, key):
        """Of one of request b's keys: page, token in page."""
        return int(self.table[b, key // self.page]), key % self.page

    def call(self, single=False, lse=True, stream=None, ws=None, out=None):
        out = torch.full((self.T, self.ld), 7.0, dtype=TORCH[self.dtype], device=DEV) if out is None else out
        total = torch.full((self.T, self.Hq), 7.0, device=DEV) if lse else None
        nb = L.cgbn_prefix_attention_workspace_bytes(self.T, self.B, self.Hq, self.Hk, self.D, self.prefix, self.most * self.page, self.dtype)
        own = ws is None
        ws = workspace(nb) if own else ws
        self.keep = (ints(self.rows), ints(self.lengths), ints(self.prefix_table), ints(self.table))
        rows, lengths, shared, table = self.keep
        L.cgbn_prefix_attention(self.q, self.ld, self.T, self.B, None if single else rows, lengths, self.Hq, self.Hk, self.D, self.scale, self.k, self.v,
                                self.pages, self.page, shared, self.prefix, table, self.most, out, self.ld, total, self.dtype, ws, nb, stream)
        torch.cuda.synchronize()
        if own:
            check_guard(ws, nb)
        return out, total

    def row(self, b, j, h):
        """The definition's result of one row and how far a right one may be from it.

        A score is off by (D + 8) 2^-24 of its terms' sizes, and by 2^-24 of it and of the largest score four times (scaled, subtracted,
        the exponential); its weight by that, relatively, and by a rounding to the type where that is bfloat16; sums of n by n 2^-24."""
        own_k, own_v = self.own[b]
        sees = min(max(self.lengths[b] - self.fresh[b] + j + 1, 0), self.lengths[b])
        head = h // (self.Hq // self.Hk)
        k = np.concatenate([self.shared[0][head], own_k[head, :sees]])
        v = np.concatenate([self.shared[1][head], own_v[head, :sees]])
        q = f64(self.q[self.rows[b] + j, h * self.D:(h + 1) * self.D])
        with np.errstate(invalid="ignore"):
            o, lse, w = V.attention(q, k, v, self.scale)
            if len(k) == 0:
                return o, lse, np.zeros(self.D), 0.0
            s = np.abs(k @ q) * abs(self.scale)
            ep = (self.D + 8) * F * (np.abs(k) @ np.abs(q)) * abs(self.scale) + 4 * F * (s + s.max() + 1)
            n = len(k) + 64
            off = float(w @ ep) + n * F
            rounding = UNIT["bf16"] if self.dtype == "bf16" else 0.0
            tol = (w * (ep + rounding + n * F)) @ np.abs(v) + off * np.abs(o)
        return o, lse, tol * (1 + UNIT[self.dtype]) + UNIT[self.dtype] * np.abs(o) + 1e-37, off + 4 * F * (1 + abs(lse))

    def check(self, out, total, rows=None):
        got, sums = f64(out), None if total is None else f64(total)
        name = f"{self.dtype} fresh {self.fresh[:9]} lengths {self.lengths[:9]} prefix {self.prefix} page {self.page} heads {self.Hq}/{self.Hk} of {self.D}"
        for b in range(self.B):
            for j in (range(self.fresh[b]) if rows is None else [r for r in rows if r < self.fresh[b]]):
                t = self.rows[b] + j
                for h in range(self.Hq):
                    o, lse, tol, tol_lse = self.row(b, j, h)
                    near(torch.from_numpy(got[t, h * self.D:(h + 1) * self.D]), o, tol, f"row {b}, {j}, head {h}: {name}")
                    if sums is not None:
                        assert sums[t, h] == lse or abs(sums[t, h] - lse) <= tol_lse, (b, j, h, sums[t, h], lse, tol_lse, name)
        # what is no result stays as it was
        assert bool((out[:, self.Hq * self.D:] == 7.0).all()) and bool((out[sum(self.fresh):] == 7.0).all())
        if total is not None:
            assert bool((total[sum(self.fresh):] == 7.0).all())
