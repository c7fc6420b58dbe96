"""Shared plumbing of the GPU tests of the layers beside the normalization: inputs, calls through the binding, and how far a
correct result may be from the oracle's.

Tolerances are per value, from the formats: `unit` is half a unit in the last place of the stored type, at most 2^-8 of a value in bfloat16 (8 significant bits), 2^-24 in
float (24); a sum of n products in 32 bits in any order is off by at most (n + 8) 2^-24 times the sum of their magnitudes (8: the
operations around it), and what is rounded on the way adds its own half unit, carried through with magnitudes."""

from __future__ import annotations

import numpy as np
import torch

from oracle import layers_oracle as Y
from paper_1711_07240_amd import cgbn as L

DEV = "cuda:0"
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
UNIT = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
F = 2.0 ** -24
# the steepest slope of the activations, and of act' (GELU's at 0 is 2 phi(0) = 0.798, SiLU's 0.5)
STEEP = 1.13
# an activation or its slope in float: a few units of its value, and of 1 where it is a difference of such
ACT_ERR = 8 * F


def normal(rng, *shape, scale=1.0, dtype="f32"):
    t = torch.from_numpy((rng.standard_normal(shape) * scale).astype(np.float32)).to(TORCH[dtype])
    return t.to(DEV)


def f64(t):
    return t.detach().cpu().double().numpy()


def near(got, want, tol, what):
    got = f64(got)
    assert got.shape == want.shape, what
    bad = ~(np.abs(got - want) <= tol)
    if bad.any():
        i = np.unravel_index(int(np.argmax(np.where(bad, np.abs(got - want) - tol, -np.inf))), got.shape)
        raise AssertionError(f"{what}: {int(bad.sum())} of {got.size} values off, worst at {i}: {got[i]!r}, oracle {want[i]!r}, "
                             f"allowed {np.broadcast_to(tol, got.shape)[i]:.3g}")


def workspace(nbytes):
    # the bytes behind the workspace are the tests' own: they must stay
    return torch.full((nbytes + 512,), 0x5A, dtype=torch.uint8, device=DEV)


def check_guard(ws, nbytes):
    assert bool((ws[nbytes:] == 0x5A).all()), "written behind the workspace"


class Linear:
    def __init__(self, M, N, K, dtype, seed=0, scale=1.0):
        rng = np.random.default_rng(1000 * seed + M + 7 * N + 31 * K)
        self.size, self.dtype = (M, N, K), dtype
        self.x, self.w = normal(rng, M, K, dtype=dtype, scale=scale), normal(rng, N, K, scale=K ** -0.5, dtype=dtype)
        self.bias, self.residual = normal(rng, N), normal(rng, M, N, dtype=dtype)
        self.dy = normal(rng, M, N, dtype=dtype)
        self.saved = normal(rng, M, N, dtype=dtype)

    def forward(self, act, bias=True, residual=True, save=True):
        M, N, K = self.size
        y = torch.full((M, N), 7.0, dtype=TORCH[self.dtype], device=DEV)
        z = torch.full_like(y, 7.0) if save else None
        nb = L.cgbn_linear_workspace_bytes(M, N, K, self.dtype, False)
        ws = workspace(nb)
        L.cgbn_linear_forward(self.x, self.w, self.bias if bias else None, self.residual if residual else None, M, N, K, act, y, z,
                              self.dtype, ws, nb)
        torch.cuda.synchronize()
        check_guard(ws, nb)
        return y, z

    def check_forward(self, act, bias=True, residual=True, save=True):
        y, z = self.forward(act, bias, residual, save)
        x, w = f64(self.x), f64(self.w)
        b, r = f64(self.bias) if bias else None, f64(self.residual) if residual else None
        want_y, want_z = Y.linear_forward(x, w, b, r, act)
        size = np.abs(x) @ np.abs(w).T + (np.abs(b) if bias else 0) + (np.abs(r) if residual else 0)
        err = (self.size[2] + 8) * F * size
        u = UNIT[self.dtype]
        if save:
            near(z, want_z, err + u * np.abs(want_z) + 1e-37, f"z {self.size} {self.dtype} {act}")
        near(y, want_y, STEEP * err * (1 + u) + u * np.abs(want_y) + ACT_ERR * (1 + np.abs(want_z)) + 1e-37, f"y {self.size} {self.dtype} {act}")

    def backward(self, act, want=("dx", "dw", "dbias", "dresidual")):
        M, N, K = self.size
        dt = TORCH[self.dtype]
        out = {"dx": torch.full((M, K), 7.0, dtype=dt, device=DEV), "dw": torch.full((N, K), 7.0, dtype=dt, device=DEV),
               "dbias": torch.full((N,), 7.0, device=DEV), "dresidual": torch.full((M, N), 7.0, dtype=dt, device=DEV)}
        out = {k: v if k in want else None for k, v in out.items()}
        saved = self.saved.clamp(min=0) if act == "relu" else self.saved
        nb = L.cgbn_linear_workspace_bytes(M, N, K, self.dtype, True)
        ws = workspace(nb)
        L.cgbn_linear_backward(self.dy, self.x, self.w, None if act == "none" else saved, M, N, K, act, out["dx"], out["dw"], out["dbias"],
                               out["dresidual"], self.dtype, ws, nb)
        torch.cuda.synchronize()
        check_guard(ws, nb)
        return out, f64(saved)

    def check_backward(self, act, want=("dx", "dw", "dbias", "dresidual")):
        M, N, K = self.size
        out, saved = self.backward(act, want)
        dy, x, w, u = f64(self.dy), f64(self.x), f64(self.w), UNIT[self.dtype]
        ref = Y.linear_backward(dy, x, w, saved, act)
        dz = np.abs(ref["dz"])
        off = 0.0 if act in ("none", "relu") else ACT_ERR * np.abs(dy) * (1 + np.abs(saved))       # of dz before it is rounded
        stored = off + u * (dz + off)                                                              # ... and after
        name = f"{self.size} {self.dtype} {act}"
        if out["dx"] is not None:
            near(out["dx"], ref["dx"], u * np.abs(ref["dx"]) + (stored + (N + 8) * F * dz) @ np.abs(w) * (1 + u) + 1e-37, "dx " + name)
        if out["dw"] is not None:
            near(out["dw"], ref["dw"], u * np.abs(ref["dw"]) + (stored + (M + 8) * F * dz).T @ np.abs(x) * (1 + u) + 1e-37, "dw " + name)
        if out["dbias"] is not None:
            near(out["dbias"], ref["dbias"], (off + (M + 8) * F * dz).sum(0) + 1e-37, "dbias " + name)
        if out["dresidual"] is not None:
            near(out["dresidual"], ref["dz"], stored + 1e-37, "dresidual " + name)


class Gated:
    def __init__(self, M, F_, K, dtype, seed=0):
        rng = np.random.default_rng(2000 * seed + M + 7 * F_ + 31 * K)
        self.size, self.dtype = (M, F_, K), dtype
        self.x = normal(rng, M, K, dtype=dtype)
        self.wg, self.wu = normal(rng, F_, K, scale=K ** -0.5, dtype=dtype), normal(rng, F_, K, scale=K ** -0.5, dtype=dtype)
        self.dh, self.gate, self.up = (normal(rng, M, F_, dtype=dtype) for _ in range(3))

    def check_forward(self, act, save=True):
        M, F_, K = self.size
        h = torch.full((M, F_), 7.0, dtype=TORCH[self.dtype], device=DEV)
        gate, up = (torch.full_like(h, 7.0), torch.full_like(h, 7.0)) if save else (None, None)
        nb = L.cgbn_gated_workspace_bytes(M, F_, K, self.dtype, False)
        ws = workspace(nb)
        L.cgbn_gated_forward(self.x, self.wg, self.wu, M, F_, K, act, h, gate, up, self.dtype, ws, nb)
        torch.cuda.synchronize()
        check_guard(ws, nb)
        x, wg, wu, u = f64(self.x), f64(self.wg), f64(self.wu), UNIT[self.dtype]
        want, g, up64 = Y.gated_forward(x, wg, wu, act)
        eg, eu = ((K + 8) * F * (np.abs(x) @ np.abs(w).T) for w in (wg, wu))
        name = f"{self.size} {self.dtype} {act}"
        if save:
            near(gate, g, eg + u * np.abs(g) + 1e-37, "gate " + name)
            near(up, up64, eu + u * np.abs(up64) + 1e-37, "up " + name)
        ea = STEEP * eg + ACT_ERR * (1 + np.abs(g))
        a = np.abs(Y.act(g, act))
        near(h, want, u * np.abs(want) + (ea * np.abs(up64) + eu * a + ea * eu) * (1 + u) + 2 * F * np.abs(want) + 1e-37, "h " + name)

    def check_backward(self, act, dx=True, dw=True):
        M, F_, K = self.size
        dt = TORCH[self.dtype]
        out = {"dx": torch.full((M, K), 7.0, dtype=dt, device=DEV) if dx else None}
        for k in ("dwg", "dwu"):
            out[k] = torch.full((F_, K), 7.0, dtype=dt, device=DEV) if dw else None
        nb = L.cgbn_gated_workspace_bytes(M, F_, K, self.dtype, True)
        ws = workspace(nb)
        L.cgbn_gated_backward(self.dh, self.x, self.wg, self.wu, self.gate, self.up, M, F_, K, act, out["dx"], out["dwg"], out["dwu"], self.dtype,
                              ws, nb)
        torch.cuda.synchronize()
        check_guard(ws, nb)
        dh, x, wg, wu, g, up = (f64(t) for t in (self.dh, self.x, self.wg, self.wu, self.gate, self.up))
        u = UNIT[self.dtype]
        ref = Y.gated_backward(dh, x, wg, wu, g, up, act)
        adg, adu = np.abs(ref["dg"]), np.abs(ref["du"])
        exact = act in ("none", "relu")
        og = 4 * F * adg + (0 if exact else ACT_ERR * np.abs(dh * up) * (1 + np.abs(g)))
        ou = 4 * F * adu + (0 if exact else ACT_ERR * np.abs(dh) * (1 + np.abs(g)))
        sg, su = og + u * (adg + og), ou + u * (adu + ou)
        name = f"{self.size} {self.dtype} {act}"
        if dx:
            tol = (sg + (2 * F_ + 8) * F * adg) @ np.abs(wg) + (su + (2 * F_ + 8) * F * adu) @ np.abs(wu)
            near(out["dx"], ref["dx"], u * np.abs(ref["dx"]) + tol * (1 + u) + 1e-37, "dx " + name)
        if dw:
            near(out["dwg"], ref["dwg"], u * np.abs(ref["dwg"]) + (sg + (M + 8) * F * adg).T @ np.abs(x) * (1 + u) + 1e-37, "dwg " + name)
            near(out["dwu"], ref["dwu"], u * np.abs(ref["dwu"]) + (su + (M + 8) * F * adu).T @ np.abs(x) * (1 + u) + 1e-37, "dwu " + name)
