"""Float64 definitions of the layers beside the normalization: linear with bias, residual and activation, the gated
feed-forward block, the per-head norm with rotation; forward and backward.  Test infrastructure: plain numpy, written from
the formulas, sharing no code with the kernels.

    linear     z = x W^T + bias + residual, y = act(z)
               dz = dy act'(z), dx = dz W, dW = dz^T x, dbias = sum of dz over rows, dresidual = dz
    gated      g = x Wg^T, u = x Wu^T, h = act(g) u
               dg = dh u act'(g), du = dh act(g), dx = dg Wg + du Wu, dWg = dg^T x, dWu = du^T x
    head norm  n = w x / sqrt(mean(x^2) + eps); the first R values turned by the position's angles
"""

from __future__ import annotations

import math

import numpy as np

_erf = np.vectorize(math.erf, otypes=[np.float64])


def phi(z):
    """Distribution function of the standard normal."""
    return 0.5 * (1.0 + _erf(z / math.sqrt(2.0))) if z.size else np.zeros_like(z)


def sigmoid(z):
    return np.where(z >= 0, 1.0 / (1.0 + np.exp(-np.abs(z))), np.exp(-np.abs(z)) / (1.0 + np.exp(-np.abs(z))))


def act(z, name):
    z = np.asarray(z, np.float64)
    if name == "none":
        return z.copy()
    if name == "relu":
        return np.maximum(z, 0.0)
    if name == "gelu":
        return z * phi(z)
    if name == "silu":
        return z * sigmoid(z)
    raise ValueError(name)


def act_slope(z, name):
    z = np.asarray(z, np.float64)
    if name == "none":
        return np.ones_like(z)
    if name == "relu":
        return (z > 0).astype(np.float64)
    if name == "gelu":
        return phi(z) + z * np.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    if name == "silu":
        s = sigmoid(z)
        return s * (1.0 + z * (1.0 - s))
    raise ValueError(name)


def linear_forward(x, w, bias, residual, name):
    z = x @ w.T
    if bias is not None:
        z = z + bias
    if residual is not None:
        z = z + residual
    return act(z, name), z


def linear_backward(dy, x, w, saved, name):
    """`saved`: y for relu, z for gelu and silu (relu's slope is the same at y as at z)."""
    dz = dy * act_slope(saved, name) if name != "none" else dy
    return dict(dx=dz @ w, dw=dz.T @ x, dbias=dz.sum(0), dresidual=dz, dz=dz)


def gated_forward(x, wg, wu, name):
    g, u = x @ wg.T, x @ wu.T
    return act(g, name) * u, g, u


def gated_backward(dh, x, wg, wu, g, u, name):
    dg, du = dh * u * act_slope(g, name), dh * act(g, name)
    return dict(dx=dg @ wg + du @ wu, dwg=dg.T @ x, dwu=du.T @ x, dg=dg, du=du)


def pair_indices(R, style):
    i = np.arange(R // 2)
    return (i, i + R // 2) if style == "halves" else (2 * i, 2 * i + 1)


def rotate(x, positions, cos, sin, R, style, sign=1.0):
    """x [T, H, D]; cos, sin [rows, R / 2]."""
    y = x.copy()
    if R:
        first, second = pair_indices(R, style)
        c, s = cos[positions][:, None, :], sign * sin[positions][:, None, :]
        y[..., first] = x[..., first] * c - x[..., second] * s
        y[..., second] = x[..., second] * c + x[..., first] * s
    return y


def head_norm_forward(x, w, eps, positions, cos, sin, R, style):
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    return rotate(x * r * w, positions, cos, sin, R, style)


def head_norm_backward(dy, x, w, eps, positions, cos, sin, R, style):
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    e = rotate(dy, positions, cos, sin, R, style, -1.0)
    n, t = x * r, e * w
    return r * (t - n * (t * n).mean(-1, keepdims=True)), (e * n).sum((0, 1))
