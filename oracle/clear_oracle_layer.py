"""fp64 CPU oracle of the operators around the attention call: layer norm, rotary positions, and the gradients of both and of the Q/K
preparation.

TEST INFRASTRUCTURE ONLY: only the tests use it.  It imports nothing from the CUDA package and shares no code with it.  Plain numpy in
fp64, one definition per function; the gradients are the formulas themselves, pinned by the tests to central differences of the forward
definitions and to torch's derivatives.
"""
from __future__ import annotations

import math

import numpy as np


def layer_norm(x, weight, bias, offset, eps):
    """x: [B, N, C]; weight, bias: None, [C] or [B, C].  Returns (y, mean, rstd)."""
    x = np.asarray(x, dtype=np.float64)
    mean = x.mean(-1)
    var = ((x - mean[..., None]) ** 2).mean(-1)
    rstd = 1.0 / np.sqrt(var + eps)
    y = (x - mean[..., None]) * rstd[..., None] * _gain(weight, offset)
    if bias is not None:
        y = y + _rows(bias)
    return y, mean, rstd


def layer_norm_grad(x, dy, weight, mean, rstd, offset, per_batch):
    """(dx, dweight, dbias) for given statistics."""
    x, dy = np.asarray(x, dtype=np.float64), np.asarray(dy, dtype=np.float64)
    r = np.asarray(rstd, dtype=np.float64)[..., None]
    h = (x - np.asarray(mean, dtype=np.float64)[..., None]) * r
    g = dy * _gain(weight, offset)
    dx = r * (g - g.mean(-1, keepdims=True) - h * (g * h).mean(-1, keepdims=True))
    rows = 1 if per_batch else (0, 1)
    return dx, (dy * h).sum(rows), dy.sum(rows)


def _rows(p):
    p = np.asarray(p, dtype=np.float64)
    return p[:, None, :] if p.ndim == 2 else p


def _gain(weight, offset):
    return 1.0 if weight is None else offset + _rows(weight)


def frequencies(dim, theta, scaling="none", factor=1.0, trained=1.0, fast=32.0, slow=1.0):
    out = []
    for k in range(dim // 2):
        base = theta
        if scaling == "ntk" and dim > 2:
            base = theta * factor ** (dim / (dim - 2.0))
        w = base ** (-2.0 * k / dim)
        if scaling == "linear":
            w = w / factor
        if scaling == "parts":
            wavelength = 2.0 * math.pi / w
            turns = trained / wavelength
            if turns <= slow:
                w = w / factor
            elif turns < fast:
                share = (turns - slow) / (fast - slow)
                w = (1.0 - share) * w / factor + share * w
        out.append(w)
    return np.array(out)


def rotate(x, positions, freqs, axes_dim, half, factor, inverse=False):
    """x: [B, H, N, d]; positions: [B or 1, N, axes]; freqs: one per pair."""
    x = np.asarray(x, dtype=np.float64)
    pairs = sum(axes_dim) // 2
    out = x.copy()
    p = 0
    for axis, dim in enumerate(axes_dim):
        for _ in range(dim // 2):
            t = positions[:, :, axis].astype(np.float64)[:, None, :] * float(freqs[p])   # [B or 1, 1, N]
            if inverse:
                t = -t
            i, j = (p, p + pairs) if half else (2 * p, 2 * p + 1)
            out[..., i] = factor * (x[..., i] * np.cos(t) - x[..., j] * np.sin(t))
            out[..., j] = factor * (x[..., i] * np.sin(t) + x[..., j] * np.cos(t))
            p += 1
    return out


def qk_prep_grad(x, dy, gain, positions, axes_dim, theta, ntk, eps, factor):
    """Gradient of factor * rotate(rms_norm(x) * gain) for one tensor: (dx, dgain).  positions: [N, 3]."""
    x = np.asarray(x, dtype=np.float64)
    d = x.shape[-1]
    freqs = np.concatenate([frequencies(n, theta, "ntk", ntk) for n in axes_dim if n] or [np.zeros(0)])
    u = rotate(dy, positions[None], freqs, axes_dim, False, factor, inverse=True)
    g = np.ones(d) if gain is None else np.asarray(gain, dtype=np.float64)
    inv = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    s = u * g
    dx = inv * (s - x * inv ** 2 * (s * x).mean(-1, keepdims=True))
    return dx, (u * x * inv).reshape(-1, d).sum(0)
