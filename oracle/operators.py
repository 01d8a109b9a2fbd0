"""Plain 64-bit references of the 4-bit format, its products and sampling
(test infrastructure; numpy, independent of the kernels' layout and steps)."""

from __future__ import annotations

import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def mx4_values(x):
    """x [..][K] (float64 array of float32 or bf16 values) rounded to the
    4-bit format along its last axis: every element goes to the nearest grid
    value by distance, of two equally near to the one of even code."""
    x = np.asarray(x, np.float64)
    out = np.empty_like(x)
    K = x.shape[-1]
    for k in range(0, K, 32):
        b = x[..., k:k + 32]
        top = np.abs(b).max(axis=-1, keepdims=True)
        finite = np.isfinite(top)
        _, e = np.frexp(np.where(finite, top, 1.0))
        e = np.where(top > 0, e - 1, -127) - 2
        scale = np.ldexp(1.0, np.maximum(e, -127))
        a = np.abs(np.where(finite, b, 0.0)) / scale
        d = np.abs(a[..., None] - GRID)
        near = d == d.min(axis=-1, keepdims=True)
        even = near & (np.arange(8) % 2 == 0)
        code = np.where(even.any(-1), even.argmax(-1), near.argmax(-1))
        v = GRID[code] * scale
        out[..., k:k + 32] = np.where(finite, np.where(np.signbit(b), -v, v), np.nan)
    return out


def mx4_scale_bytes(x):
    """The scale byte of every block of 32 of the last axis."""
    x = np.asarray(x, np.float64)
    out = []
    for k in range(0, x.shape[-1], 32):
        top = np.abs(x[..., k:k + 32]).max(axis=-1)
        _, e = np.frexp(np.where(np.isfinite(top), top, 1.0))
        out.append(np.where(np.isfinite(top), np.where(top > 0, np.maximum(e - 1 + 125, 0), 0), 255))
    return np.stack(out, axis=-1) if out else np.zeros((*x.shape[:-1], 0), np.int64)


def order(z):
    """Token indices in descending order of the logits, the lower index first
    among equal ones (the two zeros are equal)."""
    z = np.asarray(z, np.float64) + 0.0
    return np.lexsort((np.arange(z.size), -z))


def mass_of(w):
    """The masses of float32 weights: the whole part of w 2^31 + 1/2, rounded to
    float32 (both terms and the sum before its rounding are exact in float64
    wherever the result is not 0)."""
    return np.floor((np.asarray(w, np.float32).astype(np.float64) * 2.0 ** 31 + 0.5).astype(np.float32)).astype(np.int64)


def sample_masses(z, temperature):
    """Whole-number masses of one row's tokens, and their weights: the scaled
    logits in float32, operation by operation, the power in float64, rounded to
    float32."""
    z = np.asarray(z, np.float32)
    top = z.max()
    with np.errstate(over="ignore", invalid="ignore", divide="ignore"):
        c = (np.float32(1.0) / np.float32(temperature)) * np.float32(np.log2(np.e))
        t = np.where(z == top, np.float32(0), (z - top) * c).astype(np.float64)
        w = np.where(z == -np.inf, 0.0, np.exp2(np.where(np.isnan(t), -np.inf, t))).astype(np.float32)
    return mass_of(w), w


def sample(z, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """One row: (token, mass, kept mass, mass before it, order, kept count),
    in Python's whole numbers; token -1 for a row of NaN or of -inf alone."""
    z = np.asarray(z, np.float32)
    if np.isnan(z).any() or z.max() == -np.inf:
        return -1, 0, 0, 0, None, 0
    with np.errstate(over="ignore", divide="ignore"):
        c = (np.float32(1.0) / np.float32(temperature)) * np.float32(np.log2(np.e))
    idx = order(z)
    if not temperature > 0 or np.isinf(c):
        return int(idx[0]), 1, 1, 0, idx, 1
    mass, w = sample_masses(z, temperature)
    mass, w = [int(v) for v in mass[idx]], w[idx]
    n = top_k if 0 < top_k < z.size else z.size
    total = sum(mass[:n])
    keep, before = 0, 0
    limit = max(1, int(np.ceil(np.float64(np.float32(top_p)) * total))) if top_p < 1 else total
    while keep < n and before < limit:
        before += mass[keep]
        keep += 1
    floor = min(np.float32(min_p), np.float32(1))
    while keep > 0 and w[keep - 1] < floor:
        keep -= 1
    total = sum(mass[:keep])
    u = np.float64(np.float32(u))
    target = min(max(int(u * total), 0) if u == u else 0, total - 1)
    before = 0
    for i in range(keep):
        if before + mass[i] > target:
            return int(idx[i]), mass[i], total, before, idx, keep
        before += mass[i]
    raise AssertionError("no token holds the target")
