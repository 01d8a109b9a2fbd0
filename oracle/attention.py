"""Plain 64-bit references of attention over paged 4-bit caches: heads normed
and rotated with their gradients, attention, and the pages' tables (test
infrastructure; numpy, independent of the kernels' layout and steps)."""

from __future__ import annotations

import numpy as np

from .operators import mx4_values

U32 = 2.0 ** -24  # half a step of float32, relative


def turn(x, positions, freqs, interleaved, back=False, size=False):
    """The first 2 len(freqs) elements of x [..][T][H][D] turned; positions
    [T] or [..][T].  With `size`, every term's magnitude in place of the term."""
    x = np.asarray(x, np.float64)
    out = np.abs(x) if size else x.copy()
    half = len(freqs)
    a = np.asarray(positions, np.float64)[..., None, None] * np.asarray(freqs, np.float64)
    c, s = np.cos(a), np.sin(a) * (-1 if back else 1)
    for i in range(half):
        p, q = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        u, v, ci, si = x[..., p], x[..., q], c[..., i], s[..., i]
        if size:
            out[..., p], out[..., q] = abs(u * ci) + abs(v * si), abs(u * si) + abs(v * ci)
        else:
            out[..., p], out[..., q] = u * ci - v * si, u * si + v * ci
    return out


def _weight(w):
    w = np.asarray(w, np.float64)
    return w if w.ndim == 1 else w[:, None, None, :]


def rotate_heads(x, w, positions, freqs, eps, interleaved):
    """(y, what bounds the float32 error of y: the magnitudes of its terms)."""
    x = np.asarray(x, np.float64)
    if w is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * _weight(w)
    return turn(x, positions, freqs, interleaved), turn(x, positions, freqs, interleaved, size=True)


def rotate_heads_grads(dy, x, w, positions, freqs, eps, interleaved):
    """(dx, dw, magnitudes of dx's terms, of dw's)."""
    g = turn(dy, positions, freqs, interleaved, back=True)
    size = turn(dy, positions, freqs, interleaved, back=True, size=True)
    if w is None:
        return g, None, size, None
    x, shape = np.asarray(x, np.float64), np.shape(w)
    r = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    n, gw, sw = x * r, g * _weight(w), size * abs(_weight(w))
    dx = r * (gw - n * (gw * n).mean(-1, keepdims=True))
    bound = r * (sw + abs(n) * (sw * abs(n)).mean(-1, keepdims=True))
    axes = tuple(range(x.ndim - 1)) if len(shape) == 1 else (-3, -2)
    return dx, (g * n).sum(axes), bound, (size * abs(n)).sum(axes)


def attend(q, k, v, scale, window=0):
    """One sequence: q [n][HQ][D], k and v [L][HK][D], the values that the cache
    holds; (out, bound): out [n][HQ][D] and what a float32 computation may be
    off by, before the rounding to the output's type, where a weight is held
    as the sum of three bf16 numbers (see `weight_error` for fewer).

    A sum of n terms in any order with additions that are off by 2^-23 at most
    (truncation) is off by (n - 1) 2^-23 of the sum of their magnitudes; the
    float32 exponent scale log2(e) (s - m) is off by 2^-24 (|m| + |s - m| + 2
    |s - m|) scale log2(e) for its operations, and the power by 2 2^-23."""
    q, k, v = (np.asarray(a, np.float64) for a in (q, k, v))
    n, HQ, D = q.shape
    L, HK = k.shape[:2]
    out, bound = np.zeros(q.shape), np.zeros(q.shape)
    where = np.arange(L)
    for i in range(n):
        at = L - n + i
        seen = (where <= at) & ((where > at - window) if window > 0 else True)
        if not seen.any():
            continue
        for h in range(HQ):
            kk, vv = k[seen, h // (HQ // HK)], v[seen, h // (HQ // HK)]
            with np.errstate(invalid="ignore"):
                s = scale * (kk @ q[i, h])
                if np.all(s == -np.inf):
                    continue
                ds = scale * 2.0 ** -23 * (np.count_nonzero(kk * q[i, h], axis=1) * 3) * (abs(kk) @ abs(q[i, h]))
                p = np.exp(s - s.max())
                total = p.sum()
                o = (p @ vv) / total
                # The reference may be another row's maximum, up to 8 powers of two below.
                e = ds + ds.max() + U32 * (abs(s).max() + 4 * (s.max() - s) + 16) + 2.0 ** -22
                e = np.where(p > 0, e, 0)
                terms = 3 * len(p) * 2.0 ** -23
                out[i, h] = o
                bound[i, h] = 1.01 * ((p * (e + terms)) @ abs(vv) / total + abs(o) * ((p @ e) / total + terms)) + \
                    2.0 ** -124 * abs(vv).sum(0)
    return out, bound


def weight_error(q, k, v, scale, window=0, rel=2.0 ** -17):
    """What weights that are off by `rel` of themselves add to the bound:
    rel sum_j p_j |v_j|."""
    out, _ = attend(q, k, abs(np.asarray(v, np.float64)), scale, window)
    return rel * out


def extend_pages(tables, lengths, counts, free, page, tokens):
    """The rule request by request, on Python's lists; `free` is the stack."""
    tables = [list(t) for t in tables]
    lengths, free = list(lengths), list(free)
    starts, positions, slots = [0], [], []
    asked_pages = asked_tokens = 0
    room = len(free)
    for b, count in enumerate(counts):
        held, count = max(lengths[b], 0), max(count, 0)
        have, want = -(-held // page), -(-(held + count) // page)
        if want > len(tables[b]):
            count = 0
        else:
            asked_pages += want - have
            asked_tokens += count
        if count and (want == have or asked_pages <= room) and asked_tokens <= tokens:
            for j in range(have, want):
                tables[b][j] = free.pop()
            for p in range(held, held + count):
                positions.append(p)
                at = tables[b][p // page]
                slots.append(at * page + p % page if at >= 0 else -1)
            lengths[b] = held + count
        starts.append(len(positions))
    pad = tokens - len(positions)
    return tables, lengths, free, starts, positions + [0] * pad, slots + [-1] * pad


def truncate_pages(tables, lengths, keep, free, page):
    tables = [list(t) for t in tables]
    lengths, free = list(lengths), list(free)
    back = []
    for b, k in enumerate(keep):
        held = max(lengths[b], 0)
        left = min(held, max(k, 0))
        for j in range(-(-left // page), -(-held // page)):
            back.append(tables[b][j])
            tables[b][j] = -1
        lengths[b] = left
    return tables, lengths, free + back[::-1]


def cached(x):
    """The values that a cache holds of heads x [..][D]."""
    return mx4_values(x)
