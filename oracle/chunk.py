"""fp64 reference of the calls on chunks of new tokens: position rotation, the 16-bit pool's order, attention with its masks
and biases, verification of drafts.

TEST INFRASTRUCTURE ONLY.  Written from the definitions in ``include/isv.h``, one sequence at a time.
"""
from __future__ import annotations

import numpy as np

BT = 16
HALVES, ADJACENT = 0, 1
HALF_STEP = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8, "f32": 2.0 ** -24}


def rotate(x, pos, freq, rotary: int, pairs: int, axis=None, magnitude: float = 1.0):
    """x [n, heads, d], pos [n] or [axes, n], freq [rotary / 2] -> (turned x, how far 32-bit arithmetic may be from it).

    The fraction of a turn is off by 2^-24 (its rounding to 32 bits) and 2^-53 of the turns it was taken from, i.e. the angle by
    2 pi of that; the sine and cosine of an exact fraction by 2^-23 each; two products and a sum round by 2^-24 of the
    terms' magnitudes each, the magnitude by 2^-24 more."""
    x = np.asarray(x, np.float64)
    y, off = x.copy(), np.zeros(x.shape)
    pos = np.asarray(pos)
    for i in range(rotary // 2):
        p = (pos if pos.ndim == 1 else pos[int(axis[i]) if axis is not None else 0]).astype(np.float64)
        angle = np.multiply(p, float(freq[i]), dtype=np.longdouble)
        c, s = (np.asarray(f(angle), np.float64)[:, None] for f in (np.cos, np.sin))
        a, b = (i, i + rotary // 2) if pairs == HALVES else (2 * i, 2 * i + 1)
        y[..., a] = (x[..., a] * c - x[..., b] * s) * magnitude
        y[..., b] = (x[..., b] * c + x[..., a] * s) * magnitude
        turns = np.asarray(np.abs(angle), np.float64)[:, None] / (2 * np.pi)
        e = 2 * np.pi * (2.0 ** -24 + 2 * 2.0 ** -53 * turns) + 2.0 ** -23 + 4 * 2.0 ** -24
        off[..., a] = off[..., b] = (np.abs(x[..., a]) + np.abs(x[..., b])) * e * abs(magnitude)
    return y, off


def places(d: int):
    """[16, d]: where in its row element e of token t of a page is stored."""
    out = np.empty((BT, d), np.int64)
    for t in range(BT):
        for c in range(d // 8):
            at = (c ^ (t % 8)) if c < d // 64 * 8 else c
            out[t, 8 * c:8 * c + 8] = 8 * at + np.arange(8)
    return out


def history(pool, table, n: int):
    """pool [pages, 2, H, 16, d] (any numbers), one table row -> K, V [H, n, d] and which tokens have a page [n]."""
    pages, _, H, _, d = pool.shape
    w = places(d)
    kv = np.zeros((2, H, n, d), pool.dtype)
    there = np.zeros(n, bool)
    for b in range((n + BT - 1) // BT):
        page = int(table[b])
        if not 0 <= page < pages:
            continue
        m = min(BT, n - b * BT)
        tile = np.take_along_axis(pool[page], np.broadcast_to(w, pool[page].shape), -1)
        kv[:, :, b * BT:b * BT + m] = tile[:, :, :m]
        there[b * BT:b * BT + m] = True
    return kv[0], kv[1], there


def visible(pos, n: int, window: int = 0, prefix: int = 0):
    """[queries, n]: which tokens the queries at positions pos see."""
    j = np.arange(n)[None]
    p = np.asarray(pos)[:, None]
    seen = j <= p
    if window:
        seen &= p - j < window
    return seen | (j < prefix)


def attend(q, K, V, pos, seen, scale: float, cap: float = 0.0, slopes=None, weight_step: float = 2.0 ** -20):
    """q [T, Hq, d], K, V [H, n, d], seen [T, n] -> (out [T, Hq, d], how far an evaluation in 32 bits may be from it).

    As :func:`oracle.q8.attend_typical`: a score is off by a few of the 2^-23 A that its sums and factors round by, A the sum
    of the magnitudes that enter it (products, cap, bias, the score itself), a weight by ``weight_step`` of its own on
    top (2^x, and its rounding to 16 bits where it is kept in one 16-bit number); independent errors add like the root of
    their squares, 4 times that is allowed.  The sums over tiles and partial results round by 2^-23 of a = sum w |v| each."""
    T, Hq, d = q.shape
    H, n = K.shape[:2]
    g = Hq // H
    out, tol = np.zeros((T, Hq, d)), np.zeros((T, Hq, d))
    if n == 0 or T == 0:
        return out, tol
    far = np.abs(np.asarray(pos)[:, None] - np.arange(n)[None]).astype(np.float64)
    some = seen.any(1)
    for h in range(Hq):
        k, v = K[h // g].astype(np.float64), V[h // g].astype(np.float64)
        with np.errstate(invalid="ignore", over="ignore"):
            x = (q[:, h] @ k.T) * scale
            A = (np.abs(q[:, h]) @ np.abs(k).T) * abs(scale)
            if cap:
                x = cap * np.tanh(x / cap)
                A = A + 2 * cap
            if slopes is not None:
                x = x - slopes[h] * far
                A = A + 2 * np.abs(slopes[h]) * far
            x = np.where(seen, x, -np.inf)
            top = np.where(some, x.max(1), 0.0)[:, None]
            w = np.where(seen, np.exp(x - top), 0.0)
            w = w / np.where(some, w.sum(1), 1.0)[:, None]
            fine = np.isfinite(v).all(1)
            vf = np.where(fine[:, None], v, 0.0)
            o = w @ vf
            for j in np.flatnonzero(~fine):                 # they reach those only that see them
                o = o + np.where(seen[:, j, None], w[:, j, None] * v[j], 0.0)
            # a score of minus infinity is exact: its weight is 0, however large what it was summed from
            e = np.where(seen & (w != 0), w * (4 * 2.0 ** -23 * (A + np.abs(np.where(seen, x, 0.0))) + weight_step), 0.0)
            spread = np.sqrt(np.square(e) @ np.square(vf) + np.square(e).sum(1)[:, None] * np.square(o))
            tol[:, h] = 4 * spread + (16 + np.sqrt(n / BT)) * 2.0 ** -23 * (w @ np.abs(vf))
        out[:, h] = o
    return out, tol


def verify(target, draft, drafted, u):
    """target [n + 1, V], draft [n, V] or None, drafted [n], u [n + 1] (the last one for the draw) -> (a, next token).
    Probabilities that are negative or NaN count as 0."""
    def positive(z):
        z = np.asarray(z, np.float64)
        return np.where(z > 0, z, 0.0)

    target, draft = positive(target), None if draft is None else positive(draft)
    n = len(drafted)
    a = n
    for i in range(n):
        x = int(drafted[i])
        if not 0 <= x < target.shape[1]:
            a = i
            break
        q = 1.0 if draft is None else float(draft[i, x])
        if not float(u[i]) * q < float(target[i, x]):
            a = i
            break

    p = target[a]
    w = p
    if a < n:
        if draft is None:
            r = p.copy()
            if 0 <= int(drafted[a]) < len(r):
                r[int(drafted[a])] = 0.0
        else:
            r = positive(p - draft[a])
        if r.sum() > 0:
            w = r
    if not w.sum() > 0:
        return a, -1
    up = np.cumsum(w)
    hit = np.flatnonzero((up > float(u[n]) * up[-1]) & (w > 0))
    return a, int(hit[0]) if len(hit) else int(np.flatnonzero(w > 0)[-1])
