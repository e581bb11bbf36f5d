"""fp64 reference of the 8-bit KV cache: quantisation of a block, its byte layout, and attention over it.

TEST INFRASTRUCTURE ONLY.  Written from the definitions (scale = absmax / 127 or / 448 rounded to fp32, code = the
rounding of x / scale, ties to even) and from the byte order that ``include/isv.h`` documents, one byte at a time.
"""
from __future__ import annotations

from functools import lru_cache

import numpy as np

BT = 16
INT8, E4M3 = 0, 1


@lru_cache(None)
def places(d: int):
    """(k, v): k[t, x] / v[t, x] = byte, inside a unit's K / V part, of the code of token t, dim x."""
    P = d // 32
    k = np.full((BT, d), -1)
    v = np.full((BT, d), -1)
    for b in range(BT * d):
        if b < 512 * P:
            lane, p, i = (b % 512) // 16, b // 512, (b % 16) // 8
        else:
            lane, p, i = (b - 512 * P) // 8, P, 0
        g, c, h, j = lane // 4, lane % 4, (b % 8) // 4, b % 4
        dim = 32 * p + 8 * c + 4 * i + j if p < P else 32 * P + 4 * c + j
        k[g + 8 * h, dim] = b
        v[2 * c + j % 2 + 8 * (j // 2), g * (d // 8) + 2 * (2 * p + i) + h] = b
    return k, v


@lru_cache(None)
def e4m3_values():
    """The 256 values of e4m3 by bit pattern (1 sign, 4 exponent with bias 7, 3 mantissa; S.1111.111 is NaN)."""
    out = np.empty(256)
    for b in range(256):
        e, m = (b >> 3) & 15, b & 7
        mag = np.nan if (e, m) == (15, 7) else (m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7))
        out[b] = -mag if b >> 7 else mag
    return out


def encode(z: np.ndarray, fmt: int) -> np.ndarray:
    """Nearest code of each number, ties to even, largest magnitude beyond the range; as uint8 bits."""
    if fmt == INT8:
        return np.clip(np.rint(z), -127, 127).astype(np.int8).view(np.uint8)
    grid = e4m3_values()[:127]                               # 0 .. 448, ascending
    a = np.minimum(np.abs(z), 448.0)
    up = np.clip(np.searchsorted(grid, a), 1, 126)
    lo, hi = grid[up - 1], grid[up]
    down = (a - lo < hi - a) | ((a - lo == hi - a) & ((up - 1) % 2 == 0))
    code = np.where(down, up - 1, up).astype(np.uint8)
    return np.where(np.signbit(z), code | 0x80, code).astype(np.uint8)


def decode(codes: np.ndarray, fmt: int) -> np.ndarray:
    return codes.view(np.int8).astype(np.float64) if fmt == INT8 else e4m3_values()[codes]


def quantise(x: np.ndarray, fmt: int):
    """x [..., 16, d] float64 -> (codes uint8, same shape; scale float32 [...])."""
    x = np.asarray(x, np.float64)
    top = np.max(np.abs(x), axis=(-1, -2))
    with np.errstate(invalid="ignore"):
        scale = (top / (127.0 if fmt == INT8 else 448.0)).astype(np.float32)
    bad = ~np.isfinite(top)
    scale = np.where(bad, np.float32(np.nan), scale)
    s = np.where(bad | (scale == 0), 1.0, scale.astype(np.float64))[..., None, None]
    z = np.where((bad | (scale == 0))[..., None, None], 0.0, np.where(np.isfinite(x), x, 0.0) / s)
    return encode(z, fmt), scale


def unit(k: np.ndarray, v: np.ndarray, fmt: int):
    """Bytes [..., 32 d + 16] of blocks k, v [..., 16, d], and the dequantised blocks."""
    d = k.shape[-1]
    kp, vp = places(d)
    lead = k.shape[:-2]
    out = np.zeros(lead + (32 * d + 16,), np.uint8)
    deq = []
    for i, (x, p) in enumerate(((k, kp), (v, vp))):
        codes, scale = quantise(x, fmt)
        out[..., i * BT * d + p.reshape(-1)] = codes.reshape(lead + (BT * d,))
        out[..., 32 * d + 4 * i:32 * d + 4 * i + 4] = scale[..., None].view(np.uint8)
        deq.append(decode(codes, fmt) * scale.astype(np.float64)[..., None, None])
    return out, deq[0], deq[1]


def attend(q: np.ndarray, K: np.ndarray, V: np.ndarray) -> np.ndarray:
    """One sequence: q [Hq, d], K, V [Hkv, n, d] -> softmax(q K^T / sqrt d) V, zeros where n = 0."""
    g = q.shape[0] // K.shape[0]
    out = np.zeros(q.shape)
    if K.shape[1] == 0:
        return out
    for h in range(q.shape[0]):
        s = K[h // g] @ q[h] / np.sqrt(q.shape[1])
        w = np.exp(s - s.max())
        out[h] = (w / w.sum()) @ V[h // g]
    return out


def attend_error(q: np.ndarray, K: np.ndarray, V: np.ndarray) -> float:
    """How far an fp32 evaluation of one sequence may be from :func:`attend`.

    A score is a sum of d exact products: each of its d + 3 fp32 operations (sums, scale factors) is off by at most
    2^-23 of the sum of the magnitudes (2^-24 by rounding, twice that where the sum truncates).  A score off by e
    changes a weight by a factor within exp(+-e), so a quotient of weighted sums by 2 e of the largest |v|.  Weights carry 2^-21 of
    their own (exp2, their split into 16-bit parts), and the two sums over n tokens and at most 600 partial results
    n + 600 roundings of at most 2^-23 each.  Twice that for the running maximum's rescaling."""
    if K.shape[1] == 0:
        return 0.0
    g, d = q.shape[0] // K.shape[0], q.shape[1]
    mag = max(np.max(np.abs(K[h // g]) @ np.abs(q[h])) for h in range(q.shape[0])) / np.sqrt(d)
    e = (d + 3) * 2.0 ** -23 * mag
    return float(2 * np.max(np.abs(V)) * (2 * e + 2.0 ** -20 + 2 * (K.shape[1] + 600) * 2.0 ** -23))


def attend_typical(q: np.ndarray, K: np.ndarray, V: np.ndarray, q_step=None) -> np.ndarray:
    """How far the results [Hq, d] of an evaluation in fp32 may be from :func:`attend`, output by output: several times
    what independent roundings add up to, where :func:`attend_error` is what they could at worst, for the largest output.

    With weights w, results o and A = sum |q K| / sqrt d of a token: its score is off by a few of the 2^-23 A that its sums
    and factors round by (4 of them are counted), its weight by 2^-20 of its own on top (2^x, splits into 16-bit parts,
    units).  An error e of a score moves the result by w e (v - o), and independent ones add like the
    root of their squares; 4 times that is allowed.  Each of the n / 16 blocks, and each partial result, is one
    rounded addition to sums that stay below a = sum w |v|: sqrt(n / 16) of 2^-23 a, and 8 more for the
    products within a block and the last factors.

    q_step [Hq]: where the elements of q are held in a fixed step (rows of bf16 as fp16 numbers whose largest lies in [2^15, 2^16):
    steps of 2^-24, i.e. 2^-39 of the power of two below the row's largest), half a step of each
    element is off at most, and a score by that times sum |K| / sqrt d."""
    out = np.zeros(q.shape)
    n = K.shape[1]
    if n == 0:
        return out
    g, d = q.shape[0] // K.shape[0], q.shape[1]
    o = attend(q, K, V)
    for h in range(q.shape[0]):
        k, v = K[h // g], V[h // g]
        s = k @ q[h] / np.sqrt(d)
        w = np.exp(s - s.max())
        w /= w.sum()
        e = w * (4 * 2.0 ** -23 * (np.abs(k) @ np.abs(q[h])) / np.sqrt(d) + 2.0 ** -20)
        if q_step is not None:
            e = e + w * q_step[h] / 2 * np.abs(k).sum(1) / np.sqrt(d)
        spread = np.sqrt(np.square(e) @ np.square(v - o[h]))
        out[h] = 4 * spread + (8 + np.sqrt(n / BT)) * 2.0 ** -23 * (w @ np.abs(v))
    return out
