"""What the error bounds of the references let through and what they do not: an evaluation in fp32 passes, one that
loses a block, a partial result or precision does not.  CPU only; mistakes are planted here, in numpy."""
import numpy as np
import pytest
import torch

from oracle import linear as ol
from oracle import q8 as oq


def _bf16(x):
    return torch.from_numpy(np.asarray(x, np.float64)).to(torch.bfloat16).double().numpy()


def _f16(x):
    return np.asarray(x, np.float64).astype(np.float16).astype(np.float64)


def _two_f16(scale):
    """A number as an fp16 value and its fp16 remainder, after a multiplication by `scale`."""
    def both(x):
        hi = _f16(x * scale)
        return (hi + _f16(x * scale - hi)) / scale
    return both


def history(n, heads, d, seed, touch=None):
    """K, V [heads][n][d] as an int8 cache holds them (the open block in 16 bits), its codes and scales of K; normal, one
    entry in 100 eight times as large."""
    rng = np.random.default_rng(seed)
    kv = []
    for i in range(2):
        x = rng.standard_normal((heads, n, d))
        x = np.where(rng.random(x.shape) < 0.01, 8 * x, x)
        kv.append(_f16(touch(i, x) if touch else x))
    full, out = n // 16 * 16, []
    for x in kv:
        codes, scale = oq.quantise(x[:, :full].reshape(heads, -1, 16, d), oq.INT8)
        rows = (oq.decode(codes, oq.INT8) * scale.astype(np.float64)[..., None, None]).reshape(heads, full, d)
        out.append((np.concatenate([rows, x[:, full:]], 1), oq.decode(codes, oq.INT8).reshape(heads, full, d), scale))
    return out[0][0], out[1][0], out[0][1], out[0][2]


def queries(heads, d, seed, K, first=None, mean=0.0):
    """Normal around `mean`; `first`: the score (in nats) that the first token gets."""
    q = np.random.default_rng(seed + 1).standard_normal((heads, d)) + mean
    if first is not None:
        g = heads // K.shape[0]
        for h in range(heads):
            k = K[h // g][0]
            q[h] += (first * np.sqrt(d) - q[h] @ k) / (k @ k) * k
    return _f16(q)


def in_fp32(q, K, V, weights=None, without=(), scores=None):
    """Attention block by block in fp32."""
    g, (d, n) = q.shape[0] // K.shape[0], (q.shape[1], K.shape[1])
    out = np.zeros(q.shape)
    f = np.float32(1.4426950408889634 / np.sqrt(d))
    for h in range(q.shape[0]):
        s = np.zeros(n, np.float32)
        if scores is not None:
            s = scores(h)
        else:
            for x in range(0, d, 16):
                s = s + K[h // g][:, x:x + 16].astype(np.float32) @ q[h, x:x + 16].astype(np.float32)
        p = np.exp2(s * f - (s * f).max()).astype(np.float32)
        l = p.sum()
        if weights:
            p = weights(p).astype(np.float32)
        acc = np.zeros(d, np.float32)
        for b in range(0, n, 16):
            if b // 16 not in without:
                acc = acc + p[b:b + 16] @ V[h // g][b:b + 16].astype(np.float32)
        out[h] = acc / l
    return out


def ratio(got, q, K, V):
    """The largest error in units of the bound."""
    return np.max(np.abs(got - oq.attend(q, K, V)) / oq.attend_typical(q, K, V))


@pytest.mark.parametrize("n,hq,hkv,d", [(15, 2, 1, 64), (704, 4, 2, 64), (9000, 4, 4, 80), (20011, 4, 1, 128)])
def test_attention_bound_lets_fp32_through_and_nothing_less(n, hq, hkv, d):
    K, V, _, _ = history(n, hkv, d, n)
    q = queries(hq, d, n, K)
    assert ratio(in_fp32(q, K, V), q, K, V) < 0.3
    assert ratio(in_fp32(q, K, V, weights=_two_f16(2.0 ** 15)), q, K, V) < 0.3
    if n > 16:
        for gone in ((0,), (1,), (n // 32,), ((n - 1) // 16,), range(n // 160, n // 160 + 5)):
            assert ratio(in_fp32(q, K, V, without=gone), q, K, V) > 10, gone
    assert ratio(in_fp32(q, K, V, weights=_bf16), q, K, V) > 10
    assert ratio(in_fp32(q, K, V, weights=_f16), q, K, V) > 3


def test_attention_bound_sees_small_weights_that_lose_bits():
    """A first token 11 nats above the rest with one large entry of V: fp16 ends at 2^-24."""
    def touch(i, x):
        if i:
            x[:, 5, 7] = 64
        return x
    K, V, _, _ = history(8192, 2, 128, 5, touch)
    q = queries(4, 128, 5, K, first=11)
    assert ratio(in_fp32(q, K, V), q, K, V) < 0.3
    assert ratio(in_fp32(q, K, V, weights=_two_f16(2.0 ** 15)), q, K, V) < 0.3
    assert ratio(in_fp32(q, K, V, weights=_two_f16(2.0 ** -5)), q, K, V) > 10


def test_attention_bound_sees_scores_that_carry_an_offset():
    """Two large channels of K, a query with a mean: sums of (code + 128) q less 128 sum q lose what the codes are small by."""
    def touch(i, x):
        if i == 0:
            x[..., 3] += 200
            x[..., 17] -= 200
        return x
    K, V, codes, scale = history(4096, 2, 128, 7, touch)
    q = queries(4, 128, 7, K, mean=2.0)

    def offset(h):
        s = np.zeros(4096, np.float32)
        for x in range(0, 128, 16):
            s = s + (codes[h // 2][:, x:x + 16] + 128).astype(np.float32) @ q[h, x:x + 16].astype(np.float32)
        return (s - np.float32(128 * q[h].sum())) * np.repeat(scale[h // 2], 16)
    assert ratio(in_fp32(q, K, V), q, K, V) < 0.3
    assert ratio(in_fp32(q, K, V, scores=offset), q, K, V) > 1


@pytest.mark.parametrize("K,group", [(64, 32), (4096, 128), (12800, 64), (11008, 32)])
def test_linear_bound_lets_fp32_through_and_nothing_less(K, group):
    M, N, rng = 2, 40, np.random.default_rng(K)
    x = _bf16(rng.standard_normal((M, K)))
    w4 = rng.integers(0, 256, (N, K // 2), dtype=np.uint8)
    scales = _bf16(rng.standard_normal((N, K // group)) / np.sqrt(K))
    u = np.empty((N, K))
    u[:, 0::2], u[:, 1::2] = w4 & 15, w4 >> 4
    u -= 8
    want, bound = ol.linear4(x, w4, scales, group), ol.linear4_typical(x, w4, scales, group)

    def by_groups(rounded, upto=K):
        total = np.zeros((M, N), np.float32)
        for i in range(upto // group):
            part = np.zeros((M, N), np.float32)
            for k in range(i * group, (i + 1) * group, 16):
                part = part + x[:, k:k + 16].astype(np.float32) @ u[:, k:k + 16].T.astype(np.float32)
            total = total + rounded(part).astype(np.float32) * scales[:, i].astype(np.float32)
        return np.max(np.abs(total - want) / bound)
    assert by_groups(lambda p: p) < 0.3
    assert by_groups(_bf16) > 10 and by_groups(lambda p: p, K - group) > 10
    assert np.max(np.abs(x @ _bf16(u * np.repeat(scales, group, 1)).T - want) / bound) > 10
