"""Attention over the 8-bit cache keeps the precision of fp32 (oracle.q8.attend_typical): long histories, tokens that
dominate one, small weights next to large ones, large channels, scales far apart."""
import numpy as np
import pytest
import torch

from oracle import q8 as oq
from paper_2504_11816_b200 import binding as B
from test_gpu_q8 import FORMATS, Cache

pytestmark = pytest.mark.gpu


def near(c, rows=None, steps=False):
    """Attends and compares every output with the bound; with `steps` also where bf16 rows of q span more than fp16 holds: elements
    below 2^-32 of the largest are multiples of 2^-39 of the power of two below that, which is the header's promise."""
    _, out32 = c.attend()
    for s in range(len(c.lens)) if rows is None else rows:
        _, K, V = c.units(s)
        q = c.q[s].double().cpu().numpy()
        off = np.abs(out32[s].double().cpu().numpy() - oq.attend(q, K, V))
        bound = oq.attend_typical(q, K, V, 2.0 ** (np.floor(np.log2(np.abs(q).max(1))) - 39) if steps else None)
        assert np.all(off <= bound), (s, c.lens[s], float(np.max(off / np.maximum(bound, 1e-300))))


def scores_of_the_first(c, nats):
    """Moves every query along its KV head's first key until that token's score is `nats`."""
    for s in range(len(c.lens)):
        for h in range(c.Hq):
            k = c.k[s][0, h // (c.Hq // c.H)].double()
            q = c.q[s, h].double().cpu()
            c.q[s, h] = (q + (nats * c.d ** 0.5 - q @ k) / (k @ k) * k).to(c.dt).cuda()


def second(change):
    """For Cache's `make`: changes V only (K and V of a sequence are made in turn)."""
    made = [0]

    def make(x):
        made[0] += 1
        return change(x) if made[0] % 2 == 0 else x
    return make


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("lens,hq,hkv,d,dtype", [
    ([20011], 8, 2, 128, "bf16"), ([5000, 3, 9000, 16], 4, 4, 80, "f16"), ([700, 31, 257], 12, 1, 64, "bf16"),
    ([1000, 15, 48], 32, 2, 128, "f16"), ([4111] * 2, 8, 2, 128, "bf16")])
def test_long_and_ragged(lens, hq, hkv, d, dtype, fmt):
    with Cache(lens, hq, hkv, d, dtype, fmt, seed=41) as c:
        near(c.fill())


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("d,dtype,hq,hkv", [(128, "f16", 4, 2), (128, "bf16", 16, 1), (80, "f16", 2, 2), (64, "bf16", 4, 1)])
@pytest.mark.parametrize("nats", [9, 14])
def test_a_first_token_that_dominates(nats, d, dtype, hq, hkv, fmt):
    """Its weight is e^9 or e^14 times another's, and the others together weigh as much or matter in its zero entries."""
    def change(x):
        x[:16, :, 8:] = 0
        if x.shape[0] > 20:
            x[5, :, 7] = 64                     # and the first block's scale of V is far above the others'
        return x
    for make in (None, second(change)):
        with Cache([8192, 3000, 45], hq, hkv, d, dtype, fmt, seed=42, make=make) as c:
            c.fill()
            scores_of_the_first(c, nats)
            near(c)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("order", [1, -1])
def test_small_weights_on_blocks_of_smaller_values(order, fmt):
    """Block scales of V fall or rise by 2^7 and more, with scores that favour the large ones or the small ones."""
    def change(x):
        for b in range((x.shape[0] + 15) // 16):
            x[16 * b:16 * b + 16, :, :] *= 2.0 ** (-order * 2 * (b % 6))
            x[16 * b:16 * b + 16, :, b % 6::6] = 0
        return x
    for nats in (0, 8):
        with Cache([6 * 16 * 20 + 7, 100], 4, 2, 128, "bf16", fmt, seed=43, make=second(change)) as c:
            c.fill()
            scores_of_the_first(c, nats)
            near(c)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("mean", [0, 2])
@pytest.mark.parametrize("d,dtype", [(128, "f16"), (80, "bf16"), (64, "f16")])
def test_large_channels_of_k(d, dtype, mean, fmt):
    """Four channels of K are far from zero, q has a mean: the scores are small sums of codes that are small next to 128."""
    made = [0]

    def make(x):
        made[0] += 1
        if made[0] % 2:
            x[..., 3] += 200
            x[..., 17] -= 200
            x[..., 40] += 50
            x[..., 41] -= 50
        return x
    with Cache([4096, 1003], 4, 2, d, dtype, fmt, seed=44, make=make) as c:
        c.q += mean
        near(c.fill())


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("d", [64, 80, 128])
def test_queries_whose_elements_lie_far_apart(d, fmt):
    """One element of each query is 2^10 to 2^30 times the others, on a channel where K is zero: the others make the scores.
    And rows of q from 2^-120 to 2^100 on keys that bring the scores back to ordinary size."""
    made = [0]

    def make(x):
        made[0] += 1
        if made[0] % 2:
            x[..., 9] = 0
        return x
    with Cache([300, 47, 900], 8, 2, d, "bf16", fmt, seed=45, make=make) as c:
        c.fill()
        for h in range(8):
            c.q[:, h, 9] = 2.0 ** (10 + 3 * h) * (-1) ** h
        near(c, steps=True)
    for e in (-120, -60, 60, 100):
        made[0] = 0

        def keys(x):
            made[0] += 1
            return x * 2.0 ** -e if made[0] % 2 else x
        with Cache([300, 47], 4, 2, d, "bf16", fmt, seed=46, make=keys) as c:
            c.q.mul_(2.0 ** e)
            near(c.fill())
