"""Pins of the references for the 8-bit cache and the page operations.  CPU only."""
import numpy as np
import pytest
import torch

from oracle import linear as ol
from oracle import pages as op
from oracle import q8 as oq


@pytest.mark.parametrize("d", [64, 80, 128])
def test_places_are_permutations(d):
    for p in oq.places(d):
        assert sorted(p.reshape(-1)) == list(range(16 * d))


def test_e4m3_table_and_rounding_agree_with_torch():
    bits = torch.arange(256, dtype=torch.uint8)
    assert np.array_equal(oq.e4m3_values(), bits.view(torch.float8_e4m3fn).double().numpy(), equal_nan=True)
    # every midpoint of two neighbours, its neighbours in fp32, and random numbers
    grid = oq.e4m3_values()[:127]
    mid = ((grid[1:] + grid[:-1]) / 2).astype(np.float32)
    x = np.concatenate([mid, np.nextafter(mid, np.float32(0)), np.nextafter(mid, np.float32(1000)), grid.astype(np.float32),
                        np.random.default_rng(0).uniform(0, 448, 4000).astype(np.float32)])
    x = np.concatenate([x, -x])
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(oq.encode(x.astype(np.float64), oq.E4M3), want)


def test_quantise_is_the_nearest_code_and_handles_edges():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((3, 16, 64)).astype(np.float16).astype(np.float64)
    for fmt, top in ((oq.INT8, 127), (oq.E4M3, 448)):
        codes, scale = oq.quantise(x, fmt)
        values = np.arange(-127, 128) if fmt == oq.INT8 else np.unique(oq.e4m3_values()[np.isfinite(oq.e4m3_values())])
        z = x / scale.astype(np.float64)[:, None, None]
        best = np.min(np.abs(z[..., None] - values), axis=-1)
        assert np.array_equal(np.abs(oq.decode(codes, fmt) - z), best)
        assert np.allclose(scale, np.abs(x).max((-1, -2)) / top, rtol=2.0 ** -24)
        zeros, s = oq.quantise(np.zeros((16, 64)), fmt)
        assert s == 0 and not zeros.any()
        for bad in (np.inf, -np.inf, np.nan):
            y = x[0].copy()
            y[3, 5] = bad
            assert np.isnan(oq.quantise(y, fmt)[1])


def test_attend_on_closed_forms():
    rng = np.random.default_rng(2)
    K, V = rng.standard_normal((2, 2, 5, 8))
    assert np.array_equal(oq.attend(np.zeros((4, 8)), K[:, :0], V[:, :0]), np.zeros((4, 8)))
    assert np.allclose(oq.attend(rng.standard_normal((4, 8)), K[:, :1], V[:, :1]), np.repeat(V[:, 0], 2, 0))
    assert np.allclose(oq.attend(np.zeros((4, 8)), K, V), np.repeat(V.mean(1), 2, 0))


def test_page_references_keep_what_they_must():
    rng = np.random.default_rng(3)
    for _ in range(200):
        R, most, n_pages, o = int(rng.integers(1, 7)), int(rng.integers(1, 6)), int(rng.integers(8, 60)), int(rng.integers(0, 2))
        lens = rng.integers(0, most * 16 + 1, R)
        ids = rng.permutation(n_pages)[:R * most] if R * most <= n_pages else rng.integers(0, n_pages, R * most)
        table = ids.reshape(R, most)
        content = rng.integers(0, 1000, n_pages)
        # compaction: the pages that rows see do not change, ids are dense
        t, src, dst, n = op.compact(table, lens, most, o, n_pages)
        moved = content.copy()
        moved[dst] = content[src]
        for s in range(R):
            b = op.blocks(int(lens[s]), most, o)[0]
            assert np.array_equal(moved[t[s, :b]], content[table[s, :b]]) and np.all(t[s, b:] == -1)
        assert op.live(t, n_pages) == set(range(n)) and not set(src) & set(dst)
        # fork: rows see their parent's contents; open blocks are nobody else's
        parent = rng.integers(-1, R, int(rng.integers(1, 8)))
        if R * most > n_pages:
            continue
        t, n2, src, dst, short = op.fork(table, lens, parent, most, o, n_pages)
        if short:
            continue
        moved = content.copy()
        moved[dst[dst >= 0]] = content[src[src >= 0]]
        last = []
        for s, p in enumerate(parent):
            b = op.blocks(int(n2[s]), most, o)[0]
            assert n2[s] == (lens[p] if p >= 0 else 0)
            if p >= 0:
                assert np.array_equal(moved[t[s, :b]], content[table[p, :b]])
            if o and n2[s] % 16:
                last.append(t[s, b - 1])
        assert len(set(last)) == len(last)


def test_resize_reference_on_a_small_case():
    t, short = op.resize(np.array([[5, 9, 9], [2, 3, 4]]), [20, 48], [33, 16], 3, 1, 8)
    assert t.tolist() == [[5, 9, 0], [2, -1, -1]] and not short
    t, short = op.resize(np.array([[0, 9, 9], [9, 9, 9]]), [16, 0], [48, 32], 3, 1, 4)
    assert t.tolist() == [[0, 1, 2], [3, -1, -1]] and short


def test_linear4_by_loops():
    rng = np.random.default_rng(4)
    w4 = rng.integers(0, 256, (3, 32), dtype=np.uint8)
    scales = rng.standard_normal((3, 2))
    x = rng.standard_normal((2, 64))
    y = ol.linear4(x, w4, scales, 32)
    for m in range(2):
        for n in range(3):
            acc = sum(x[m, k] * ((int(w4[n, k // 2]) >> (4 * (k % 2)) & 15) - 8) * scales[n, k // 32] for k in range(64))
            assert abs(acc - y[m, n]) < 1e-12
