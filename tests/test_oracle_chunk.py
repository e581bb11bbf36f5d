"""The reference of chunks of new tokens against closed forms and library routines.  CPU only."""
import numpy as np
import pytest
import torch

from oracle import chunk as oc


def test_rotation_is_a_complex_product_and_keeps_relative_positions():
    rng = np.random.default_rng(0)
    x, y = rng.standard_normal((2, 3, 2, 64))
    freq = (10000.0 ** (-np.arange(16) / 16)).astype(np.float32)
    for pairs in (oc.HALVES, oc.ADJACENT):
        a, off = oc.rotate(x, [5, 6, 7], freq, 32, pairs, magnitude=1.5)
        i = np.arange(16)
        one, two = (i, i + 16) if pairs == oc.HALVES else (2 * i, 2 * i + 1)
        z = (x[..., one] + 1j * x[..., two]) * np.exp(1j * np.array([5, 6, 7])[:, None, None] * freq.astype(np.float64)) * 1.5
        assert np.allclose(a[..., one], z.real) and np.allclose(a[..., two], z.imag)
        assert np.array_equal(a[..., 32:], x[..., 32:]) and (off[..., 32:] == 0).all() and (off[..., :32] > 0).all()
        # the product of a turned query and a turned key depends on the distance alone
        p = (oc.rotate(x, [100] * 3, freq, 32, pairs)[0] * oc.rotate(y, [90] * 3, freq, 32, pairs)[0]).sum(-1)
        r = (oc.rotate(x, [1000010] * 3, freq, 32, pairs)[0] * oc.rotate(y, [1000000] * 3, freq, 32, pairs)[0]).sum(-1)
        assert np.allclose(p, r, atol=1e-9)


def test_rotation_by_axes():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((4, 1, 64))
    freq = np.ones(8, np.float32) / 7
    axis = np.array([0, 1, 2, 0, 1, 2, 0, 1])
    pos = rng.integers(0, 100, (3, 4))
    y, _ = oc.rotate(x, pos, freq, 16, oc.ADJACENT, axis)
    for i in range(8):
        z, _ = oc.rotate(x, pos[axis[i]], freq, 16, oc.ADJACENT)
        assert np.array_equal(y[..., 2 * i:2 * i + 2], z[..., 2 * i:2 * i + 2])


@pytest.mark.parametrize("d", [64, 80, 128])
def test_places_are_a_permutation_of_chunks(d):
    w = oc.places(d)
    assert (np.sort(w, 1) == np.arange(d)).all()
    assert w[0].tolist() == list(range(d)) and w[3, 0] == 24 and (d != 80 or w[3, 64] == 64) and (d != 128 or w[3, 64] == 64 + 24)


def test_attention_matches_the_library_and_masks():
    g = torch.Generator().manual_seed(0)
    q, k, v = (torch.randn((7, 4, 64), generator=g, dtype=torch.float64) for _ in range(3))
    k, v = (torch.randn((2, 19, 64), generator=g, dtype=torch.float64) for _ in range(2))
    pos = np.arange(12, 19)
    for window, prefix in ((0, 0), (5, 0), (1, 3), (0, 17)):
        seen = oc.visible(pos, 19, window, prefix)
        want = torch.nn.functional.scaled_dot_product_attention(q.transpose(0, 1), k.repeat_interleave(2, 0), v.repeat_interleave(2, 0),
                                                                attn_mask=torch.tensor(seen))
        got, tol = oc.attend(q.numpy(), k.numpy(), v.numpy(), pos, seen, 1 / 8)
        assert np.allclose(got, want.transpose(0, 1).numpy()) and (tol > 0).all() and tol.max() < 1e-4
    assert oc.visible([4], 6, 2, 0).tolist() == [[False, False, False, True, True, False]]
    assert oc.visible([1], 4, 1, 3).tolist() == [[True, True, True, False]]


def test_caps_biases_and_empty_rows():
    rng = np.random.default_rng(2)
    q, k, v = rng.standard_normal((3, 2, 64)), rng.standard_normal((1, 5, 64)), rng.standard_normal((1, 5, 64))
    seen = np.array([[1, 1, 1, 0, 0], [0, 0, 0, 0, 0], [1, 1, 1, 1, 1]], bool)
    o, _ = oc.attend(q, k, v, [2, 3, 4], seen, 0.5, 3.0, np.array([0.25, 0.0]))
    assert (o[1] == 0).all()
    x = 3.0 * np.tanh(k[0, :3] @ q[0, 0] * 0.5 / 3.0) - 0.25 * np.array([2, 1, 0])
    w = np.exp(x) / np.exp(x).sum()
    assert np.allclose(o[0, 0], w @ v[0, :3])
    v[0, 4] = np.inf                                           # only the last query sees it
    p, _ = oc.attend(q, k, v, [2, 3, 4], seen, 0.5, 3.0)
    assert np.isfinite(p[:2]).all() and np.isinf(p[2]).all()


def test_tolerances_reject_a_lost_token_and_a_wrong_mask():
    rng = np.random.default_rng(3)
    n = 300
    q, k, v = rng.standard_normal((4, 2, 64)), rng.standard_normal((2, n, 64)), rng.standard_normal((2, n, 64))
    pos = np.arange(n - 4, n)
    seen = oc.visible(pos, n)
    for step in (2.0 ** -17, 2.0 ** -8):
        o, tol = oc.attend(q, k, v, pos, seen, 1 / 8, weight_step=step)
        for bad in (oc.visible(pos + 1, n + 1)[:, :n], seen & (np.arange(n) != 7)):
            x, _ = oc.attend(q, k, v, pos, bad, 1 / 8)
            rows = (bad != seen).any(1)
            off = np.abs(x - o)[rows] / tol[rows]
            assert off.max() > 1, (step, off.max())


def test_verification_keeps_the_targets_distribution():
    rng = np.random.default_rng(4)
    V, N = 5, 40000
    p, q = rng.dirichlet(np.ones(V)), rng.dirichlet(np.ones(V))
    seen = np.zeros(V)
    for _ in range(N):
        x = rng.choice(V, p=q)
        a, t = oc.verify(np.stack([p, p]), q[None], [x], rng.random(2))
        seen[x if a else t] += 1
    assert np.abs(seen / N - p).max() < 5 * np.sqrt(0.25 / N)          # five standard deviations


def test_verification_rules():
    p = np.array([[0.5, 0.5, 0.0], [0.2, 0.3, 0.5]])
    q = np.array([[0.5, 0.25, 0.25]])
    assert oc.verify(p, q, [0], [0.999, 0.0]) == (1, 0)
    assert oc.verify(p, q, [2], [0.0, 0.9]) == (0, 1)                   # a probability of 0 never stands
    assert oc.verify(p, None, [0], [0.5, 0.0]) == (0, 1)                # 0.5 < 0.5 does not hold; the residual leaves the draft out
    assert oc.verify(p, None, [1], [0.4, 0.5]) == (1, 2)                # 0.5 > 0.5 does not hold
    assert oc.verify(p[:1], None, [], [0.5]) == (0, 1)
    assert oc.verify(p, p[:1], [2], [0.5, 0.7]) == (0, 1)               # an empty residual: the target itself
    assert oc.verify(np.zeros((2, 3)), q, [0], [0.5, 0.5]) == (0, -1)
    odd = np.array([[np.nan, -0.5, 0.75]])                              # count as 0: the residual of the target beyond them is all of it
    assert oc.verify(p, odd, [2], [0.0, 0.0]) == (0, 0) and oc.verify(p, odd, [2], [0.0, 0.5]) == (0, 1)
    assert oc.verify(p, odd, [0], [0.9, 0.0]) == (1, 0) and oc.verify(p, odd, [1], [0.9, 0.0]) == (1, 0)
    assert oc.verify(np.stack([-p[0], p[1]]), odd, [1], [0.9, 0.0]) == (0, -1)
    assert oc.verify(p, q, [7], [0.0, 0.0]) == (0, 1)
