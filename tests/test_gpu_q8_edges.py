"""The 8-bit KV cache at the edges of its ranges, through the C ABI, against the fp64 reference."""
import pytest
import torch

from oracle import q8 as oq
from paper_2504_11816_b200 import binding as B
from test_gpu_q8 import Cache

pytestmark = pytest.mark.gpu


def test_rows_longer_than_32_bit_lengths_are_refused():
    """16 * max_blocks + 15 tokens, the longest length of a row, is rounded up to blocks in 32 bits: 2^27 - 2 is the most."""
    with Cache([16], 2, 2, 64) as c:
        c.fill()
        lens = torch.tensor([16], dtype=torch.int32, device="cuda")
        out = torch.zeros_like(c.q)
        for most, fine in ((2 ** 27 - 2, True), (2 ** 27 - 1, False)):
            attn = (c.h, c.pool, c.n_pages, c.tails, c.table, most, most, lens, c.q, out, None, 1)
            write = (c.h, c.pool, c.n_pages, c.tails, c.table, most, most, lens, None, *c.kept[:2], 16 * 128, 128, 1, 16)
            for fn, args in ((B.isv_q8_attn, attn), (B.isv_q8_write, write)):
                if fine:
                    fn(*args)
                    continue
                with pytest.raises(B.IsvError) as ei:
                    fn(*args)
                assert ei.value.code == B.ISV_EINVAL and "table row" in ei.value.message
        torch.cuda.synchronize()
        c.check(out, None)
        c.check_bytes()


def _aligned(c, factor):
    """Makes every query a multiple of its KV head's first key, so that the scores have that factor's sign, all of them."""
    g = c.Hq // c.H
    for s in range(len(c.lens)):
        for h in range(c.Hq):
            k = c.k[s][0, h // g].double()
            c.q[s, h] = (k / k.norm() ** 2 * factor).to(c.dt).cuda()


@pytest.mark.parametrize("fmt", [B.ISV_Q8_INT8, B.ISV_Q8_E4M3])
@pytest.mark.parametrize("factor", [-1e20, -1e31, -1e34, -1e37, 1e34])
def test_scores_of_any_size(factor, fmt):
    """One token: whatever its score, the result is its V.  Equal keys: whatever the score, the mean of the V."""
    for lens in ([1, 15], [16, 47], [3000]):
        def make(x):
            x[:] = x[:1]                                                # the same row throughout
            return x
        with Cache(lens, 4, 2, 64, "bf16", fmt, seed=31, make=make) as c:
            c.fill()
            _aligned(c, factor)
            out, out32 = c.attend()
            for s, n in enumerate(lens):
                _, _, V = c.units(s)
                want = V.mean(1).repeat(2, 0)
                # rows of complete blocks and of the open one differ by roundings of their codes; any mean of them lies in between
                room = 2 * abs(V - V[:, :1]).max() + 1e-5 * abs(V).max()
                assert abs(out32[s].double().cpu().numpy() - want).max() <= room, (n, factor)


@pytest.mark.parametrize("fmt", [B.ISV_Q8_INT8, B.ISV_Q8_E4M3])
@pytest.mark.parametrize("sizes", [(1, 1e-37, 2.0 ** -133, 1), (2.0 ** -133, 1e-37, 1, 1e-37), (2.0 ** -133,), (1e-37, 1), (1e30, 1e-37, 1e30)])
def test_values_whose_blocks_lie_at_the_ends_of_bf16(sizes, fmt):
    """Ordinary blocks of V before and behind blocks of the smallest and of very large numbers: finite results, as exact as
    the largest block asks for.  The sizes go round block by block; the open block has the next one."""
    made = [0]

    def make(x):
        made[0] += 1
        if made[0] % 2 == 0:
            for b in range((x.shape[0] + 15) // 16):
                y = x[16 * b:16 * b + 16]
                y.clamp_(-3, 3).div_(3).mul_(sizes[b % len(sizes)])
        return x
    lens = [len(sizes) * 16 * 30, 16 * len(sizes) * 2 + 5, 16 * len(sizes), 37, 4]
    with Cache(lens, 4, 2, 64, "bf16", fmt, seed=33, make=make) as c:
        c.fill()
        _, out32 = c.attend()
        for s in range(len(lens)):
            _, K, V = c.units(s)
            q = c.q[s].double().cpu().numpy()
            off = abs(out32[s].double().cpu().numpy() - oq.attend(q, K, V))
            # half a step of fp32's smallest numbers, each block's and the products' own
            assert (off <= oq.attend_typical(q, K, V) + lens[s] * 2.0 ** -148).all(), s


@pytest.mark.parametrize("fmt", [B.ISV_Q8_INT8, B.ISV_Q8_E4M3])
@pytest.mark.parametrize("sizes", [(3.3e38,), (1, 1e38, 2.0 ** -133), (3e38, 1)])
@pytest.mark.parametrize("max_ctas", [0, 3])
def test_sums_of_values_beyond_the_largest_number(max_ctas, sizes, fmt):
    """The weighted mean of V is finite where the weighted sum over many tokens is not, in one warp and in partial results."""
    made = [0]

    def make(x):
        made[0] += 1
        if made[0] % 2 == 0:
            for b in range((x.shape[0] + 15) // 16):
                y = x[16 * b:16 * b + 16]
                y.clamp_(-3, 3).div_(3).mul_(sizes[b % len(sizes)])
        return x
    lens = [5003, 16, 300, 9]
    with Cache(lens, 8, 2, 128, "bf16", fmt, seed=34, make=make, max_ctas=max_ctas) as c:
        c.fill()
        _, out32 = c.attend()
        for s in range(len(lens)):
            _, K, V = c.units(s)
            q = c.q[s].double().cpu().numpy()
            off = abs(out32[s].double().cpu().numpy() - oq.attend(q, K, V))
            assert (off <= oq.attend_typical(q, K, V)).all(), s


@pytest.mark.parametrize("fmt", [B.ISV_Q8_INT8, B.ISV_Q8_E4M3])
@pytest.mark.parametrize("dtype,hq,hkv,d", [("f16", 4, 2, 64), ("bf16", 8, 1, 128), ("f16", 12, 1, 80), ("bf16", 2, 2, 80)])
def test_infinities_in_the_open_block(dtype, hq, hkv, d, fmt):
    """V of a token that is still held in 16 bits: an infinity of either sign gives one in its dim, two of both signs or a NaN
    give NaN, every other dim is as exact as ever.  K: an infinite score leaves the token out or makes the head NaN."""
    with Cache([37, 613, 5], hq, hkv, d, dtype, fmt, seed=35) as c:
        c.fill()
        inf = float("inf")
        for s in range(3):
            for t, x, value in ((0, 3, inf), (2, 5, -inf), (1, 7, inf), (3, 7, -inf), (4, 9, float("nan")), (1, d - 1, inf)):
                c.tails[s, 1, 0, t, x] = value
                c.v[s][c.lens[s] // 16 * 16 + t, 0, x] = value
        _, out32 = c.attend()
        assert B.isv_q8_status(c.h) == 0
        g = hq // hkv
        for s in range(3):
            _, K, V = c.units(s)
            q, got = c.q[s].double().cpu().numpy(), out32[s].double().cpu().numpy()
            assert (got[:g, [3, d - 1]] == inf).all() and (got[:g, 5] == -inf).all()
            assert (got[:g, [7, 9]] != got[:g, [7, 9]]).all()
            V = V.copy()
            V[0][:, [3, 5, 7, 9, d - 1]] = 0
            got[:g, [3, 5, 7, 9, d - 1]] = 0
            assert (abs(got - oq.attend(q, K, V)) <= oq.attend_typical(q, K, V)).all(), s
    with Cache([20, 300], hq, hkv, d, dtype, fmt, seed=36) as c:
        c.fill()
        c.q[:, :, 11] = abs(c.q[:, :, 11]) + 0.5
        for s in range(2):
            c.tails[s, 0, 0, 1, 11] = -inf                  # the score is -inf: the weight is 0
        _, out32 = c.attend()
        for s in range(2):
            _, K, V = c.units(s)
            q, got = c.q[s].double().cpu().numpy(), out32[s].double().cpu().numpy()
            keep = [t for t in range(c.lens[s]) if t != c.lens[s] // 16 * 16 + 1]
            want, room = oq.attend(q, K[:, keep], V[:, keep]), oq.attend_typical(q, K[:, keep], V[:, keep])
            assert (abs(got - want) <= room)[:hq // hkv].all(), s
            c.tails[s, 0, 0, 1, 11] = inf                   # the score is inf
        _, out32 = c.attend()
        assert torch.isnan(out32[:, :hq // hkv]).all() and torch.isfinite(out32[:, hq // hkv:]).all()
