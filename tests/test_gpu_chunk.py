"""Attention of chunks of new tokens over the paged cache against the fp64 reference, through the C ABI."""
import numpy as np
import pytest
import torch

from _chunk import Case, dev, f64, run_and_check
from oracle import chunk as oc
from paper_2504_11816_b200 import binding as B
from paper_2504_11816_b200 import workloads as W

pytestmark = pytest.mark.gpu

HEADS = [(1, 1), (4, 4), (8, 2), (7, 1), (12, 1), (6, 2), (16, 1), (34, 2)]      # query heads, KV heads


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("d", [64, 80, 128])
@pytest.mark.parametrize("Hq,H", HEADS)
def test_head_layouts(Hq, H, d, dtype):
    run_and_check(Case([0, 5, 130, 300, 16], [1, 3, 40, 2, 16], Hq, H, d, dtype, seed=Hq + d))


@pytest.mark.parametrize("d,dtype", [(64, "bf16"), (80, "f16"), (128, "f16"), (128, "bf16")])
@pytest.mark.parametrize("starts,news", [
    ([0], [1]), ([0, 0, 0], [0, 0, 0]), ([0, 0], [1, 0]), ([15], [1]), ([16], [1]), ([0], [16]), ([0], [17]), ([111], [17]), ([127], [1]),
    ([128], [1]), ([127], [2]), ([0], [127]), ([0], [128]), ([0], [129]), ([1], [255]), ([0], [256]), ([0], [257]), ([255], [258]),
    ([100] * 40, [1] * 40), (list(range(0, 400, 10)), [j % 7 for j in range(40)]), ([2000], [1]), ([2000, 0, 3], [5, 700, 1])])
def test_lengths(starts, news, d, dtype):
    run_and_check(Case(starts, news, 8, 4, d, dtype, seed=sum(starts) + sum(news)), outputs=("both", "16"))


def test_a_long_history_of_one_user():
    for d, dtype, T, Hq, H in ((128, "bf16", 1, 32, 8), (64, "f16", 9, 4, 1), (80, "bf16", 33, 8, 8)):
        run_and_check(Case([20001], [T], Hq, H, d, dtype), outputs=("both",))


def test_more_sequences_than_sms_and_a_full_handle():
    rng = np.random.default_rng(0)
    run_and_check(Case(rng.integers(0, 60, 700), rng.integers(0, 4, 700), 4, 2, 64, "bf16"), outputs=("both",))


@pytest.mark.parametrize("d,dtype", [(64, "f16"), (80, "bf16"), (128, "f16"), (128, "bf16")])
@pytest.mark.parametrize("window", [1, 15, 16, 100, 128, 129, 1000])
def test_windows(window, d, dtype):
    run_and_check(Case([0, 300, 511, 40], [33, 150, 2, 300], 4, 2, d, dtype, seed=window), window=window, outputs=("both", "16"))


@pytest.mark.parametrize("d,dtype", [(64, "bf16"), (80, "f16"), (128, "bf16")])
def test_prefixes(d, dtype):
    c = Case([0, 0, 100, 300, 64], [40, 200, 30, 2, 140], 6, 3, d, dtype)
    for prefix in ([0, 200, 130, 1, 100], [40, 150, 110, 302, 204], [-5, 1000, 0, 17, 128]):
        run_and_check(c, prefix=prefix, outputs=("both", "16"))
        run_and_check(c, prefix=prefix, window=20, outputs=("16",))


@pytest.mark.parametrize("d,dtype", [(64, "f16"), (80, "bf16"), (128, "bf16"), (128, "f16")])
def test_caps_biases_and_scales(d, dtype):
    c = Case([0, 10, 500], [20, 300, 3], 8, 2, d, dtype)
    slopes = 2.0 ** -np.arange(1, 9)
    run_and_check(c, softcap=5.0)
    run_and_check(c, slopes=slopes)
    run_and_check(c, slopes=-slopes / 8, outputs=("both",))
    run_and_check(c, scale=0.5, softcap=30.0, slopes=slopes, window=100, prefix=[3, 200, 400])
    run_and_check(c, scale=-0.25, outputs=("both",))


def test_a_bias_that_outweighs_all_but_the_last_tokens_and_capped_large_scores():
    c = Case([700], [5], 2, 1, 128, "bf16")
    run_and_check(c, slopes=np.array([300.0, 1e4]), outputs=("both",))
    c.qkv *= 30
    run_and_check(c, softcap=20.0, outputs=("both",))


def test_weights_far_below_the_largest_count():
    """One token with a score far above all others, whose V is zero: the result comes from weights 2^-20 and less of the
    largest, which must keep their precision."""
    for dtype in ("f16", "bf16"):
        c = Case([4000], [3], 2, 1, 64, dtype)
        K, V, _ = oc.history(f64(c.pool), c.table[0], 4003)
        qd = f64(c.q[c.firsts[0]:c.firsts[0] + 3]).mean((0, 1))
        page, slot = int(c.table[0, 2000 // 16]), 2000 % 16
        w = torch.tensor(oc.places(64)[slot])
        c.qkv[:, :2] = torch.tensor(np.sign(qd)).to(c.qkv.dtype)             # all queries alike: their product with the sink is 14 * 8
        c.pool[page, 0, 0, slot, w] = torch.tensor(np.sign(qd) * 14 / 8).to(c.pool.dtype)
        c.pool[page, 1, 0, slot] = 0
        run_and_check(c, outputs=("both", "16"))


def test_infinities_and_nan_in_tokens_that_a_query_does_not_see_change_nothing():
    for d, dtype in ((64, "bf16"), (80, "f16"), (128, "bf16")):
        c = Case([0, 200, 5], [20, 150, 300], 4, 2, d, dtype)
        for s, j, what in ((0, 10, "nan"), (0, 11, "inf"), (1, 260, "inf"), (1, 340, "nan"), (2, 304, "-inf"), (2, 150, "nan")):
            page, slot = int(c.table[s, j // 16]), j % 16
            c.pool[page, 1, 0, slot, :5] = float(what)                        # V of head 0; head 1 stays clean
            if s != 2:
                c.pool[page, 0, 1, slot, 3] = float(what)                     # K of head 1
        # queries that see such a K get NaN from the reference where it was NaN (or an infinity of either sign)
        with np.errstate(all="ignore"):
            run_and_check(c, outputs=("both", "16"))


def test_large_values_do_not_overflow_the_sums():
    c = Case([900], [3], 2, 1, 64, "bf16")
    c.pool[:, 1] *= 1e37
    want, tol = c.want(weight_step=2.0 ** -16)
    D, h = c.to_gpu(), c.handle()
    try:
        f32 = torch.full((c.rows, c.Hq, c.d), 7.0, device="cuda")
        c.attend(h, None, f32)
        c.check(f32, want, tol)
    finally:
        B.isv_chunk_free(h)
    c = Case([900], [3], 2, 1, 64, "bf16")
    c.pool[:, 1] *= 1e-30
    run_and_check(c, outputs=("32",))


def test_pages_that_are_missing_or_bad():
    c = Case([100, 500, 40], [20, 150, 3], 4, 2, 128, "bf16")
    c.table[0, 3] = B.ISV_BLOCK_NONE
    c.table[1, 0] = c.table[1, 20] = c.table[1, 40] = B.ISV_BLOCK_NONE        # the last one is its own chunk's
    c.table[2, :3] = B.ISV_BLOCK_NONE                                         # nothing left: zeros
    run_and_check(c)
    c.table[0, 2] = c.n_pages
    c.table[1, 5] = -2
    D, h = c.to_gpu(), c.handle()
    try:
        f32 = torch.full((c.rows, c.Hq, c.d), 7.0, device="cuda")
        c.attend(h, None, f32)
        c.check(f32, *c.want(weight_step=2.0 ** -16))
        with pytest.raises(B.IsvError) as ei:
            B.isv_chunk_status(h)
        assert ei.value.code == B.ISV_EDEVICE_STATUS and B.isv_chunk_status(h) == 0
    finally:
        B.isv_chunk_free(h)


def test_bad_lengths_and_rows_are_clamped_and_flagged():
    c = Case([30, 0, 100], [5, 0, 30], 4, 2, 64, "f16", gaps=False)
    for what, value in (("lens", 16 * c.blocks + 9), ("lens", -3), ("news", 31), ("news", -1), ("firsts", -1), ("firsts", c.rows + 5),
                        ("firsts", c.rows - 2)):
        D, h = c.to_gpu(), c.handle()
        try:
            D[what][0] = value
            f32 = torch.full((c.rows, c.Hq, c.d), 7.0, device="cuda")
            c.attend(h, None, f32)
            with pytest.raises(B.IsvError) as ei:
                B.isv_chunk_status(h)
            assert ei.value.code == B.ISV_EDEVICE_STATUS, (what, value)
            other = slice(c.firsts[2], c.firsts[2] + 30)                      # the sequence behind it is as it should be
            want, tol = c.want(weight_step=2.0 ** -16)
            assert (np.abs(f64(f32[other]) - want[other]) <= tol[other]).all()
            if (what, value) == ("firsts", c.rows - 2):                       # its first two tokens fit
                first = slice(c.firsts[0], c.firsts[0] + 2)
                K, V, _ = oc.history(f64(c.pool), c.table[0], 35)
                o, room = oc.attend(f64(c.q[-2:]), K, V, [30, 31], oc.visible([30, 31], 35), 1 / 8, weight_step=2.0 ** -16)
                assert (np.abs(f64(f32[-2:]) - o) <= room).all() and (f32[first] == 7).all()
        finally:
            B.isv_chunk_free(h)


def test_without_new_lens_and_row_starts():
    c = Case([30, 0, 77], [6, 6, 6], 4, 2, 80, "bf16", gaps=False, spare=0)
    c.firsts = np.arange(3) * 6
    D, h = c.to_gpu(), c.handle()
    try:
        f32 = torch.full((c.rows, c.Hq, c.d), 7.0, device="cuda")
        B.isv_chunk_attn(h, D["pool"], c.n_pages, D["table"], c.stride, c.blocks, D["lens"], None, None, 18, D["q"], D["q"].stride(0), None,
                         None, 0, None, f32, 3, 6)
        c.check(f32, *c.want(weight_step=2.0 ** -16))
        assert B.isv_chunk_status(h) == 0
    finally:
        B.isv_chunk_free(h)


def test_one_handle_for_calls_of_other_sizes_streams_and_graphs():
    big = Case([300, 40, 900], [200, 1, 30], 8, 2, 128, "bf16")
    small = Case([10, 20], [1, 2], 8, 2, 128, "bf16", seed=5)
    h = big.handle(max_seqs=64)
    try:
        outs = []
        for c in (big, small, big, small):
            c.to_gpu()
            f32 = torch.full((c.rows, c.Hq, c.d), 7.0, device="cuda")
            c.attend(h, None, f32)
            c.check(f32, *c.want(weight_step=2.0 ** -16))
            outs.append(f32)
        assert torch.equal(outs[0], outs[2]) and torch.equal(outs[1], outs[3])
        side = torch.cuda.Stream()
        f32 = torch.full((big.rows, 8, 128), 7.0, device="cuda")
        torch.cuda.synchronize()
        big.attend(h, None, f32, stream=side.cuda_stream)
        side.synchronize()
        assert torch.equal(f32, outs[0])
        # a captured step: the lengths of a replay are those on the device then
        f32.fill_(7.0)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            for _ in range(3):
                big.attend(h, None, f32, stream=torch.cuda.current_stream().cuda_stream)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(f32, outs[0])
        big.starts[0], big.lens[0] = big.starts[0] - 77, big.lens[0] - 77
        big.D["lens"].copy_(dev(big.lens))
        graph.replay()
        torch.cuda.synchronize()
        # tokens behind the new length are another sequence's business now
        big.check(f32, *big.want(weight_step=2.0 ** -16))
        assert B.isv_chunk_status(h) == 0
    finally:
        B.isv_chunk_free(h)


def test_fewer_ctas_give_the_same_numbers():
    c = Case([3000, 0, 77], [20, 300, 1], 8, 4, 64, "f16")
    want, tol = c.want(weight_step=2.0 ** -16)
    for ctas in (1, 2, 7, 1000):
        D, h = c.to_gpu(), c.handle(max_ctas=ctas)
        try:
            f32 = torch.full((c.rows, c.Hq, c.d), 7.0, device="cuda")
            c.attend(h, None, f32)
            c.check(f32, want, tol)
        finally:
            B.isv_chunk_free(h)


def test_handles_on_two_streams_at_once():
    cases = [Case([700, 3], [60, 9], 8, 2, 128, "bf16", seed=1), Case([200, 900], [5, 300], 4, 4, 64, "f16", seed=2)]
    hs, streams, outs = [c.handle() for c in cases], [torch.cuda.Stream() for _ in cases], []
    try:
        for c in cases:
            c.to_gpu()
            outs.append(torch.full((c.rows, c.Hq, c.d), 7.0, device="cuda"))
        torch.cuda.synchronize()
        for _ in range(20):
            for c, h, st, o in zip(cases, hs, streams, outs):
                c.attend(h, None, o, stream=st.cuda_stream)
        torch.cuda.synchronize()
        for c, o in zip(cases, outs):
            c.check(o, *c.want(weight_step=2.0 ** -16))
    finally:
        for h in hs:
            B.isv_chunk_free(h)
