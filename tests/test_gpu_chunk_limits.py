"""Chunks of new tokens at their limits: refused arguments, lost copies and waits that run out, tables of pages at the far
end of their ranges, lengths that change between replays."""
import numpy as np
import pytest
import torch

from _chunk import Case, dev, f64
from oracle import chunk as oc
from paper_2504_11816_b200 import binding as B

pytestmark = pytest.mark.gpu

A = 1 << 20        # an aligned address; refused calls do not follow it


def _refused(text, fn, *a, **kw):
    with pytest.raises(B.IsvError) as ei:
        fn(*a, **kw)
    assert ei.value.code == B.ISV_EINVAL and text in ei.value.message, ei.value


@pytest.fixture
def handle():
    h = B.isv_chunk_create(q_heads=8, kv_heads=2, head_dim=64, dtype=B.ISV_BF16, max_seqs=4, rotary_dim=64)
    yield h
    B.isv_chunk_free(h)


def _attn(**kw):
    d = dict(pool=A, n_pages=10, block_table=A, table_stride=4, max_blocks_per_seq=4, seq_lens=A, new_lens=A, row_starts=A, n_rows=8, q=A,
             q_stride=512, slopes=None, prefix_lens=None, window=0, out=2 * A, out_f32=None, n_seqs=2, T=4)
    d.update(kw)
    return d


def _write(**kw):
    d = dict(pool=A, n_pages=10, block_table=A, table_stride=4, max_blocks_per_seq=4, seq_lens=A, new_lens=A, row_starts=A, n_rows=8, k=A, v=A,
             kv_stride=128, q=A, q_stride=512, q_out=2 * A, inv_freq=A, positions=None, pair_axis=None, magnitude=1.0, n_seqs=2, T=4)
    d.update(kw)
    return d


COMMON = [(dict(pool=None), "required"), (dict(block_table=None), "required"), (dict(seq_lens=None), "required"), (dict(pool=A + 8), "16-byte"),
          (dict(n_seqs=5), "n_seqs"), (dict(n_seqs=-1), "n_seqs"), (dict(n_pages=0), "page count"), (dict(table_stride=3), "table row"),
          (dict(max_blocks_per_seq=0), "table row"), (dict(max_blocks_per_seq=1 << 27, table_stride=1 << 27), "table row"), (dict(T=-1), "bad T"),
          (dict(T=1 << 28), "bad T"), (dict(n_rows=-1), "n_rows"), (dict(row_starts=None, n_rows=7), "n_rows"), (dict(n_pages=1 << 25), "too many pages")]


@pytest.mark.parametrize("kw,text", COMMON + [
    (dict(q=None), "q and one output"), (dict(out=None), "q and one output"), (dict(q=A + 8), "16-byte"), (dict(out=A + 2), "16-byte"),
    (dict(out_f32=A + 4), "16-byte"), (dict(q_stride=511), "stride"), (dict(q_stride=504), "stride"), (dict(window=-1), "window"),
    (dict(out=A), "overlap"), (dict(out_f32=A), "overlap"), (dict(out_f32=2 * A), "overlap")])
def test_attn_refuses(handle, kw, text):
    _refused(text, B.isv_chunk_attn, handle, **_attn(**kw))


@pytest.mark.parametrize("kw,text", COMMON + [
    (dict(k=None), "k and v"), (dict(v=A + 8), "k and v"), (dict(q=A + 8), "16-byte"), (dict(q=None), "q_out without q"), (dict(kv_stride=120), "strides"),
    (dict(kv_stride=132), "strides"), (dict(q_stride=256), "strides"), (dict(inv_freq=None), "inv_freq"), (dict(pair_axis=A), "pair_axis"),
    (dict(magnitude=float("inf")), "magnitude"), (dict(q_out=A, q_stride=1024), "q_out is q")])
def test_write_refuses(handle, kw, text):
    _refused(text, B.isv_chunk_write, handle, **_write(**kw))


def test_calls_without_work_are_fine(handle):
    B.isv_chunk_attn(handle, **_attn(n_seqs=0, row_starts=None, n_rows=0))
    B.isv_chunk_attn(handle, **_attn(T=0))
    B.isv_chunk_attn(handle, **_attn(n_rows=0))
    B.isv_chunk_write(handle, **_write(n_seqs=0))
    B.isv_chunk_write(handle, **_write(T=0))
    assert B.isv_chunk_status(handle) == 0


@pytest.mark.parametrize("news,d,dtype", [([40], 128, "bf16"), ([3], 64, "f16"), ([30], 80, "bf16"), ([100], 64, "bf16")])
def test_a_lost_copy_ends_in_a_status_not_a_hang(news, d, dtype):
    """A page of the first visit is expected and never copied: the waits run out, the call is reported once, and the handle works on."""
    c = Case([500], news, 8, 2, d, dtype)
    want, tol = c.want(weight_step=2.0 ** -16)
    c.to_gpu()
    h = c.handle()
    f32 = torch.full((c.rows, c.Hq, c.d), 7.0, device="cuda")
    try:
        B.isv_chunk_set_wait_limit(h, 20000)
        B.isv_chunk_inject_lost_copy(h, 1)
        c.attend(h, None, f32)
        with pytest.raises(B.IsvError) as ei:
            B.isv_chunk_status(h)
        assert ei.value.code == B.ISV_EDEVICE_STATUS and "0x2" in ei.value.message
        assert B.isv_chunk_status(h) == 0
        B.isv_chunk_set_wait_limit(h, 0)
        f32.fill_(7.0)
        c.attend(h, None, f32)
        c.check(f32, want, tol)
        assert B.isv_chunk_status(h) == 0
    finally:
        B.isv_chunk_free(h)


@pytest.mark.parametrize("news,d", [(48, 128), (20, 64), (6, 80)])
def test_rows_that_take_long_do_not_run_out_the_waits_of_others(news, d):
    """The value of the last token is infinite: every other row is computed token by token, while the rest of the CTA waits."""
    n = 4000 + news
    c = Case([4000], [news], 16, 2, d, "f16")
    c.pool[c.table[0, (n - 1) // 16], 1, :, (n - 1) % 16] = float("inf")
    want, tol = c.want(weight_step=2.0 ** -16)
    c.to_gpu()
    h = c.handle(max_ctas=1)
    f32 = torch.full((c.rows, c.Hq, c.d), 7.0, device="cuda")
    try:
        B.isv_chunk_set_wait_limit(h, 2000)
        c.attend(h, None, f32)
        assert B.isv_chunk_status(h) == 0
        c.check(f32, want, tol)
    finally:
        B.isv_chunk_free(h)


def test_knobs_validate_their_arguments(handle):
    _refused("negative", B.isv_chunk_inject_lost_copy, handle, -1)
    _refused("null", B.isv_chunk_set_wait_limit, None, 5)
    B.isv_chunk_inject_lost_copy(handle, 0)


def test_more_query_heads_than_a_tile_has_rows():
    """150 query heads on one KV head: two passes of 75; 128 and 129 at the border."""
    for Hq, H, news in ((150, 1, [3, 1]), (256, 2, [2, 0]), (129, 1, [1, 5])):
        c = Case([60, 300], news, Hq, H, 64, "bf16")
        c.to_gpu()
        h = c.handle()
        f32 = torch.full((c.rows, c.Hq, c.d), 7.0, device="cuda")
        try:
            c.attend(h, None, f32)
            c.check(f32, *c.want(weight_step=2.0 ** -16))
        finally:
            B.isv_chunk_free(h)


def test_the_largest_single_sequence_positions_and_a_wide_stride():
    """A sequence of 300000 tokens, most of whose table is empty: positions far behind, one page of them there."""
    n = 300000
    d, H, Hq = 64, 2, 4
    g = torch.Generator().manual_seed(0)
    blocks = (n + 15) // 16
    table = torch.full((1, blocks), -1, dtype=torch.int32)
    there = [0, 7, blocks // 2, blocks - 1]
    table[0, there] = torch.arange(4, dtype=torch.int32)
    pool = torch.randn((4, 2, H, 16, d), generator=g).half()
    out = torch.zeros((3, Hq, d), device="cuda")
    h = B.isv_chunk_create(q_heads=Hq, kv_heads=H, head_dim=d, dtype=B.ISV_F16, max_seqs=1)
    try:
        base = torch.randn((3, 16, d), generator=g).half().cuda()
        qd = base[:, 8:12]
        B.isv_chunk_attn(h, pool.cuda(), 4, table.cuda(), blocks, blocks, dev([n]), dev([2]), dev([1]), 3, qd.data_ptr(), base.stride(0), None, None, 0,
                         None, out, 1, 2)
        K, V, seen = oc.history(f64(pool), table[0].tolist(), n)
        pos = np.array([n - 2, n - 1])
        want, tol = oc.attend(f64(qd[1:]), K, V, pos, oc.visible(pos, n) & seen, 1 / 8, weight_step=2.0 ** -16)
        assert (np.abs(f64(out[1:]) - want) <= tol).all() and (out[0] == 0).all()
        assert B.isv_chunk_status(h) == 0
    finally:
        B.isv_chunk_free(h)


def test_replays_follow_the_lengths_on_the_device():
    """A captured step in which every sequence grows by what it gets; starts from nothing, some sequences rest."""
    S, d, H, Hq, blocks = 5, 128, 2, 8, 20
    rng = np.random.default_rng(3)
    g = torch.Generator().manual_seed(3)
    n_pages = S * blocks
    pool = torch.randn((n_pages, 2, H, 16, d), generator=g).bfloat16()
    table = torch.tensor(rng.permutation(n_pages).reshape(S, blocks), dtype=torch.int32)
    T, rows = 7, 7 * S
    q = torch.randn((rows, Hq, d), generator=g).bfloat16()
    D = dict(pool=pool.cuda(), table=table.cuda(), lens=dev(np.zeros(S)), news=dev(np.zeros(S)), firsts=dev(np.arange(S) * T), q=q.cuda())
    out = torch.zeros((rows, Hq, d), device="cuda")
    h = B.isv_chunk_create(q_heads=Hq, kv_heads=H, head_dim=d, dtype=B.ISV_BF16, max_seqs=S)
    try:
        def call():
            B.isv_chunk_attn(h, D["pool"], n_pages, D["table"], blocks, blocks, D["lens"], D["news"], D["firsts"], rows, D["q"], Hq * d, None, None, 0,
                             None, out, S, T, torch.cuda.current_stream().cuda_stream)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        lens = np.zeros(S, int)
        for _ in range(12):
            news = rng.integers(0, T + 1, S)
            lens = lens + news + rng.integers(0, 15, S) * (news > 0)
            lens = np.minimum(lens, 16 * blocks)
            D["lens"].copy_(dev(lens)), D["news"].copy_(dev(news))
            out.fill_(7.0)
            graph.replay()
            torch.cuda.synchronize()
            for s in range(S):
                K, V, seen = oc.history(f64(pool), table[s].tolist(), int(lens[s]))
                pos = lens[s] - news[s] + np.arange(news[s])
                r = slice(s * T, s * T + news[s])
                want, tol = oc.attend(f64(q[r]), K, V, pos, oc.visible(pos, int(lens[s])) & seen, 1 / np.sqrt(d), weight_step=2.0 ** -16)
                assert (np.abs(f64(out[r]) - want) <= tol).all()
                assert (out[s * T + news[s]:(s + 1) * T] == 7).all()
        assert B.isv_chunk_status(h) == 0
    finally:
        B.isv_chunk_free(h)
