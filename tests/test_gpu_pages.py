"""Page operations against the serial reference, through the C ABI: everything exactly."""
import numpy as np
import pytest
import torch

from oracle import pages as op
from oracle import q8 as oq
from paper_2504_11816_b200 import binding as B

pytestmark = pytest.mark.gpu


def _dev(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def _state(rng, rows, most, n_pages, stride, shared=False):
    lens = rng.integers(0, most * 16 + 1, rows)
    lens[rng.random(rows) < 0.2] = 0
    if rows * most <= n_pages and not shared:
        ids = rng.permutation(n_pages)[:rows * most].reshape(rows, most)
    else:
        ids = rng.integers(0, n_pages, (rows, most))
    table = np.full((rows, stride), 12345678, np.int64)
    table[:, :most] = ids
    return table, lens


SHAPES = [  # rows, blocks of a row, pages, row stride
    (1, 1, 1, 1), (3, 2, 31, 2), (5, 7, 64, 9), (33, 10, 1000, 10), (256, 20, 6000, 24), (1, 5000, 5003, 5000), (4096, 3, 20000, 3),
    (700, 13, 4000, 13), (2, 40, 300000, 40), (16, 100, 1 << 20, 100)]


@pytest.mark.parametrize("open_in_pool", [0, 1])
@pytest.mark.parametrize("rows,most,n_pages,stride", SHAPES)
def test_fork(rows, most, n_pages, stride, open_in_pool):
    rng = np.random.default_rng(rows + most)
    for rows_out in {rows, 1, min(4096, 2 * rows + 1)}:
        table, lens = _state(rng, rows, most, n_pages, stride)
        parent = rng.integers(0, rows, rows_out)
        parent[rng.random(rows_out) < 0.3] = int(rng.integers(0, rows))      # one parent of many
        parent[rng.random(rows_out) < 0.1] = -1
        t, n, src, dst, short = op.fork(table[:, :most], lens, parent, most, open_in_pool, n_pages)
        out = torch.full((rows_out, stride), 77, dtype=torch.int32, device="cuda")
        lens_out, a, b = (torch.full((rows_out,), 77, dtype=torch.int32, device="cuda") for _ in range(3))
        status = _dev([0])
        B.isv_pages_fork(_dev(table), _dev(lens), rows, _dev(parent), out, lens_out, rows_out, stride, most, open_in_pool, n_pages, a, b,
                         status)
        assert np.array_equal(out[:, :most].cpu().numpy(), t) and (out[:, most:] == 77).all()
        assert np.array_equal(lens_out.cpu().numpy(), n)
        assert np.array_equal(a.cpu().numpy(), src) and np.array_equal(b.cpu().numpy(), dst)
        assert status.item() == (B.ISV_STATUS_NO_PAGES if short else 0)


@pytest.mark.parametrize("open_in_pool", [0, 1])
@pytest.mark.parametrize("rows,most,n_pages,stride", SHAPES)
def test_resize(rows, most, n_pages, stride, open_in_pool):
    rng = np.random.default_rng(rows * 3 + most)
    for k in range(3):
        table, lens = _state(rng, rows, most, n_pages, stride, shared=k == 1)
        lens = np.minimum(lens, [most * 16, 40, most * 8][k])
        new = np.clip(lens + rng.integers(-40, 60, rows), 0, most * 16)
        if k == 2:
            new[rng.random(rows) < 0.5] = 0
        t, short = op.resize(table[:, :most], lens, new, most, open_in_pool, n_pages)
        dev, status = _dev(table), _dev([0])
        B.isv_pages_resize(dev, _dev(lens), _dev(new), rows, stride, most, open_in_pool, n_pages, status)
        got = dev.cpu().numpy()
        assert np.array_equal(got[:, :most], t) and np.array_equal(got[:, most:], table[:, most:])
        assert status.item() == (B.ISV_STATUS_NO_PAGES if short else 0)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("open_in_pool", [0, 1])
@pytest.mark.parametrize("rows,most,n_pages,stride", SHAPES)
def test_compact(rows, most, n_pages, stride, open_in_pool, in_place):
    rng = np.random.default_rng(rows * 5 + most)
    for shared in (False, True):
        table, lens = _state(rng, rows, most, n_pages, stride, shared)
        t, src, dst, live = op.compact(table[:, :most], lens, most, open_in_pool, n_pages)
        dev = _dev(table)
        out = dev if in_place else torch.full_like(dev, 77)
        m = n_pages // 2 + 3
        a, b = (torch.full((m,), 77, dtype=torch.int32, device="cuda") for _ in range(2))
        counts, status = _dev([77, 77]), _dev([0])
        B.isv_pages_compact(dev, _dev(lens), rows, stride, most, open_in_pool, n_pages, out, a, b, m, counts, status)
        assert np.array_equal(out[:, :most].cpu().numpy(), t)
        assert counts.tolist() == [live, len(src)] and status.item() == 0
        pad = [-1] * (m - len(src))
        assert a.tolist() == src + pad and b.tolist() == dst + pad


def test_bad_entries_and_lengths_are_flagged():
    table = np.array([[3, 500, -1], [1 << 30, 2, 4], [0, 1, 5]])
    lens, bad_lens = [48, 48, 20], [-5, 49, 20]
    for ls, flag in ((lens, B.ISV_STATUS_BAD_BLOCK_ID), (bad_lens, B.ISV_STATUS_BAD_LENGTH | B.ISV_STATUS_BAD_BLOCK_ID)):
        out, a, b, counts, status = torch.empty(3, 3, dtype=torch.int32, device="cuda"), *(torch.empty(8, dtype=torch.int32, device="cuda")
                                                                                  for _ in range(2)), _dev([0, 0]), _dev([0])
        B.isv_pages_compact(_dev(table), _dev(ls), 3, 3, 3, 1, 16, out, a, b, 8, counts, status)
        t, src, dst, live = op.compact(table, ls, 3, 1, 16)
        assert np.array_equal(out.cpu().numpy(), t) and status.item() == flag and counts.tolist() == [live, len(src)]
    # fork: parents that do not exist give empty rows; ids of other pools are carried along and never split
    out, lens_out, a, b, status = torch.empty(4, 3, dtype=torch.int32, device="cuda"), *(_dev([9] * 4) for _ in range(3)), _dev([0])
    parent = [3, -2, 0, 0]
    B.isv_pages_fork(_dev(table), _dev([47, 0, 0]), 3, _dev(parent), out, lens_out, 4, 3, 3, 1, 16, a, b, status)
    t, n, src, dst, _ = op.fork(table, [47, 0, 0], parent, 3, 1, 16)
    assert np.array_equal(out.cpu().numpy(), t) and np.array_equal(lens_out.cpu().numpy(), n)
    assert a.tolist() == list(src) and b.tolist() == list(dst) and status.item() == B.ISV_STATUS_BAD_BLOCK_ID
    dev, status = _dev(table), _dev([0])
    B.isv_pages_resize(dev, _dev([48, 48, 20]), _dev([16, -3, 70]), 3, 3, 3, 1, 16, status)
    assert np.array_equal(dev.cpu().numpy(), op.resize(table, [48, 48, 20], [16, -3, 70], 3, 1, 16)[0])
    assert status.item() & B.ISV_STATUS_BAD_LENGTH


def test_no_rows_and_no_status_word():
    out, a, b, counts = torch.empty(1, dtype=torch.int32, device="cuda"), _dev([7] * 4), _dev([7] * 4), _dev([7, 7])
    B.isv_pages_compact(out, out.clone(), 0, 1, 1, 1, 8, out, a, b, 4, counts)
    assert counts.tolist() == [0, 0] and a.tolist() == [-1] * 4 and b.tolist() == [-1] * 4
    t = _dev([[-1]])
    B.isv_pages_resize(t, _dev([0]), _dev([16]), 1, 1, 1, 1, 8)
    assert t.tolist() == [[0]]


@pytest.mark.parametrize("page,layers", [(16, 1), (80, 3), (2064, 2), (32896, 1), (65536, 2), (1048592, 1)])
def test_copy(page, layers):
    rng = np.random.default_rng(page)
    n_src, n_dst = 40, 50
    src = torch.randint(0, 256, (layers, n_src + 2, page), dtype=torch.uint8, device="cuda")
    dst = torch.randint(0, 256, (layers, n_dst + 1, page), dtype=torch.uint8, device="cuda")
    for n in (1, 7, 33):
        a, b = rng.integers(0, n_src, n), rng.permutation(n_dst)[:n]
        a[rng.random(n) < 0.2] = -1
        b[rng.random(n) < 0.2] = -1
        for limit in (None, n // 2, n + 5, -3):
            want = dst.clone()
            upto = n if limit is None else max(0, min(n, limit))
            for i in range(upto):
                if a[i] >= 0 and b[i] >= 0:
                    want[:, b[i]] = src[:, a[i]]
            status = _dev([0])
            B.isv_pages_copy(dst, n_dst, src, n_src, page, layers, (n_dst + 1) * page, (n_src + 2) * page, _dev(a), _dev(b), n,
                             None if limit is None else _dev([limit]), status)
            assert torch.equal(dst, want) and status.item() == 0
    # page i where no destinations are given; ids outside the pools
    ids = _dev([5, n_src, -1, -9, 0])
    want = dst.clone()
    want[:, 0], want[:, 4] = src[:, 5], src[:, 0]
    status = _dev([0])
    B.isv_pages_copy(dst, n_dst, src, n_src, page, layers, (n_dst + 1) * page, (n_src + 2) * page, ids, None, 5, None, status)
    assert torch.equal(dst, want) and status.item() == B.ISV_STATUS_BAD_BLOCK_ID


def test_copy_within_a_pool_beyond_four_gigabytes():
    page = 1 << 20
    n = 5000
    pool = torch.zeros((n, page), dtype=torch.uint8, device="cuda")
    pool[4998] = 7
    pool[3] = 9
    B.isv_pages_copy(pool, n, pool, n, page, 1, 0, 0, _dev([4998, 3]), _dev([1, 4999]), 2)
    assert (pool[1] == 7).all() and (pool[4999] == 9).all() and (pool[4998] == 7).all()


def test_a_replayed_step_on_a_side_stream():
    """Lengths grow by one, pages are handed out, all in one captured graph."""
    rows, most, n_pages = 5, 4, 30
    table = torch.full((rows, most), -1, dtype=torch.int32, device="cuda")
    old, new = torch.zeros(rows, dtype=torch.int32, device="cuda"), _dev([0, 3, 15, 16, 30])
    B.isv_pages_resize(table, old, new, rows, most, most, 1, n_pages)
    want = op.resize(np.full((rows, most), -1), [0] * rows, [0, 3, 15, 16, 30], most, 1, n_pages)[0]
    status = _dev([0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        old.copy_(new)
        new += 1
        B.isv_pages_resize(table, old, new, rows, most, most, 1, n_pages, status, torch.cuda.current_stream().cuda_stream)
    n = np.array([0, 3, 15, 16, 30])
    for _ in range(34):
        graph.replay()
        want = op.resize(want, n, n + 1, most, 1, n_pages)[0]
        n = n + 1
        assert np.array_equal(table.cpu().numpy(), want)
    assert status.item() == 0


@pytest.mark.parametrize("fmt", [B.ISV_Q8_INT8, B.ISV_Q8_E4M3])
def test_a_generation_with_forks_and_compaction(fmt):
    """The calls together: an 8-bit cache whose rows grow, fork (tail slots copied along), end, and are made dense; every
    step's attention is checked against a plain record of the rows."""
    rng = np.random.default_rng(7)
    R, H, Hq, d, most, n_pages = 6, 2, 4, 64, 6, 40
    page, tail = B.isv_q8_sizes(H, d)
    pool = torch.zeros((n_pages, page), dtype=torch.uint8, device="cuda")
    tails = [torch.zeros((R, tail), dtype=torch.uint8, device="cuda") for _ in range(2)]
    tables = [torch.full((R, most), -1, dtype=torch.int32, device="cuda") for _ in range(2)]
    lens = [torch.zeros(R, dtype=torch.int32, device="cuda") for _ in range(2)]
    src, dst = (torch.zeros(n_pages // 2, dtype=torch.int32, device="cuda") for _ in range(2))
    counts, status = _dev([0, 0]), _dev([0])
    record = [(np.zeros((H, 0, d)), np.zeros((H, 0, d))) for _ in range(R)]
    h = B.isv_q8_create(q_heads=Hq, kv_heads=H, head_dim=d, dtype=B.ISV_F16, format=fmt, max_seqs=R)
    try:
        for step in range(60):
            grow = torch.tensor(rng.integers(0, 4, R) * (rng.random(R) < 0.8), dtype=torch.int32)
            grow = torch.minimum(grow, 16 * most + 15 - lens[0].cpu())
            new = lens[0] + grow.cuda()
            B.isv_pages_resize(tables[0], lens[0], new, R, most, most, 0, n_pages, status)
            lens[0].copy_(new)
            k, v = (torch.randn((R, 4, H, d)).half().cuda() for _ in range(2))
            B.isv_q8_write(h, pool, n_pages, tails[0], tables[0], most, most, lens[0], grow.cuda(), k, v, 4 * H * d, H * d, R, 4)
            for s in range(R):
                record[s] = tuple(np.concatenate([old, x[s, :grow[s]].double().cpu().numpy().transpose(1, 0, 2)], 1)
                                  for old, x in zip(record[s], (k, v)))
            q = torch.randn((R, Hq, d)).half().cuda()
            out = torch.empty((R, Hq, d), device="cuda")
            B.isv_q8_attn(h, pool, n_pages, tails[0], tables[0], most, most, lens[0], q, None, out, R)
            for s in range(R):
                rows = []
                for x in record[s]:
                    full = x.shape[1] // 16 * 16
                    blocks = x[:, :full].reshape(H, -1, 16, d)
                    codes, scale = oq.quantise(blocks, fmt)
                    rows.append(np.concatenate([(oq.decode(codes, fmt) * scale.astype(np.float64)[..., None, None]).reshape(H, full, d),
                                                x[:, full:]], 1))
                qs = q[s].double().cpu().numpy()
                assert np.max(np.abs(out[s].double().cpu().numpy() - oq.attend(qs, *rows))) <= oq.attend_error(qs, *rows), (step, s)
            if step % 3 == 1:
                parent = rng.integers(0, R, R)
                parent[rng.random(R) < 0.2] = -1
                B.isv_pages_fork(tables[0], lens[0], R, _dev(parent), tables[1], lens[1], R, most, most, 0, n_pages, src, dst, status)
                B.isv_pages_copy(tails[1], R, tails[0], R, tail, 1, 0, 0, _dev(parent), None, R, None, status)
                tables.reverse(), lens.reverse(), tails.reverse()
                record = [record[p] if p >= 0 else (np.zeros((H, 0, d)),) * 2 for p in parent]
            if step % 5 == 4:
                B.isv_pages_compact(tables[0], lens[0], R, most, most, 0, n_pages, tables[0], src, dst, n_pages // 2, counts, status)
                B.isv_pages_copy(pool, n_pages, pool, n_pages, page, 1, 0, 0, src, dst, n_pages // 2, counts[1:], status)
        assert status.item() == 0 and B.isv_q8_status(h) == 0
    finally:
        B.isv_q8_free(h)


def test_forked_rows_of_a_sixteen_bit_pool_go_their_own_ways():
    """fork + copy next to isv_attn_decode_static: siblings share complete pages, their open blocks are their own."""
    R, H, d, most, n_pages = 4, 2, 64, 3, 20
    pool = torch.randn((n_pages, 2, H, 16, d), device="cuda").half()
    before = pool.clone()
    table, lens = _dev([[4, 7, 9], [2, 1, 0], [3, 5, 6], [8, 10, 11]]), _dev([40, 16, 0, 5])
    out, lens_out, a, b, status = torch.empty_like(table), *(torch.empty_like(lens) for _ in range(3)), _dev([0])
    parent = [0, 0, 0, 1]
    B.isv_pages_fork(table, lens, R, _dev(parent), out, lens_out, R, most, most, 1, n_pages, a, b, status)
    B.isv_pages_copy(pool, n_pages, pool, n_pages, 2 * H * 16 * d * 2, 1, 0, 0, a, b, R, None, status)
    assert out.tolist() == [[4, 7, 9], [4, 7, 0], [4, 7, 1], [2, -1, -1]] and status.item() == 0
    assert torch.equal(pool[0], before[9]) and torch.equal(pool[1], before[9])
    q = torch.randn((1, 2, d), device="cuda").half().expand(R, 2, d).contiguous()
    res = torch.empty((R, 2, d), device="cuda")
    B.isv_attn_decode_static(pool, n_pages, out, most, lens_out, R, most, 2, H, d, 16, B.ISV_F16, 0, q, None, res, status)
    torch.cuda.synchronize()
    assert torch.equal(res[0], res[1]) and torch.equal(res[0], res[2]) and not torch.equal(res[0], res[3]) and status.item() == 0
