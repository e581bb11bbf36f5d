"""Storing chunks with the position rotation, verification of drafts, and the calls together, through the C ABI."""
import numpy as np
import pytest
import torch

from _chunk import CODE, Case, dev, f64
from oracle import chunk as oc
from paper_2504_11816_b200 import binding as B
from paper_2504_11816_b200 import workloads as W

pytestmark = pytest.mark.gpu


def _freq(rotary):
    return (10000.0 ** (-np.arange(rotary // 2) * 2 / max(rotary, 1))).astype(np.float32)


def _write(c, h, rotary, q_out=None, positions=None, axis=None, magnitude=1.0, q=True, stream=0):
    D = c.D
    B.isv_chunk_write(h, D["pool"], c.n_pages, D["table"], c.stride, c.blocks, D["lens"], D["news"], D["firsts"], c.rows, D["k"], D["v"],
                      D["k"].stride(0), D["q"] if q else None, D["q"].stride(0) if q else 0, q_out, dev(_freq(rotary), torch.float32),
                      positions, axis, magnitude, c.S, c.T, stream)


def _check(c, pool, q, rotary, pairs, positions=None, axis=None, magnitude=1.0, q_before=None):
    """Every byte of the pool and of q: turned elements within their tolerance, everything else bit for bit."""
    half = oc.HALF_STEP[c.dtype]
    before, after = c.pool.clone(), pool.cpu()
    w = torch.tensor(oc.places(c.d))
    bits = lambda x: x.contiguous().view(torch.int16)  # noqa: E731
    want_q = (q_before if q_before is not None else c.q).clone()
    for s in range(c.S):
        n = int(c.news[s])
        if not n:
            continue
        rows = slice(c.firsts[s], c.firsts[s] + n)
        pos = c.starts[s] + np.arange(n)
        if positions is not None:
            pos = positions[:, rows]
        k, koff = oc.rotate(f64(c.k[rows]), pos, _freq(rotary), rotary, pairs, axis, magnitude)
        qq, qoff = oc.rotate(f64(c.q[rows]), pos, _freq(rotary), rotary, pairs, axis, magnitude)
        if q is not None:
            got = f64(q[rows])
            assert (np.abs(got - qq) <= qoff + half * (np.abs(qq) + qoff) + 2.0 ** -25)[..., :rotary].all()
            assert torch.equal(bits(q.cpu()[rows][..., rotary:]), bits(c.q[rows][..., rotary:]))
            want_q[rows] = q.cpu()[rows]
        for t in range(n):
            j = int(c.starts[s]) + t
            page = int(c.table[s, j // 16])
            if not 0 <= page < c.n_pages:
                continue
            row = torch.gather(after[page, 0, :, j % 16], -1, w[j % 16].expand(c.H, c.d))
            got = f64(row)
            assert (np.abs(got - k[t]) <= koff[t] + half * (np.abs(k[t]) + koff[t]) + 2.0 ** -25)[..., :rotary].all()
            assert torch.equal(bits(row[..., rotary:]), bits(c.k[rows][t][..., rotary:]))
            v = torch.gather(after[page, 1, :, j % 16], -1, w[j % 16].expand(c.H, c.d))
            assert torch.equal(bits(v), bits(c.v[rows][t]))
            before[page, :, :, j % 16] = after[page, :, :, j % 16]
    assert torch.equal(bits(before), bits(after))                             # nothing else was written
    if q is not None:
        assert torch.equal(bits(q.cpu()), bits(want_q))


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("pairs", [B.ISV_ROTARY_HALVES, B.ISV_ROTARY_ADJACENT])
@pytest.mark.parametrize("d,rotary", [(64, 64), (64, 32), (64, 0), (80, 80), (80, 32), (80, 16), (128, 128), (128, 64), (128, 112)])
def test_rotation_and_places(d, rotary, pairs, dtype):
    for Hq, H, starts, news in ((4, 4, [0, 15, 33, 7], [1, 2, 40, 0]), (8, 1, [0], [1]), (3, 3, [100000], [5]), (14, 2, [5] * 50, [1] * 50)):
        c = Case(starts, news, Hq, H, d, dtype, seed=d + rotary)
        D, h = c.to_gpu(), c.handle(rotary_dim=rotary, rotary_pairs=pairs)
        try:
            q = torch.full((c.rows, Hq, d), 3.0, dtype=W.torch_dtype(dtype), device="cuda")
            _write(c, h, rotary, q)
            _check(c, D["pool"], q, rotary, pairs, q_before=torch.full((c.rows, Hq, d), 3.0).to(c.q.dtype))
            D = c.to_gpu()
            _write(c, h, rotary, q=False)                                     # keys and values alone
            _check(c, D["pool"], None, rotary, pairs)
            assert torch.equal(D["qkv"].cpu(), c.qkv)
            D = c.to_gpu()
            _write(c, h, rotary)                                              # queries in place
            _check(c, D["pool"], D["q"], rotary, pairs)
            assert torch.equal(D["k"].cpu(), c.k) and torch.equal(D["v"].cpu(), c.v)
            assert B.isv_chunk_status(h) == 0
        finally:
            B.isv_chunk_free(h)


@pytest.mark.parametrize("axes", [1, 2, 3, 4])
def test_positions_with_axes_and_magnitude(axes):
    rng = np.random.default_rng(axes)
    c = Case([3, 90], [50, 7], 4, 2, 128, "bf16")
    positions = rng.integers(-50, 3000, (axes, c.rows))
    axis = rng.integers(0, axes, 32)
    D, h = c.to_gpu(), c.handle(rotary_dim=64, rotary_pairs=B.ISV_ROTARY_ADJACENT, rotary_axes=axes)
    try:
        q = torch.zeros((c.rows, 4, 128), dtype=torch.bfloat16, device="cuda")
        _write(c, h, 64, q, dev(positions), dev(axis, torch.uint8), 1.25)
        _check(c, D["pool"], q, 64, B.ISV_ROTARY_ADJACENT, positions, axis, 1.25, q_before=torch.zeros_like(c.q))
        _write(c, h, 64, q, dev(positions), None, 1.25)                       # all pairs by the first axis
        _check(c, D["pool"], q, 64, B.ISV_ROTARY_ADJACENT, positions, np.zeros(32, int), 1.25, q_before=torch.zeros_like(c.q))
    finally:
        B.isv_chunk_free(h)


def test_far_positions_keep_their_angle():
    c = Case([0], [4], 2, 1, 64, "f16")
    positions = np.zeros((1, c.rows), np.int64)
    positions[0, c.firsts[0]:c.firsts[0] + 4] = [2 ** 31 - 1, 2 ** 30 + 12345, -2 ** 31, 123456789]
    D, h = c.to_gpu(), c.handle(rotary_dim=64)
    try:
        q = torch.zeros((c.rows, 2, 64), dtype=torch.float16, device="cuda")
        _write(c, h, 64, q, dev(positions))
        _check(c, D["pool"], q, 64, B.ISV_ROTARY_HALVES, positions, np.zeros(32, int), q_before=torch.zeros_like(c.q))
    finally:
        B.isv_chunk_free(h)


def test_tokens_without_a_page_and_bad_lengths():
    c = Case([10, 60], [20, 40], 4, 2, 64, "f16")
    c.table[0, 1] = B.ISV_BLOCK_NONE
    c.table[1, 4] = c.n_pages
    D, h = c.to_gpu(), c.handle(rotary_dim=64)
    try:
        q = torch.zeros((c.rows, 4, 64), dtype=torch.float16, device="cuda")
        _write(c, h, 64, q)
        _check(c, D["pool"], q, 64, B.ISV_ROTARY_HALVES, q_before=torch.zeros_like(c.q))
        with pytest.raises(B.IsvError) as ei:
            B.isv_chunk_status(h)
        assert ei.value.code == B.ISV_EDEVICE_STATUS and B.isv_chunk_status(h) == 0
        for what, value in (("lens", -1), ("lens", 16 * c.blocks + 1), ("news", 100), ("news", -7), ("firsts", -2), ("firsts", c.rows - 3)):
            D = c.to_gpu()
            D[what][0] = value
            _write(c, h, 64, q)
            with pytest.raises(B.IsvError) as ei:
                B.isv_chunk_status(h)
            assert ei.value.code == B.ISV_EDEVICE_STATUS
    finally:
        B.isv_chunk_free(h)


def test_write_is_captured_and_replayed():
    c = Case([100, 7], [1, 1], 8, 2, 128, "bf16")
    D, h = c.to_gpu(), c.handle(rotary_dim=128)
    try:
        q = torch.zeros((c.rows, 8, 128), dtype=torch.bfloat16, device="cuda")
        freq = dev(_freq(128), torch.float32)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            B.isv_chunk_write(h, D["pool"], c.n_pages, D["table"], c.stride, c.blocks, D["lens"], D["news"], D["firsts"], c.rows, D["k"], D["v"],
                              D["k"].stride(0), D["q"], D["q"].stride(0), q, freq, None, None, 1.0, c.S, c.T,
                              torch.cuda.current_stream().cuda_stream)
        graph.replay()
        torch.cuda.synchronize()
        _check(c, D["pool"], q, 128, B.ISV_ROTARY_HALVES, q_before=torch.zeros_like(c.q))
    finally:
        B.isv_chunk_free(h)


# ---------------------------------------------------------------- drafts

def _drafts(S, K, V, dtype, seed, given=True):
    g = torch.Generator().manual_seed(seed)
    rng = np.random.default_rng(seed)
    t = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[dtype]
    x = torch.randn((S, K + 1, V), generator=g) * 2
    target = torch.softmax(x, -1).to(t)
    near = torch.softmax(x[:, :K] + torch.randn((S, K, V), generator=g) * 0.7, -1)
    drafted = torch.multinomial(near.flatten(0, 1), 1, generator=g).view(S, K).int()
    counts = rng.integers(0, K + 1, S)
    u = torch.rand((S, K + 1), generator=g)
    return target, near.to(t) if given else None, drafted, counts, u


def _verify(target, draft, drafted, counts, u, V, dtype, firsts=None, n_rows=None, lens=None, status=None, stream=0):
    S, K = drafted.shape
    tokens = torch.full((S, K + 1), 77, dtype=torch.int32, device="cuda")
    accepted, lens_out = (torch.full((S,), 77, dtype=torch.int32, device="cuda") for _ in range(2))
    B.isv_draft_verify(target, firsts, n_rows if n_rows is not None else S * (K + 1), draft, V, CODE[dtype], drafted, counts, u, lens, S, K,
                       tokens, accepted, lens_out if lens is not None else None, status, stream)
    return tokens.cpu().numpy(), accepted.cpu().numpy(), lens_out.cpu().numpy()


def _hold(got, target, draft, drafted, counts, u):
    tokens, accepted, _ = got
    S, K = drafted.shape
    for s in range(S):
        n = int(counts[s])
        a, t = oc.verify(f64(target[s][:n + 1]), None if draft is None else f64(draft[s][:n]), drafted[s][:n].tolist(),
                         u[s][:n].tolist() + [float(u[s, K])])
        want = drafted[s][:a].tolist() + [t] + [-1] * (K - a)
        assert accepted[s] == a and tokens[s].tolist() == want, (s, accepted[s], a, tokens[s], want)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("given", [True, False])
@pytest.mark.parametrize("S,K,V", [(1, 1, 1), (1, 1, 2), (3, 4, 7), (5, 2, 511), (40, 3, 1000), (2, 8, 50257), (1, 4, 32000), (200, 1, 4099),
                                   (3, 40, 2048), (2, 3, 151936), (1, 1, 1 << 20)])
def test_drafts_are_verified(S, K, V, given, dtype):
    target, draft, drafted, counts, u = _drafts(S, K, V, dtype, S + K + V, given)
    lens = np.random.default_rng(V).integers(50, 90, S)
    status = dev([0])
    got = _verify(target.cuda(), draft.cuda() if given else None, drafted.cuda(), dev(counts), u.cuda(), V, dtype, lens=dev(lens), status=status)
    _hold(got, target, draft, drafted, counts, u)
    assert np.array_equal(got[2], lens - counts + got[1]) and status.item() == 0


def test_every_border_of_a_draw():
    """Uniforms from 0 to the number below 1 over a row whose probabilities are exact: the index is the definition's."""
    V = 700
    p = np.random.default_rng(0).integers(0, 3, V) / 1024.0                   # a third of them zero
    target = torch.tensor(np.stack([p, p]), dtype=torch.float32)[None].repeat(64, 1, 1)
    u = torch.zeros((64, 2))
    u[:, 1] = torch.tensor(np.append(np.arange(63) / 63, 1 - 2.0 ** -24), dtype=torch.float32)
    drafted = torch.zeros((64, 1), dtype=torch.int32)
    got = _verify(target.cuda(), None, drafted.cuda(), dev(np.zeros(64)), u.cuda(), V, "f32")
    _hold(got, target, None, drafted, np.zeros(64, int), u)
    bad = u.clone()
    bad[0, 1], bad[1, 1], bad[2, 1] = -1.0, 1.0, float("nan")                 # clamped: the first and the last with any weight
    tokens = _verify(target.cuda(), None, drafted.cuda(), dev(np.zeros(64)), bad.cuda(), V, "f32")[0]
    some = np.flatnonzero(p)
    assert tokens[:3, 0].tolist() == [some[0], some[-1], some[-1]]


def test_zero_probabilities_bad_tokens_and_counts():
    V, K, S = 300, 3, 6
    target, draft, drafted, counts, u = _drafts(S, K, V, "f32", 9)
    counts[:] = K
    target[0] = 0                                                              # nothing to draw from
    draft[1] = target[1, :K]                                                   # accepted whatever u is: equal probabilities
    drafted[2, 0] = V
    drafted[3, 1] = -1
    target[4, 0, 5:] = float("nan")
    target[4, 0, :5] = -1.0
    target[4, 0, 3] = 0.25
    status = dev([0])
    got = _verify(target.cuda(), draft.cuda(), drafted.cuda(), dev(counts), u.cuda(), V, "f32", status=status)
    _hold(got, target, draft, drafted, counts, u)
    assert got[0][0].tolist() == [-1] * 4 and got[1][1] == K and got[1][2] == 0 and got[1][3] <= 1 and got[0][4, 0] == 3
    assert status.item() == B.ISV_STATUS_BAD_TOKEN
    for n in (-4, K + 1):
        status.zero_()
        counts[5] = n
        again = _verify(target.cuda(), draft.cuda(), drafted.cuda(), dev(counts), u.cuda(), V, "f32", status=status)
        assert status.item() == B.ISV_STATUS_BAD_TOKEN | B.ISV_STATUS_BAD_LENGTH
        counts[5] = min(max(n, 0), K)
        _hold(again, target, draft, drafted, counts, u)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("V", [64, 1003])
def test_probabilities_that_are_negative_or_no_number_count_as_zero(V, dtype):
    S, K = 60, 3
    target, draft, drafted, counts, u = _drafts(S, K, V, dtype, V)
    g = torch.Generator().manual_seed(V)
    for x in (target, draft):
        odd = torch.rand(x.shape, generator=g)
        x[odd < 0.2] *= -1
        x[odd > 0.9] = float("nan")
    for s in range(0, S, 2):                                                   # drafts that their model gave nothing
        draft[s, 0, drafted[s, 0]] = (-1.0, float("nan"))[s // 2 % 2]
    counts[:30] = K
    got = _verify(target.cuda(), draft.cuda(), drafted.cuda(), dev(counts), u.cuda(), V, dtype)
    _hold(got, target, draft, drafted, counts, u)
    got = _verify(target.cuda(), None, drafted.cuda(), dev(counts), u.cuda(), V, dtype)
    _hold(got, target, None, drafted, counts, u)


def test_target_rows_at_their_starts():
    """Rows of sequences one behind the other; rows that are not there cost their drafts, or the token."""
    S, K, V = 5, 3, 1001
    target, draft, drafted, counts, u = _drafts(S, K, V, "bf16", 3)
    counts[:] = [3, 0, 2, 1, 3]
    firsts, rows = [], []
    for s in (4, 2, 0, 1, 3):
        firsts.append((s, sum(len(r) for r in rows)))
        rows.append(target[s, :counts[s] + 1])
    starts = np.array([f for _, f in sorted(firsts)])
    packed = torch.cat(rows).cuda()
    args = (draft.cuda(), drafted.cuda(), dev(counts), u.cuda(), V, "bf16")
    _hold(_verify(packed, *args, firsts=dev(starts), n_rows=len(packed)), target, draft, drafted, counts, u)
    status = dev([0])
    tokens, accepted, _ = _verify(packed, *args, firsts=dev(starts), n_rows=len(packed) - 1, status=status)     # the last row of sequence 3
    assert status.item() == B.ISV_STATUS_BAD_LENGTH and accepted[3] == 0 and tokens[3, 0] >= 0
    for start in (-1, len(packed), 2 ** 31 - 1):
        status.zero_()
        starts[3] = start
        tokens, accepted, _ = _verify(packed, *args, firsts=dev(starts), n_rows=len(packed), status=status)
        assert status.item() & B.ISV_STATUS_BAD_LENGTH and accepted[3] == 0 and tokens[3].tolist() == [-1] * 4
        rest = [0, 1, 2, 4]
        _hold((tokens[rest], accepted[rest], None), target[rest], draft[rest], drafted[rest], counts[rest], u[rest])


def test_verification_on_a_stream_in_a_graph_and_unaligned():
    S, K, V = 3, 2, 4096
    target, draft, drafted, counts, u = _drafts(S, K, V, "f32", 1)
    flat = torch.zeros(target.numel() + 1, device="cuda")
    flat[1:] = target.flatten().cuda()
    side = torch.cuda.Stream()
    dd, xd, cd, ud = draft.cuda(), drafted.cuda(), dev(counts), u.cuda()
    torch.cuda.synchronize()
    tokens = torch.full((S, K + 1), 77, dtype=torch.int32, device="cuda")
    accepted = torch.full((S,), 77, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    B.isv_draft_verify(flat.data_ptr() + 4, None, S * (K + 1), dd, V, B.ISV_F32, xd, cd, ud, None, S, K, tokens, accepted, None, None, side.cuda_stream)
    side.synchronize()
    _hold((tokens.cpu().numpy(), accepted.cpu().numpy(), None), target, draft, drafted, counts, u)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.isv_draft_verify(flat.data_ptr() + 4, None, S * (K + 1), dd, V, B.ISV_F32, xd, cd, ud, None, S, K, tokens, accepted, None, None,
                           torch.cuda.current_stream().cuda_stream)
    u2 = torch.rand(u.shape)
    ud.copy_(u2)
    graph.replay()
    torch.cuda.synchronize()
    _hold((tokens.cpu().numpy(), accepted.cpu().numpy(), None), target, draft, drafted, counts, u2)


# ---------------------------------------------------------------- the calls together

@pytest.mark.parametrize("dtype,Hq,H,d", [("bf16", 8, 2, 128), ("f16", 4, 4, 80)])
def test_a_generation_with_drafts(dtype, Hq, H, d):
    """A prompt, then steps that store a token and its drafts, attend, verify, and give back the pages of what did not stand:
    the outputs are those of a cache that only ever held the tokens that stood."""
    rng = np.random.default_rng(0)
    t = W.torch_dtype(dtype)
    S, K, V, pages, blocks = 3, 4, 50, 64, 12
    table = torch.full((S, blocks), -1, dtype=torch.int32, device="cuda")
    pool = torch.full((pages, 2, H, 16, d), float("nan"), dtype=t, device="cuda")
    freq = dev(_freq(d), torch.float32)
    h = B.isv_chunk_create(q_heads=Hq, kv_heads=H, head_dim=d, dtype=CODE[dtype], max_seqs=S, rotary_dim=d)
    lens = torch.zeros(S, dtype=torch.int32, device="cuda")
    kept = [[np.zeros((H, 0, d)), np.zeros((H, 0, d))] for _ in range(S)]
    try:
        for step in range(12):
            news = rng.integers(1, 60, S) if step == 0 else rng.integers(1, K + 2, S)
            T, firsts = int(news.max()), np.append(0, np.cumsum(news)[:-1])
            rows = int(news.sum())
            qkv = torch.tensor(rng.standard_normal((rows, Hq + 2 * H, d)), dtype=t, device="cuda")
            q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + H], qkv[:, Hq + H:]
            grown, nd, fd = lens + dev(news), dev(news), dev(firsts)
            B.isv_pages_resize(table, lens, grown, S, blocks, blocks, 1, pages)
            turned = torch.empty((rows, Hq, d), dtype=t, device="cuda")
            B.isv_chunk_write(h, pool, pages, table, blocks, blocks, grown, nd, fd, rows, k, v, k.stride(0), q, q.stride(0), turned, freq, None,
                              None, 1.0, S, T)
            out = torch.empty((rows, Hq, d), device="cuda")
            B.isv_chunk_attn(h, pool, pages, table, blocks, blocks, grown, nd, fd, rows, turned, Hq * d, None, None, 0, None, out, S, T)
            # "probabilities" from the outputs: of the last 1 + drafts tokens of each sequence
            counts = np.zeros(S, int) if step == 0 else news - 1
            target = torch.softmax(out[:, 0, :V] * 4, -1).contiguous()
            starts = firsts + news - 1 - counts
            drafted = rng.integers(0, V, (S, K))
            u = rng.random((S, K + 1)) * (0.05 if step % 2 else 1.0)
            tokens, accepted, keep = (torch.empty(x, dtype=torch.int32, device="cuda") for x in ((S, K + 1), S, S))
            B.isv_draft_verify(target, dev(starts), rows, None, V, B.ISV_F32, dev(drafted), dev(counts), dev(u, torch.float32), grown, S, K, tokens,
                               accepted, keep)
            B.isv_pages_resize(table, grown, keep, S, blocks, blocks, 1, pages)
            for s in range(S):
                r = slice(firsts[s], firsts[s] + news[s])
                pos = int(lens[s]) + np.arange(news[s])
                kk, koff = oc.rotate(f64(k[r]), pos, _freq(d), d, oc.HALVES)
                qq, _ = oc.rotate(f64(q[r]), pos, _freq(d), d, oc.HALVES)
                K64 = np.concatenate([kept[s][0], np.swapaxes(kk, 0, 1)], 1)
                V64 = np.concatenate([kept[s][1], np.swapaxes(f64(v[r]), 0, 1)], 1)
                n = K64.shape[1]
                want, _ = oc.attend(qq, K64, V64, pos, oc.visible(pos, n), 1 / np.sqrt(d))
                # rounding q and k to 16 bits moves a score by up to two half steps of sum |q k|, an output by twice that of the largest |v|
                most = max((np.abs(qq[:, i]) @ np.abs(K64[i // (Hq // H)]).T).max() for i in range(Hq)) / np.sqrt(d)
                move = 2 * oc.HALF_STEP[dtype] * most
                assert np.abs(f64(out[r]) - want).max() <= 2 * move * np.abs(V64).max() + 1e-4
                a, tok = oc.verify(f64(target[starts[s]:starts[s] + counts[s] + 1]), None, drafted[s][:counts[s]],
                                   np.append(u[s][:counts[s]], u[s][K]).astype(np.float32))
                assert int(accepted[s]) == a and tokens[s].tolist() == drafted[s][:a].tolist() + [tok] + [-1] * (K - a)
                n = int(lens[s]) + int(news[s]) - int(counts[s]) + a
                assert int(keep[s]) == n
                kept[s] = [K64[:, :n], V64[:, :n]]
            lens = keep
            if int(lens.max()) > 16 * blocks - K - 2:
                break
        assert B.isv_chunk_status(h) == 0
    finally:
        B.isv_chunk_free(h)
