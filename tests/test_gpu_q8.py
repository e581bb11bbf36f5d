"""The 8-bit KV cache against the fp64 reference, through the C ABI: stored bytes exactly, attention within the error
that fp32 arithmetic can make (oracle.q8.attend_error)."""
import numpy as np
import pytest
import torch

from oracle import q8 as oq
from paper_2504_11816_b200 import binding as B
from paper_2504_11816_b200 import workloads as W

pytestmark = pytest.mark.gpu

HALF_STEP = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}     # half a step of the 16-bit type, relative


class Cache:
    """A caller's buffers for one layer, the handle, and the logical rows behind them."""

    def __init__(self, lens, q_heads, kv_heads, d, dtype="f16", fmt=B.ISV_Q8_INT8, seed=0, spare=3, max_ctas=0, make=None):
        self.lens, self.Hq, self.H, self.d, self.fmt = list(lens), q_heads, kv_heads, d, fmt
        self.dtype, self.dt = dtype, W.torch_dtype(dtype)
        g = torch.Generator().manual_seed(seed)
        self.k, self.v = [], []
        for n in self.lens:
            for rows in (self.k, self.v):
                x = torch.randn((n, kv_heads, d), generator=g)
                big = torch.rand(x.shape, generator=g) < 0.01
                x = torch.where(big, 8 * x, x)
                rows.append((make(x) if make else x).to(self.dt))
        self.most = max([n // 16 for n in self.lens] + [1]) + 1
        self.n_pages = sum(n // 16 for n in self.lens) + spare + 1
        self.page, self.tail = B.isv_q8_sizes(kv_heads, d)
        ids = torch.randperm(self.n_pages, generator=g).int()
        table = torch.full((len(self.lens), self.most + 1), B.ISV_BLOCK_NONE, dtype=torch.int32)
        at = 0
        for s, n in enumerate(self.lens):
            table[s, :n // 16] = ids[at:at + n // 16]
            at += n // 16
        self.table = table.cuda()
        self.pool = torch.full((self.n_pages, self.page), 0x7f, dtype=torch.uint8, device="cuda")
        self.tails = torch.full((len(self.lens), 2, kv_heads, 16, d), float("nan"), dtype=self.dt, device="cuda")
        self.q = torch.randn((len(self.lens), q_heads, d), generator=g).to(self.dt).cuda()
        self.h = B.isv_q8_create(q_heads=q_heads, kv_heads=kv_heads, head_dim=d, dtype=B.ISV_F16 if dtype == "f16" else B.ISV_BF16,
                                 format=fmt, max_seqs=max(1, len(self.lens)), max_ctas=max_ctas)

    def __enter__(self):
        return self

    def __exit__(self, *a):
        B.isv_q8_free(self.h)

    def write(self, upto, new, k=None, v=None, strides=None, T=None, stream=0):
        """Sequences get their rows [upto - new, upto)."""
        n = len(self.lens)
        T = max(list(new) + [1]) if T is None else T
        if k is None:
            k, v = (torch.zeros((n, T, self.H, self.d), dtype=self.dt) for _ in range(2))
            for s in range(n):
                k[s, :new[s]] = self.k[s][upto[s] - new[s]:upto[s]]
                v[s, :new[s]] = self.v[s][upto[s] - new[s]:upto[s]]
            k, v = k.cuda(), v.cuda()
        ss, ts = strides or (T * self.H * self.d, self.H * self.d)
        lens, news = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (list(upto), list(new)))
        B.isv_q8_write(self.h, self.pool, self.n_pages, self.tails, self.table, self.most + 1, self.most, lens, news, k, v, ss, ts,
                       n, T, stream)
        self.kept = (k, v, lens, news)

    def fill(self):
        self.write(self.lens, self.lens)
        return self

    def units(self, s):
        """Reference bytes [blocks][heads][unit] and the rows that attention sees, K, V [heads][n][d]."""
        n, full = self.lens[s], self.lens[s] // 16
        k, v = (x[s].double().numpy().reshape(n, self.H, self.d) for x in (self.k, self.v))
        kb, vb = (x[:16 * full].reshape(full, 16, self.H, self.d).transpose(0, 2, 1, 3) for x in (k, v))
        u, kd, vd = oq.unit(kb, vb, self.fmt)
        rows = [np.concatenate([b.transpose(1, 0, 2, 3).reshape(self.H, 16 * full, self.d), x[16 * full:].transpose(1, 0, 2)], 1)
                for b, x in ((kd, k), (vd, v))]
        return u, rows[0], rows[1]

    def check_bytes(self):
        pool = self.pool.cpu().numpy().reshape(self.n_pages, self.H, -1)
        tails = self.tails.cpu()
        table = self.table.cpu().numpy()
        used = set()
        for s, n in enumerate(self.lens):
            u, _, _ = self.units(s)
            for b in range(n // 16):
                page = pool[table[s, b]]
                codes = 32 * self.d
                assert np.array_equal(page[:, :codes], u[b][:, :codes]), (s, b)
                got = np.ascontiguousarray(page[:, codes:codes + 8]).view(np.float32)
                want = np.ascontiguousarray(u[b][:, codes:codes + 8]).view(np.float32)
                assert np.array_equal(got, want, equal_nan=True), (s, b)
                used.add(int(table[s, b]))
            r = n % 16
            assert torch.equal(tails[s, 0, :, :r], self.k[s][n - r:].transpose(0, 1)), s
            assert torch.equal(tails[s, 1, :, :r], self.v[s][n - r:].transpose(0, 1)), s
        for p in set(range(self.n_pages)) - used:
            assert (pool[p] == 0x7f).all(), p            # pages that no sequence owns are left alone

    def attend(self, stream=0, f32=True, lens=None, n=None):
        out = torch.full(self.q.shape, float("nan"), dtype=self.dt, device="cuda")
        out32 = torch.full(self.q.shape, float("nan"), device="cuda") if f32 else None
        lens = torch.tensor(self.lens if lens is None else lens, dtype=torch.int32, device="cuda")
        torch.cuda.synchronize()
        B.isv_q8_attn(self.h, self.pool, self.n_pages, self.tails, self.table, self.most + 1, self.most, lens, self.q, out, out32,
                      len(self.lens) if n is None else n, stream)
        torch.cuda.synchronize()
        return out, out32

    def check(self, out, out32, rows=None):
        for s in range(len(self.lens)) if rows is None else rows:
            _, K, V = self.units(s)
            q = self.q[s].double().cpu().numpy()
            want, tol = oq.attend(q, K, V), oq.attend_error(q, K, V)
            if out32 is not None:
                got = out32[s].double().cpu().numpy()
                assert np.all(np.abs(got - want) <= tol), (s, self.lens[s], np.max(np.abs(got - want)), tol)
            got = out[s].double().cpu().numpy()
            room = HALF_STEP[self.dtype] * (np.abs(want) + tol) + 2.0 ** -25      # and half a step of the smallest fp16 numbers
            assert np.all(np.abs(got - want) <= tol + room), (s, self.lens[s])


FORMATS = [B.ISV_Q8_INT8, B.ISV_Q8_E4M3]


# ---------------------------------------------------------------- storing

@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("d,dtype,heads", [(64, "f16", 3), (80, "bf16", 2), (128, "f16", 1), (128, "bf16", 8), (80, "f16", 32)])
def test_prompts_are_stored_exactly(d, dtype, heads, fmt):
    with Cache([0, 1, 15, 16, 17, 47, 160, 333], heads, heads, d, dtype, fmt, seed=d + heads) as c:
        c.fill().check_bytes()
        assert B.isv_q8_status(c.h) == 0


@pytest.mark.parametrize("fmt", FORMATS)
def test_token_by_token_and_in_chunks_store_the_same(fmt):
    lens = [70, 33, 0, 5, 64]
    with Cache(lens, 4, 2, 64, "bf16", fmt, seed=5) as c:
        for t in range(1, 71):                                  # one token a call; finished sequences sit out
            c.write([min(t, n) for n in lens], [1 if t <= n else 0 for n in lens])
        c.check_bytes()
    for cut in (3, 16, 21, 40):                                 # chunks that start and end anywhere
        with Cache(lens, 4, 2, 64, "bf16", fmt, seed=5) as c:
            done = [0] * len(lens)
            while done != lens:
                new = [min(cut, n - x) for n, x in zip(lens, done)]
                done = [x + m for x, m in zip(done, new)]
                c.write(done, new)
            c.check_bytes()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("fmt", FORMATS)
def test_values_next_to_a_border_tiny_huge_and_zero_blocks(dtype, fmt):
    top = 60000.0 if dtype == "f16" else 3.0e38
    low = 2.0 ** -24 if dtype == "f16" else 2.0 ** -133

    def make(x):
        n = x.shape[0] // 16
        for b in range(n):
            y = x[16 * b:16 * b + 16]
            if b == 0:
                y.zero_()
            elif b == 1:
                y.mul_(low * 3)                                 # the smallest numbers of the type
            elif b == 2:
                y.clamp_(-8, 8).mul_(top / 8)
            elif b == 3:                                        # x / scale is a tie wherever x = absmax / 2
                y.copy_(torch.where(y > 0, torch.full_like(y, 1.5), torch.full_like(y, 0.75)))
            elif b == 4:                                        # all sixteen-bit numbers of a range
                y.copy_(torch.linspace(0, 1, y.numel()).view(y.shape))
            elif b == 5:
                y[3, 0, 7] = float("inf")
            elif b == 6:
                y[9, 1, 2] = float("nan")
            elif b == 7:
                y.mul_(1e-30 if dtype == "bf16" else 1e-3)
                y[0, 0, 0] = top                                # everything else rounds to zero
        return x
    with Cache([8 * 16 + 3], 2, 2, 128, dtype, fmt, seed=9, make=make) as c:
        c.fill().check_bytes()


def test_rows_with_strides_a_padded_batch_and_null_new_lens():
    with Cache([40, 0, 40], 4, 2, 80, "f16", seed=3) as c:
        fused = torch.full((3, 40, 3, 2, 80), float("nan"), dtype=torch.float16, device="cuda")   # [q | k | v] rows
        for s in (0, 2):
            fused[s, :, 1], fused[s, :, 2] = c.k[s].cuda(), c.v[s].cuda()
        row = 3 * 2 * 80
        c.write([40, 0, 40], [40, 0, 40], k=fused[0, 0, 1].data_ptr(), v=fused[0, 0, 2].data_ptr(), strides=(40 * row, row), T=40)
        c.check_bytes()
        assert B.isv_q8_status(c.h) == 0
    with Cache([32, 32], 2, 2, 64, seed=4) as c:
        k, v = (torch.stack(x).cuda() for x in (c.k, c.v))
        lens = torch.tensor([32, 32], dtype=torch.int32, device="cuda")
        B.isv_q8_write(c.h, c.pool, c.n_pages, c.tails, c.table, c.most + 1, c.most, lens, None, k, v, 32 * 128, 128, 2, 32)
        c.check_bytes()


def test_bad_pages_and_lengths_are_flagged_and_skipped():
    with Cache([32, 48, 20, 16], 2, 2, 64, seed=6) as c:
        good = c.table.clone()
        c.table[0, 1] = c.n_pages
        c.table[1, 0] = -7
        c.write(c.lens, c.lens)
        with pytest.raises(B.IsvError) as ei:
            B.isv_q8_status(c.h)
        assert ei.value.code == B.ISV_EDEVICE_STATUS and "0x1" in ei.value.message
        assert B.isv_q8_status(c.h) == 0                        # reported once
        c.table.copy_(good)
        c.fill()
        lens = list(c.lens)
        for bad in (-1, 16 * c.most + 16):
            out, out32 = c.attend(lens=lens[:2] + [bad] + lens[3:])
            assert torch.isfinite(out32[[0, 1, 3]]).all()
            c.check(out, out32, rows=[0, 1, 3])
            with pytest.raises(B.IsvError) as ei:
                B.isv_q8_status(c.h)
            assert "0x4" in ei.value.message or "0x5" in ei.value.message
        # a block without a page is left out
        c.table[1, 1] = B.ISV_BLOCK_NONE
        out, out32 = c.attend()
        assert B.isv_q8_status(c.h) == 0
        _, K, V = c.units(1)
        keep = np.r_[0:16, 32:48]
        q = c.q[1].double().cpu().numpy()
        want = oq.attend(q, K[:, keep], V[:, keep])
        assert np.max(np.abs(out32[1].double().cpu().numpy() - want)) <= oq.attend_error(q, K, V)
        # more new tokens than the sequence has
        c.table.copy_(good)
        c.write(c.lens, [33, 48, 20, 16], T=48)
        with pytest.raises(B.IsvError):
            B.isv_q8_status(c.h)


def test_calls_with_a_handle_refuse_bad_arguments():
    with Cache([16], 2, 2, 64) as c:
        lens = torch.tensor([16], dtype=torch.int32, device="cuda")
        attn = dict(h=c.h, pool=c.pool, n_pages=c.n_pages, tails=c.tails, block_table=c.table, table_stride=2, max_blocks_per_seq=2,
                    seq_lens=lens, q=c.q, out=c.q.clone(), out_f32=None, n_seqs=1)
        write = {k: v for k, v in attn.items() if k not in ("q", "out", "out_f32")} | dict(
            new_lens=lens, k=c.q, v=c.q, seq_stride=2048, token_stride=128, T=16)
        for fn, base in ((B.isv_q8_attn, attn), (B.isv_q8_write, write)):
            for kw in (dict(pool=None), dict(tails=None), dict(block_table=None), dict(seq_lens=None), dict(n_seqs=2), dict(n_seqs=-1),
                       dict(n_pages=0), dict(max_blocks_per_seq=0), dict(table_stride=1), dict(pool=c.pool.data_ptr() + 8),
                       dict(tails=c.tails.data_ptr() + 2)):
                with pytest.raises(B.IsvError) as ei:
                    fn(**(base | kw))
                assert ei.value.code == B.ISV_EINVAL, kw
            fn(**(base | dict(n_seqs=0)))
        for kw in (dict(q=None), dict(out=None), dict(q=c.q.data_ptr() + 2), dict(out=c.q.data_ptr() + 2)):
            with pytest.raises(B.IsvError):
                B.isv_q8_attn(**(attn | kw))
        for kw in (dict(k=None), dict(v=None), dict(T=-1), dict(seq_stride=4), dict(token_stride=12), dict(token_stride=-128),
                   dict(k=c.q.data_ptr() + 2)):
            with pytest.raises(B.IsvError):
                B.isv_q8_write(**(write | kw))
        B.isv_q8_write(**(write | dict(T=0)))
        assert B.isv_q8_status(c.h) == 0


# ---------------------------------------------------------------- attention

@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("hq,hkv,d", [(2, 2, 64), (8, 4, 64), (5, 5, 80), (6, 2, 80), (4, 4, 128), (8, 1, 128), (14, 2, 128),
                                      (12, 1, 64), (32, 2, 128), (16, 1, 80), (17, 1, 64), (24, 1, 128), (40, 1, 80)])
def test_attention_matches_the_reference(hq, hkv, d, dtype, fmt):
    with Cache([0, 1, 2, 15, 16, 17, 31, 32, 33, 100, 257, 700], hq, hkv, d, dtype, fmt, seed=hq * 7 + d) as c:
        c.fill()
        c.check(*c.attend())
        out, _ = c.attend(f32=False)
        c.check(out, None)
        assert B.isv_q8_status(c.h) == 0


@pytest.mark.parametrize("lens,hq,hkv,d,dtype,fmt", [
    ([20011], 8, 2, 128, "bf16", B.ISV_Q8_E4M3),                    # one sequence over all SMs
    ([5000, 3, 0, 9000, 16], 4, 4, 80, "f16", B.ISV_Q8_INT8),
    ([64] * 300, 4, 1, 64, "f16", B.ISV_Q8_E4M3),                   # many short ones
    ([int(x) for x in np.random.default_rng(0).integers(0, 900, 64)], 8, 8, 128, "bf16", B.ISV_Q8_INT8)])
def test_attention_long_many_and_ragged(lens, hq, hkv, d, dtype, fmt):
    with Cache(lens, hq, hkv, d, dtype, fmt, seed=11) as c:
        c.fill()
        first = c.attend()
        c.check(*first, rows=range(0, len(lens), max(1, len(lens) // 24)))
        for _ in range(3):                                          # the same bits every time
            again = c.attend()
            assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


@pytest.mark.parametrize("max_ctas", [1, 2, 7, 100])
def test_attention_on_fewer_ctas(max_ctas):
    with Cache([300, 1, 0, 1000, 47], 8, 2, 128, "bf16", B.ISV_Q8_E4M3, seed=2, max_ctas=max_ctas) as c:
        c.fill()
        c.check(*c.attend())


@pytest.mark.parametrize("fmt", FORMATS)
def test_attention_with_scales_far_apart(fmt):
    """Blocks whose scales differ by up to 2^40, in both orders, and scores that move far."""
    made = [0]

    def make(x):                                                    # K and V rows are made in turn
        factors = [[0.05, 1, 4, 0.1, 6, 1, 8, 0.2], [2.0 ** e for e in (0, 20, -20, 3, -20, 20, 0, -9)]][made[0] % 2]
        made[0] += 1
        for b in range(x.shape[0] // 16):
            x[16 * b:16 * b + 16] *= factors[b % 8]
        return x
    with Cache([8 * 16 * 5, 130, 40], 4, 2, 64, "bf16", fmt, seed=8, make=make) as c:
        c.fill()
        c.check(*c.attend())


def test_a_block_with_an_infinity_gives_nan_and_harms_nobody_else():
    def make(x):
        if x.shape[0] == 64:
            x[20, 0, 3] = float("inf")
        return x
    with Cache([64, 70], 4, 2, 64, "f16", seed=1, make=make) as c:
        c.fill()
        out, out32 = c.attend()
        assert torch.isnan(out32[0, :2]).all() and torch.isfinite(out32[0, 2:]).all()
        c.check(out, out32, rows=[1])


def test_rows_behind_the_last_sequence_are_left_alone():
    with Cache([40, 50, 60], 4, 4, 64, seed=12) as c:
        c.fill()
        tails = c.tails.clone()
        out, out32 = c.attend(n=2)
        assert torch.isnan(out[2].float()).all() and torch.isnan(out32[2]).all()
        assert torch.equal(tails.view(torch.int16), c.tails.view(torch.int16))
        c.check(out, out32, rows=[0, 1])


def test_pages_beyond_four_gigabytes():
    with Cache([100, 37], 2, 2, 128, "f16", seed=13) as c:
        c.n_pages = (5 << 30) // c.page
        c.pool = torch.empty((c.n_pages, c.page), dtype=torch.uint8, device="cuda")
        c.table[c.table >= 0] = c.n_pages - 1 - c.table[c.table >= 0]
        c.fill()
        c.check(*c.attend())


def test_a_side_stream_and_a_replayed_graph():
    lens = [100, 0, 31, 16]
    with Cache(lens, 8, 2, 128, "bf16", B.ISV_Q8_E4M3, seed=14) as c:
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            c.write(lens, lens, stream=side.cuda_stream)
        side.synchronize()
        c.check_bytes()
        out = torch.zeros_like(c.q)
        n = torch.tensor(lens, dtype=torch.int32, device="cuda")
        torch.cuda.synchronize()
        args = (c.h, c.pool, c.n_pages, c.tails, c.table, c.most + 1, c.most, n, c.q, out, None, len(lens))
        B.isv_q8_attn(*args, side.cuda_stream)
        side.synchronize()
        c.check(out, None)
        # a captured step: append one token, attend; replayed until blocks complete, lengths advanced in the graph
        with Cache([n + 20 for n in lens], 8, 2, 128, "bf16", B.ISV_Q8_E4M3, seed=15) as e:
            e.write([n - 20 for n in e.lens], [n - 20 for n in e.lens])
            now = torch.tensor([n - 20 for n in e.lens], dtype=torch.int32, device="cuda")
            one = torch.ones(len(lens), dtype=torch.int32, device="cuda")
            k, v = (torch.empty((len(lens), 2, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
            out2 = torch.zeros_like(e.q)
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                st = torch.cuda.current_stream().cuda_stream
                now += 1
                B.isv_q8_write(e.h, e.pool, e.n_pages, e.tails, e.table, e.most + 1, e.most, now, one, k, v, 256, 256, len(lens), 1, st)
                B.isv_q8_attn(e.h, e.pool, e.n_pages, e.tails, e.table, e.most + 1, e.most, now, e.q, out2, None, len(lens), st)
            for t in range(20):
                for buf, rows in ((k, e.k), (v, e.v)):
                    buf.copy_(torch.stack([rows[s][e.lens[s] - 20 + t] for s in range(len(lens))]))
                graph.replay()
            torch.cuda.synchronize()
            e.check_bytes()
            e.check(out2, None)
            assert B.isv_q8_status(e.h) == 0


def test_two_handles_on_two_streams_at_once():
    lens = [1500, 700]
    with Cache(lens, 8, 1, 128, "f16", seed=16) as a, Cache(lens, 8, 1, 128, "f16", seed=17) as b:
        a.fill(), b.fill()
        n = torch.tensor(lens, dtype=torch.int32, device="cuda")
        outs = [torch.zeros(a.q.shape, device="cuda") for _ in range(2)]
        streams = [torch.cuda.Stream() for _ in range(2)]
        torch.cuda.synchronize()
        for _ in range(50):
            for c, o, st in zip((a, b), outs, streams):
                B.isv_q8_attn(c.h, c.pool, c.n_pages, c.tails, c.table, c.most + 1, c.most, n, c.q, None, o, 2, st.cuda_stream)
        torch.cuda.synchronize()
        for c, o in zip((a, b), outs):
            c.check(o.to(c.dt), o)


def test_as_many_sequences_as_a_handle_takes():
    lens = [int(x) for x in np.random.default_rng(3).integers(0, 40, 4096)]
    lens[5], lens[4095] = 300, 33
    with Cache(lens, 4, 2, 64, "f16", seed=18) as c:
        c.fill()
        out, out32 = c.attend()
        c.check(out, out32, rows=[0, 1, 5, 6, 1023, 1024, 2000, 4094, 4095])
        empty = [s for s, n in enumerate(lens) if n == 0]
        assert (out32[empty] == 0).all() and (out[empty] == 0).all()


def test_a_handle_serves_calls_of_fewer_sequences_and_other_pools():
    with Cache([33, 100, 7], 8, 2, 128, "bf16", B.ISV_Q8_E4M3, seed=19) as a, Cache([260], 8, 2, 128, "bf16", B.ISV_Q8_E4M3, seed=20) as b:
        a.fill()
        own, b.h = b.h, a.h                     # the second cache through the first one's handle
        b.fill().check_bytes()
        b.check(*b.attend())
        a.check(*a.attend())
        b.h = own


def test_queries_far_from_one_and_not_finite():
    """Rows of q of any size keep fp32 accuracy; an infinity or NaN in one head reaches that head only."""
    with Cache([64, 21], 8, 2, 128, "bf16", B.ISV_Q8_INT8, seed=21) as c:
        c.fill()
        c.q[0, 0] *= 1e-30
        c.q[0, 1] *= 1e-4
        c.q[0, 2] *= 20
        c.q[1, 3] = 0
        clean = c.attend()
        c.check(*clean)
        c.q[0, 5, 17] = float("nan")
        c.q[1, 7, 3] = float("inf")
        out, out32 = c.attend()
        assert torch.isnan(out32[0, 5]).all() and torch.isnan(out32[1, 7]).all()
        fine = torch.ones(2, 8, dtype=torch.bool)
        fine[0, 5] = fine[1, 7] = False
        assert torch.isfinite(out32[fine.cuda()]).all()
        assert torch.allclose(out32[fine.cuda()], clean[1][fine.cuda()], rtol=0, atol=1e-4)


def test_a_sequence_without_any_page_gives_zeros():
    with Cache([32, 50, 7], 4, 2, 64, "f16", seed=22) as c:
        c.fill()
        c.table[0] = B.ISV_BLOCK_NONE
        out, out32 = c.attend()
        assert (out32[0] == 0).all() and (out[0] == 0).all()
        c.check(out, out32, rows=[1, 2])
        assert B.isv_q8_status(c.h) == 0
