"""Cases of chunks of new tokens for the GPU tests: a pool, a table, ragged rows inside one array, and the reference's answer."""
import numpy as np
import torch

from oracle import chunk as oc
from paper_2504_11816_b200 import binding as B
from paper_2504_11816_b200 import workloads as W

CODE = {"f16": B.ISV_F16, "bf16": B.ISV_BF16, "f32": B.ISV_F32}
# what the weights of the 16-bit output may be rounded by, and of the fp32 output (two 16-bit numbers, or 32 bits)
WEIGHT_STEP = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}
FINE_STEP = 2.0 ** -16


def dev(x, dtype=torch.int32):
    return torch.tensor(np.asarray(x), dtype=dtype, device="cuda")


def bits(x):
    """NaN equals itself here."""
    return x.contiguous().view(torch.int16 if x.element_size() == 2 else torch.int32)


def f64(x):
    return x.detach().cpu().double().numpy()


class Case:
    """Sequences of `starts` tokens that get `news` more, in a pool whose pages are in random order."""

    def __init__(self, starts, news, q_heads, kv_heads, d, dtype, seed=0, gaps=True, spare=3, blocks=None):
        g = torch.Generator().manual_seed(seed)
        rng = np.random.default_rng(seed)
        self.starts, self.news = np.asarray(starts), np.asarray(news)
        self.lens = self.starts + self.news
        self.S, self.T = len(news), max(1, int(max(news)))
        self.Hq, self.H, self.d, self.dtype = q_heads, kv_heads, d, dtype
        t = W.torch_dtype(dtype)
        self.blocks = blocks or max(1, int((self.lens.max() + 15) // 16))
        self.stride = self.blocks + 2
        self.n_pages = int(((self.lens + 15) // 16).sum()) + 4
        table = np.full((self.S, self.stride), 1 << 29)
        ids = iter(rng.permutation(self.n_pages))
        for s in range(self.S):
            for b in range((self.lens[s] + 15) // 16):
                table[s, b] = next(ids)
        self.table = table
        # rows: sequences in another order than their numbers, with rows between them that belong to nobody
        self.firsts = np.zeros(self.S, int)
        at = spare
        for s in rng.permutation(self.S):
            self.firsts[s] = at
            at += self.news[s] + (int(rng.integers(0, 3)) if gaps else 0)
        self.rows = at + spare
        self.qkv = torch.randn((self.rows, q_heads + 2 * kv_heads, d), generator=g).to(t)
        self.q, self.k, self.v = self.qkv[:, :q_heads], self.qkv[:, q_heads:q_heads + kv_heads], self.qkv[:, q_heads + kv_heads:]
        # what a page holds behind its sequence's last token, and pages of nobody, may be anything
        self.pool = torch.full((self.n_pages, 2, kv_heads, 16, d), float("nan")).to(t)
        w = torch.tensor(oc.places(d))
        for s in range(self.S):
            n = int(self.lens[s])
            kv = torch.randn((2, kv_heads, n, d), generator=g).to(t)
            for b in range((n + 15) // 16):
                m = min(16, n - 16 * b)
                tile = self.pool[table[s, b]][:, :, :m]
                tile.scatter_(-1, w[:m].expand(2, kv_heads, m, d), kv[:, :, 16 * b:16 * b + m])

    def handle(self, **kw):
        return B.isv_chunk_create(**{**dict(q_heads=self.Hq, kv_heads=self.H, head_dim=self.d, dtype=CODE[self.dtype], max_seqs=self.S), **kw})

    def to_gpu(self):
        self.D = dict(pool=self.pool.cuda(), table=dev(self.table), lens=dev(self.lens), news=dev(self.news), firsts=dev(self.firsts),
                      qkv=self.qkv.cuda())
        x = self.D["qkv"]
        self.D["q"], self.D["k"], self.D["v"] = x[:, :self.Hq], x[:, self.Hq:self.Hq + self.H], x[:, self.Hq + self.H:]
        return self.D

    def attend(self, h, out, out_f32, slopes=None, prefix=None, window=0, stream=0):
        D = self.D
        B.isv_chunk_attn(h, D["pool"], self.n_pages, D["table"], self.stride, self.blocks, D["lens"], D["news"], D["firsts"], self.rows,
                         D["q"], D["q"].stride(0), slopes, prefix, window, out, out_f32, self.S, self.T, stream)

    def want(self, scale=0.0, cap=0.0, slopes=None, prefix=None, window=0, weight_step=2.0 ** -20):
        """out [rows, Hq, d] (NaN in rows of nobody) and its tolerance."""
        out = np.full((self.rows, self.Hq, self.d), np.nan)
        tol = np.zeros(out.shape)
        pool = f64(self.pool)
        for s in range(self.S):
            K, V, there = oc.history(pool, self.table[s], int(self.lens[s]))
            pos = self.starts[s] + np.arange(self.news[s])
            seen = oc.visible(pos, int(self.lens[s]), window, 0 if prefix is None else int(prefix[s])) & there
            r = slice(self.firsts[s], self.firsts[s] + self.news[s])
            out[r], tol[r] = oc.attend(f64(self.q[r]), K, V, pos, seen, scale or 1 / np.sqrt(self.d), cap, slopes, weight_step)
        return out, tol

    def check(self, got, want, tol, half_step=0.0):
        """Rows of nobody are as they were (they held 7), the others within the tolerance and half a step of the output."""
        mine = ~np.isnan(want).all((1, 2))
        live = np.zeros(self.rows, bool)
        for s in range(self.S):
            live[self.firsts[s]:self.firsts[s] + self.news[s]] = True
        got = f64(got)
        assert (got[~live] == 7).all()
        assert not (live & ~mine).any()
        room = tol + half_step * (np.abs(want) + tol) + (2.0 ** -25 if half_step else 0.0)
        off = np.abs(got - want)[live]
        assert np.array_equal(np.isfinite(got[live]), np.isfinite(want[live]))
        assert np.all((off <= room[live]) | ~np.isfinite(want[live])), (np.nanmax(off), np.nanmax(off / np.maximum(room[live], 1e-30)))


def run_and_check(c, slopes=None, prefix=None, window=0, outputs=("both", "16", "32"), **desc):
    """The call with both outputs, and with each of them alone, against the reference; twice the same bits."""
    D = c.to_gpu()
    h = c.handle(**desc)
    sd = dev(slopes, torch.float32) if slopes is not None else None
    pd = dev(prefix) if prefix is not None else None
    try:
        t = W.torch_dtype(c.dtype)
        for which in outputs:
            for again in range(2):
                out = torch.full((c.rows, c.Hq, c.d), 7.0, dtype=t, device="cuda") if which != "32" else None
                f32 = torch.full((c.rows, c.Hq, c.d), 7.0, device="cuda") if which != "16" else None
                c.attend(h, out, f32, sd, pd, window)
                if again:
                    assert all(x is None or torch.equal(bits(x), bits(y)) for x, y in zip((out, f32), before))
                before = (out, f32)
            args = dict(scale=desc.get("scale", 0.0), cap=desc.get("softcap", 0.0), slopes=slopes, prefix=prefix, window=window)
            if f32 is not None:
                c.check(f32, *c.want(**args, weight_step=FINE_STEP))
            if out is not None:
                c.check(out, *c.want(**args, weight_step=WEIGHT_STEP[c.dtype]), half_step=oc.HALF_STEP[c.dtype])
        assert B.isv_chunk_status(h) == 0
        return out, f32
    finally:
        B.isv_chunk_free(h)
