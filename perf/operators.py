"""Cases of the operators on 8-bit KV caches, on cache pages and on 4-bit weights.

``run`` computes an operator either in its plain form (elementary torch operations in 32 bits, 64 where a value next to
a rounding border needs them) or, with ``own`` set, through the framework's entry points.  ``exact`` is the definition
in 64 bits.

Layout of the 8-bit cache (both forms read and write the same bytes).  A page holds 16 tokens of all KV heads; per head
one unit of 32 * d + 16 bytes: 16 * d codes of K, 16 * d codes of V, the two fp32 scales, 8 unused bytes.  The codes of
a unit are stored in the order in which the lanes of a warp consume them (``_orders``).
"""
import math

import torch

own = False

BT = 16                      # tokens of a page
F16, BF16 = 0, 1
INT8, E4M3 = 0, 1
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}


# ---------------------------------------------------------------- cases

def listed():
    return [
        # one user of a grouped-query model with a long history: a few microseconds of reading, latency counts
        dict(name="attn one user", op="attn", batch=1, q_heads=32, kv_heads=8, d=128, len_min=8191, len_max=8191, type="bf16", format="e4m3"),
        # multi-head model of the 7B shape, batch 32, 1024 tokens of prompt and up to 128 generated
        dict(name="attn 7B", op="attn", batch=32, q_heads=32, kv_heads=32, d=128, len_min=1025, len_max=1152, type="f16", format="int8"),
        # grouped-query model, a large batch at full context: the longest reading of the set
        dict(name="attn 8B grouped", op="attn", batch=256, q_heads=32, kv_heads=8, d=128, len_min=4096, len_max=4127, type="bf16", format="e4m3"),
        # multi-head model with heads of 80, ragged from empty rows to the end of the generation
        dict(name="attn heads of 80", op="attn", batch=32, q_heads=32, kv_heads=32, d=80, len_min=0, len_max=1152, type="f16", format="int8"),
        # one decode step's append of a large batch: one token each, one sequence in 16 completes a block
        dict(name="append", op="write", batch=256, kv_heads=8, d=128, tokens=1, start_max=4096, type="bf16", format="e4m3"),
        # prompts of the 7B shape, ragged
        dict(name="prompt", op="write", batch=16, kv_heads=32, d=128, tokens=2048, start_max=0, type="f16", format="int8"),
        # one step of a beam search over a 16-bit pool: rows reorder, siblings get private copies of the open block
        dict(name="fork", op="fork", rows=256, blocks=72, kv_heads=8, d=80, layers=4, keep=0.5),
        # the pages a decode step of 512 sequences needs, from a pool of 64 Ki pages
        dict(name="resize", op="resize", rows=512, blocks=256, n_pages=65536),
        # a pool half of whose rows have left, made dense again
        dict(name="compact", op="compact", rows=96, blocks=64, kv_heads=8, d=128, layers=2, n_pages=8192),
        # attention output projection of the 7B shape for one token
        dict(name="linear one token", op="linear", M=1, N=4096, K=4096, group=128, type="bf16"),
        # gate and up projections of the 7B shape for one token
        dict(name="linear gate up", op="linear", M=1, N=22016, K=4096, group=128, type="f16"),
        # down projection of the 7B shape for a small batch
        dict(name="linear batch", op="linear", M=16, N=4096, K=11008, group=64, type="bf16"),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, even over the logarithm."""
    return min(hi, max(lo, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    op = rng.choice(["attn", "attn", "write", "fork", "resize", "compact", "linear", "linear"])
    d = rng.choice([64, 80, 128])
    t, f = rng.choice(["f16", "bf16"]), rng.choice(["int8", "e4m3"])
    if op == "attn":
        hkv, g = rng.choice([1, 2, 5, 8, 32]), rng.choice([1, 2, 3, 4, 7, 8, 12, 16])
        longest = _spread(rng, 1, 32768)
        most = (1 << 30) // (longest * hkv * d * 2)          # at most about 1 GiB of cache
        return dict(op=op, batch=_spread(rng, 1, max(1, min(256, most))), q_heads=hkv * g, kv_heads=hkv, d=d,
                    len_min=rng.choice([0, longest // 2, longest]), len_max=longest, type=t, format=f)
    if op == "write":
        hkv = rng.choice([1, 2, 5, 8, 32])
        tokens = 1 if rng.random() < 0.4 else _spread(rng, 2, 4096)
        most = (1 << 28) // (tokens * hkv * d * 4)
        return dict(op=op, batch=_spread(rng, 1, max(1, min(256, most))), kv_heads=hkv, d=d, tokens=tokens,
                    start_max=rng.choice([0, 16, 500, 4096]), type=t, format=f)
    if op == "fork":
        return dict(op=op, rows=_spread(rng, 2, 512), blocks=_spread(rng, 1, 100), kv_heads=rng.choice([1, 2, 8]), d=d,
                    layers=rng.choice([1, 2, 3]), keep=rng.choice([0.1, 0.5, 0.9]))
    if op == "resize":
        rows, blocks = _spread(rng, 1, 1024), _spread(rng, 1, 512)
        return dict(op=op, rows=rows, blocks=blocks, n_pages=rows * blocks // 2 + 2 * rows + rng.randrange(1, 5000))
    if op == "compact":
        rows, blocks = _spread(rng, 1, 128), _spread(rng, 1, 64)
        return dict(op=op, rows=rows, blocks=blocks, kv_heads=rng.choice([1, 2, 8]), d=d, layers=rng.choice([1, 2]),
                    n_pages=rows * blocks + rng.randrange(1, 2000))
    g = rng.choice([32, 64, 128])
    return dict(op=op, M=rng.choice([1, 1, 2, 3, 5, 8, 13, 16, 24, 32]), N=_spread(rng, 16, 32000),
                K=g * _spread(rng, 1, 11008 // g), group=g, type=t)


def work(c):
    if c["op"] == "attn":
        tokens = c["batch"] * (c["len_min"] + c["len_max"]) / 2
        row = 2 * c["q_heads"] * c["d"] * 2 * c["batch"]     # q in, out out
        return {"bytes": tokens * c["kv_heads"] * 2 * (c["d"] + 0.25) + row, "flops": 4.0 * tokens * c["q_heads"] * c["d"]}
    if c["op"] == "write":
        n = c["batch"] * (c["tokens"] + 1) / 2 if c["tokens"] > 1 else c["batch"]
        values = n * c["kv_heads"] * c["d"] * 2
        return {"bytes": values * 3, "flops": values * 3}
    if c["op"] == "fork":
        page = 2 * c["kv_heads"] * BT * c["d"] * 2
        copies = c["rows"] * (1 - c["keep"]) * 0.9
        return {"bytes": 2 * copies * page * c["layers"] + 8 * c["rows"] * c["blocks"], "flops": 0}
    if c["op"] == "resize":
        return {"bytes": 2 * c["rows"] * c["blocks"] + 16 * c["rows"], "flops": 0}
    if c["op"] == "compact":
        page = 2 * c["kv_heads"] * BT * c["d"] * 2
        live = c["rows"] * c["blocks"] * 3 / 8
        moves = live * (1 - live / c["n_pages"])
        return {"bytes": 2 * moves * page * c["layers"] + 6 * c["rows"] * c["blocks"], "flops": 0}
    return {"bytes": c["N"] * c["K"] * (0.5 + 2.0 / c["group"]) + 2 * c["M"] * (c["N"] + c["K"]), "flops": 2.0 * c["M"] * c["N"] * c["K"]}


# ---------------------------------------------------------------- the cache's layout

_kept_orders = {}


def _orders(d):
    """For each code of a unit's K part and of its V part: which (token * d + dim) it holds; and the inverses."""
    if d not in _kept_orders:
        pos = torch.arange(BT * d)
        whole = pos < 512 * (d // 32)
        p, b = pos // 512, (pos % 16) // 8
        rest = pos - 512 * (d // 32)
        lane = torch.where(whole, (pos % 512) // 16, rest // 8)
        half, j = (pos % 8) // 4, pos % 4
        g, c = lane // 4, lane % 4
        k_dim = torch.where(whole, 32 * p + 8 * c + 4 * b + j, 32 * (d // 32) + 4 * c + j)
        k = (g + 8 * half) * d + k_dim
        tile = torch.where(whole, 2 * p + b, d // 16 - 1)
        v = (2 * c + (j % 2) + 8 * (j // 2)) * d + g * (d // 8) + 2 * tile + half
        both = []
        for o in (k, v):
            o = o.cuda()
            back = torch.empty_like(o)
            back[o] = torch.arange(BT * d, device="cuda")
            both += [o, back]
        _kept_orders[d] = both
    return _kept_orders[d]


def _values(codes, fmt):
    """uint8 bytes -> the numbers they are (fp32)."""
    return codes.view(torch.int8 if fmt == "int8" else torch.float8_e4m3fn).float()


def _quantise(x, fmt):
    """x [..., 16, d] -> (bytes [..., 16 * d] in logical order, fp32 scales [...]).  The quotient is taken in 64 bits:
    its rounding decides between neighbouring codes."""
    x = x.double()
    scale = (x.abs().amax((-1, -2)) / (127.0 if fmt == "int8" else 448.0)).float()
    s = scale.double()[..., None, None]
    q = torch.where(s > 0, x / s, torch.zeros_like(x)).flatten(-2)
    if fmt == "int8":
        return q.round().clamp(-127, 127).to(torch.int8).view(torch.uint8), scale
    step = torch.exp2(torch.frexp(q)[1].double() - 1).clamp(min=2.0 ** -6) / 8      # 3 bits behind the leading one
    return ((q / step).round() * step).clamp(-448, 448).float().to(torch.float8_e4m3fn).view(torch.uint8), scale


def _pack(k, v, fmt):
    """k, v [..., 16, d] -> units [..., 32 d + 16] as bytes."""
    ko, _, vo, _ = _orders(k.shape[-1])
    (kc, ks), (vc, vs) = _quantise(k, fmt), _quantise(v, fmt)
    tail = torch.stack([ks, vs, torch.zeros_like(ks), torch.zeros_like(ks)], -1).view(torch.uint8)
    return torch.cat([kc[..., ko], vc[..., vo], tail], -1)


def _unpack(units, d, fmt):
    """units [..., 32 d + 16] -> k, v [..., 16, d] in fp32."""
    _, kb, _, vb = _orders(d)
    n = BT * d
    s = units[..., 2 * n:2 * n + 8].contiguous().view(torch.float32)
    shape = units.shape[:-1] + (BT, d)
    k = _values(units[..., :n][..., kb], fmt).view(shape) * s[..., 0, None, None]
    v = _values(units[..., n:2 * n][..., vb], fmt).view(shape) * s[..., 1, None, None]
    return k, v


class _Handle:
    """A handle of the framework that is released with the state that keeps it."""

    def __init__(self, made, free):
        self.h, self.free = made, free

    def __del__(self):
        try:
            self.free(self.h)
        except Exception:
            pass


def _attach(st, c):
    """The handle that a user's program keeps next to its buffers."""
    if own:
        from paper_2504_11816_b200 import binding as B
        if c["op"] in ("attn", "write"):
            st["h"] = _Handle(B.isv_q8_create(q_heads=c.get("q_heads", c["kv_heads"]), kv_heads=c["kv_heads"], head_dim=c["d"],
                                              dtype=F16 if c["type"] == "f16" else BF16,
                                              format=INT8 if c["format"] == "int8" else E4M3, max_seqs=c["batch"]), B.isv_q8_free)
        elif c["op"] == "linear":
            st["h"] = _Handle(B.isv_linear4_create(st["w"], st["scales"], c["N"], c["K"], c["group"],
                                                   F16 if c["type"] == "f16" else BF16, c["M"]), B.isv_linear4_free)
    return st


# ---------------------------------------------------------------- inputs

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _ints(g, lo, hi, shape):
    return torch.randint(lo, hi + 1, shape, generator=g, device="cuda", dtype=torch.int32)


def _kv(g, shape, dtype):
    """K or V rows: normal, one entry in 100 eight times as large."""
    x = torch.randn(shape, generator=g, device="cuda")
    big = torch.rand(shape, generator=g, device="cuda") < 0.01
    return torch.where(big, x * 8, x).to(dtype)


def prepare(c, seed):
    g = _gen(seed)
    st = {"case": c}
    if c["op"] in ("attn", "write"):
        dt, H, d, B = TYPES[c["type"]], c["kv_heads"], c["d"], c["batch"]
        unit = 32 * d + 16
        if c["op"] == "attn":
            lens = _ints(g, c["len_min"], c["len_max"], (B,))
            most = max(1, (c["len_max"] + BT - 1) // BT)
        else:
            st["T"] = T = c["tokens"]
            # a chunk of a prompt begins where a block begins; a step's token anywhere
            start = _ints(g, 0, c["start_max"], (B,)) if T == 1 else _ints(g, 0, c["start_max"] // BT, (B,)) * BT
            st["new"] = _ints(g, 1, T, (B,))
            lens = start + st["new"]
            most = (c["start_max"] + T + BT - 1) // BT
            st["k"], st["v"] = (_kv(g, (B, T, H, d), dt) for _ in range(2))
        n = B * most + 7
        st["n"], st["blocks"] = n, most
        st["lens"] = lens
        st["table"] = torch.randperm(n, generator=g, device="cuda")[:B * most].int().view(B, most).contiguous()
        if c["op"] == "attn":
            st["pool"] = torch.cat([_pack(_kv(g, (b, H, BT, d), dt), _kv(g, (b, H, BT, d), dt), c["format"])
                                    for b in [min(8192, n - i) for i in range(0, n, 8192)]])
            st["q"] = torch.randn((B, c["q_heads"], d), generator=g, device="cuda").to(dt)
            st["out"] = torch.empty_like(st["q"])
        else:
            st["pool"] = torch.zeros((n, H, unit), dtype=torch.uint8, device="cuda")
        tails = _kv(g, (B, 2, H, BT, d), dt)
        behind = torch.arange(BT, device="cuda") >= (lens - (st["new"] if c["op"] == "write" else 0))[:, None] % BT
        # rows of the open block that are not written yet hold anything
        st["tails"] = torch.where(behind[:, None, None, :, None], torch.full_like(tails, float("nan") if c["op"] == "attn" else 0.0), tails)
        return _attach(st, c)
    if c["op"] == "linear":
        dt = TYPES[c["type"]]
        st["w"] = torch.randint(0, 256, (c["N"], c["K"] // 2), generator=g, device="cuda", dtype=torch.uint8)
        st["scales"] = ((0.5 + torch.rand((c["N"], c["K"] // c["group"]), generator=g, device="cuda")) * 0.2 / math.sqrt(c["K"])).to(dt)
        st["x"] = torch.randn((c["M"], c["K"]), generator=g, device="cuda").to(dt)
        st["y"] = torch.empty((c["M"], c["N"]), dtype=dt, device="cuda")
        return _attach(st, c)

    R, NB = c["rows"], c["blocks"]
    if c["op"] == "fork":
        old = max(1, int(R * c["keep"]))                     # rows that go on, each with one child or more
        st["lens"] = _ints(g, 1, NB * BT, (R,))
        n = R * NB + R + 5
        st["table"] = torch.randperm(n, generator=g, device="cuda")[:R * NB].int().view(R, NB).contiguous()
        alive = torch.randperm(R, generator=g, device="cuda")[:old]
        st["parent"] = torch.cat([alive, alive[torch.randint(0, old, (R - old,), generator=g, device="cuda")]])[
            torch.randperm(R, generator=g, device="cuda")].int()
        st["table_out"], st["lens_out"] = torch.empty_like(st["table"]), torch.empty_like(st["lens"])
        st["from"], st["to"] = (torch.empty(R, dtype=torch.int32, device="cuda") for _ in range(2))
    elif c["op"] == "resize":
        n = c["n_pages"]
        st["lens"] = _ints(g, 0, NB * BT // 2, (R,))         # half of the rows' capacity in use on average: a quarter
        st["lens_new"] = torch.clamp(st["lens"] + _ints(g, -BT, 2 * BT, (R,)), 0, NB * BT).int()
        ids = torch.randperm(n, generator=g, device="cuda").int()
        st["table"] = torch.full((R, NB), -1, dtype=torch.int32, device="cuda")
        have = (NB + 1) // 2
        st["table"][:, :have] = ids[:R * have].view(R, have)
        st["n"] = n
        return st
    else:
        n = c["n_pages"]
        st["lens"] = _ints(g, 1, NB * BT, (R,)) * (torch.rand(R, generator=g, device="cuda") < 0.75).int()
        st["table"] = torch.randperm(n, generator=g, device="cuda")[:R * NB].int().view(R, NB).contiguous()
        st["table_out"] = torch.empty_like(st["table"])
        st["moves"] = (n + 1) // 2
        st["from"], st["to"] = (torch.empty(st["moves"], dtype=torch.int32, device="cuda") for _ in range(2))
        st["counts"] = torch.empty(2, dtype=torch.int32, device="cuda")
    st["n"] = n
    # the page behind the last one belongs to nobody
    st["pool"] = torch.randn((c["layers"], n + 1, 2, c["kv_heads"], BT, c["d"]), generator=g, device="cuda", dtype=torch.float16)
    return st


# ---------------------------------------------------------------- one pass

def run(st):
    return {"attn": _attn, "write": _write, "fork": _fork, "resize": _resize, "compact": _compact, "linear": _linear}[st["case"]["op"]](st)


def _attn(st):
    c = st["case"]
    if own:
        from paper_2504_11816_b200 import binding as B
        B.isv_q8_attn(st["h"].h, st["pool"], st["n"], st["tails"], st["table"], st["blocks"], st["blocks"], st["lens"],
                      st["q"], st["out"], None, c["batch"])
        return st["out"]
    k, v, lens = _history(st)
    n = k.shape[2]
    q = st["q"].float().view(c["batch"], c["kv_heads"], -1, c["d"])
    s = torch.matmul(q, k.transpose(2, 3)) * (1 / math.sqrt(c["d"]))
    gone = torch.arange(n, device="cuda") >= lens[:, None]
    s.masked_fill_(gone[:, None, None], float("-inf"))
    top = s.amax(-1, keepdim=True)
    e = torch.exp(s - torch.where(torch.isinf(top), torch.zeros_like(top), top))
    total = e.sum(-1, keepdim=True)
    o = torch.matmul(e, v) / torch.where(total > 0, total, torch.ones_like(total))
    return o.reshape(st["q"].shape).to(st["q"].dtype)


def _history(st):
    """All rows' keys and values in fp32, [batch, heads, tokens, d], zero behind a row's last token."""
    c = st["case"]
    B, H, d = c["batch"], c["kv_heads"], c["d"]
    lens = st["lens"].long()
    row = torch.arange(B, device="cuda")
    kv = []
    for i, x in enumerate(_unpack(st["pool"][st["table"].long()], d, c["format"])):     # [B, blocks, H, 16, d]
        x = torch.cat([x, torch.zeros_like(x[:, :1])], 1)
        x[row, lens // BT] = st["tails"][:, i].float()
        x = x.permute(0, 2, 1, 3, 4).reshape(B, H, -1, d)
        gone = torch.arange(x.shape[2], device="cuda") >= lens[:, None]
        kv.append(x.masked_fill_(gone[:, None, :, None], 0.0))
    return kv[0], kv[1], lens


def _write(st):
    c = st["case"]
    if own:
        from paper_2504_11816_b200 import binding as B
        row = c["kv_heads"] * c["d"]
        B.isv_q8_write(st["h"].h, st["pool"], st["n"], st["tails"], st["table"], st["blocks"], st["blocks"], st["lens"],
                       st["new"], st["k"], st["v"], st["T"] * row, row, c["batch"], st["T"])
        return _cache_of(st)
    B, H, d, T = c["batch"], c["kv_heads"], c["d"], st["T"]
    lens, new = st["lens"].long(), st["new"].long()
    start = lens - new
    nb = (T + BT - 2) // BT + 1                              # blocks that the new tokens can touch
    at = (start // BT * BT)[:, None] + torch.arange(nb * BT, device="cuda")              # positions of those blocks
    index = (at - start[:, None]).clamp(0, T - 1)
    fresh = ((at >= start[:, None]) & (at < lens[:, None])).view(B, nb, 1, BT, 1)
    block = torch.arange(nb, device="cuda") + (start // BT)[:, None]
    done = (block + 1) * BT <= lens[:, None]                 # complete now
    opened = (block == (lens // BT)[:, None]) & (lens % BT > 0)[:, None]
    row = torch.arange(B, device="cuda")
    both, tails = [], []
    for i, x in enumerate((st["k"], st["v"])):
        x = torch.gather(x, 1, index[..., None, None].expand(-1, -1, H, d)).view(B, nb, BT, H, d).transpose(2, 3)
        held = torch.zeros_like(x)
        held[:, 0] = st["tails"][:, i]
        both.append(torch.where(fresh, x, held))
        last = (lens // BT - start // BT).clamp(max=nb - 1)
        now = both[i][row, last]
        keep = opened.any(1)[:, None, None, None] & (fresh[row, last])
        tails.append(torch.where(keep, now, st["tails"][:, i]))
    units = _pack(both[0], both[1], c["format"])             # [B, nb, H, unit]
    st["tails"] = torch.stack(tails, 1)
    ids = torch.gather(st["table"].long(), 1, block.clamp(max=st["blocks"] - 1))
    ids = ids[done]
    st["pool"][ids] = units[done]
    return _cache_of(st)


def _cache_of(st):
    """The cache as its numbers: codes (whole numbers, or 8-bit floats), scales and the 16-bit rows of the open blocks."""
    c = st["case"]
    n = 32 * c["d"]
    units = st["pool"].view(st["n"], c["kv_heads"], n + 16)
    codes = units.view(torch.int8 if c["format"] == "int8" else torch.float8_e4m3fn)[..., :n]
    return {"codes": codes, "scales": units.view(torch.float32)[..., n // 4:n // 4 + 2], "tails": st["tails"]}


def _free_first(live):
    """live [n] of truth values -> the free ids in ascending order, filled up with -1."""
    n = live.numel()
    rank = torch.where(live, torch.full((n,), n, device="cuda"), torch.cumsum((~live).long(), 0) - 1)
    out = torch.full((n + 1,), -1, dtype=torch.long, device="cuda")
    out[rank] = torch.arange(n, device="cuda")
    out[n] = -1
    return out


def _live(table, blocks, n):
    """Which of n pages the first blocks[s] entries of each row s name."""
    used = torch.arange(table.shape[1], device="cuda") < blocks[:, None]
    live = torch.zeros(n + 1, dtype=torch.bool, device="cuda")
    live[torch.where(used, table.long(), torch.full_like(table, n).long())] = True
    return live[:n]


def _copied(st, src, dst):
    """Pages src[i] -> dst[i] in every layer; -1 stands for the page that belongs to nobody."""
    n = st["n"]
    st["pool"][:, torch.where(dst < 0, n, dst)] = st["pool"][:, torch.where(src < 0, n, src)]


def _fork(st):
    c, n = st["case"], st["n"]
    R, NB = c["rows"], c["blocks"]
    if own:
        from paper_2504_11816_b200 import binding as B
        page = 2 * c["kv_heads"] * BT * c["d"] * 2
        B.isv_pages_fork(st["table"], st["lens"], R, st["parent"], st["table_out"], st["lens_out"], R, NB, NB, 1, n, st["from"], st["to"])
        B.isv_pages_copy(st["pool"], n, st["pool"], n, page, c["layers"], (n + 1) * page, (n + 1) * page, st["from"], st["to"], R)
        return {"table": st["table_out"], "lens": st["lens_out"], "from": st["from"], "to": st["to"], "pool": st["pool"]}
    parent = st["parent"].long()
    lens = st["lens"].long()[parent]
    nb = (lens + BT - 1) // BT
    table = torch.where(torch.arange(NB, device="cuda") < nb[:, None], st["table"].long()[parent], -1)
    row = torch.arange(R, device="cuda")
    first = torch.full((R,), R, device="cuda").scatter_reduce_(0, parent, row, "amin")
    private = (lens % BT > 0) & (first[parent] < row)
    free = _free_first(_live(table, nb, n))
    dst = torch.where(private, free[(torch.cumsum(private.long(), 0) - 1).clamp(min=0)], -1)
    last = (nb - 1).clamp(min=0)
    src = torch.where(private, table[row, last], -1)
    table[row, last] = torch.where(private, dst, table[row, last])
    _copied(st, src, dst)
    return {"table": table.int(), "lens": lens.int(), "from": src.int(), "to": dst.int(), "pool": st["pool"]}


def _resize(st):
    c, n = st["case"], st["n"]
    R, NB = c["rows"], c["blocks"]
    if own:
        from paper_2504_11816_b200 import binding as B
        B.isv_pages_resize(st["table"], st["lens"], st["lens_new"], R, NB, NB, 1, n)
        return st["table"]
    a, b = (st["lens"].long() + BT - 1) // BT, (st["lens_new"].long() + BT - 1) // BT
    free = _free_first(_live(st["table"], torch.minimum(a, b), n))
    at = torch.arange(NB, device="cuda")
    more = (at >= a[:, None]) & (at < b[:, None])
    rank = torch.cumsum(more.flatten().long(), 0) - 1
    fresh = free[rank.clamp(min=0, max=n)].view(R, NB)
    st["table"].copy_(torch.where(more, fresh, torch.where(at < b[:, None], st["table"].long(), -1)))
    return st["table"]


def _compact(st):
    c, n = st["case"], st["n"]
    R, NB = c["rows"], c["blocks"]
    if own:
        from paper_2504_11816_b200 import binding as B
        page = 2 * c["kv_heads"] * BT * c["d"] * 2
        B.isv_pages_compact(st["table"], st["lens"], R, NB, NB, 1, n, st["table_out"], st["from"], st["to"], st["moves"], st["counts"])
        B.isv_pages_copy(st["pool"], n, st["pool"], n, page, c["layers"], (n + 1) * page, (n + 1) * page, st["from"], st["to"],
                         st["moves"], st["counts"][1:])
        return {"table": st["table_out"], "from": st["from"], "to": st["to"], "counts": st["counts"], "pool": st["pool"]}
    nb = (st["lens"].long() + BT - 1) // BT
    live = _live(st["table"], nb, n)
    total = live.sum()
    ids = torch.arange(n, device="cuda")
    before = torch.cumsum(live.long(), 0) - live.long()
    hole, over = ~live & (ids < total), live & (ids >= total)
    moves = hole.sum()
    m = st["moves"]
    dst = torch.full((m + 1,), -1, dtype=torch.long, device="cuda")
    src = dst.clone()
    dst[torch.where(hole, ids - before, m)] = ids
    src[torch.where(over, before - (total - moves), m)] = ids
    src, dst = src[:m], dst[:m]
    there = torch.cat([ids, ids.new_full((1,), -1)])
    there[torch.where(src < 0, n, src)] = torch.where(src < 0, -1, dst)
    table = torch.where(torch.arange(NB, device="cuda") < nb[:, None], there[st["table"].long()], -1)
    _copied(st, src, dst)
    return {"table": table.int(), "from": src.int(), "to": dst.int(), "counts": torch.stack([total, moves]).int(), "pool": st["pool"]}


def _linear(st):
    c = st["case"]
    if own:
        from paper_2504_11816_b200 import binding as B
        B.isv_linear4_forward(st["h"].h, st["x"], st["y"], None, c["M"])
        return st["y"]
    w = torch.stack([st["w"] & 15, st["w"] >> 4], -1).flatten(1).float() - 8
    w = (w.view(c["N"], -1, c["group"]) * st["scales"].float()[..., None]).view(c["N"], c["K"])
    return torch.matmul(st["x"].float(), w.t()).to(st["x"].dtype)


# ---------------------------------------------------------------- the definition in 64 bits

def exact(c, seed):
    if c["op"] not in ("attn", "write", "linear"):
        return None                                          # copies and whole numbers: nothing is rounded
    st = prepare(c, seed)
    if c["op"] == "linear":
        out = torch.empty((c["M"], c["N"]), dtype=torch.float64, device="cuda")
        nibble = torch.zeros((c["N"], c["K"]), dtype=torch.float64, device="cuda")
        nibble[:, 0::2] = (st["w"] % 16).double()
        nibble[:, 1::2] = (st["w"] // 16).double()
        for i in range(c["M"]):
            y = ((nibble - 8.0) * st["x"][i].double()).view(c["N"], -1, c["group"]).sum(-1)
            out[i] = (y * st["scales"].double()).sum(-1)
        return out
    H, d = c["kv_heads"], c["d"]
    ko, _, vo, _ = _orders(d)
    lens = st["lens"].tolist()
    if c["op"] == "write":
        if c["batch"] * c["tokens"] > 1 << 18:
            return None
        pool = {"codes": torch.zeros((st["n"], H, 32 * d), dtype=torch.float64, device="cuda"),
                "scales": torch.zeros((st["n"], H, 2), dtype=torch.float64, device="cuda")}
        tails = st["tails"].double()
        new, top = st["new"].tolist(), 127.0 if c["format"] == "int8" else 448.0
        grid = torch.arange(256, device="cuda", dtype=torch.uint8).view(torch.float8_e4m3fn).double()
        grid = grid[torch.isfinite(grid)].unique()
        for s in range(c["batch"]):
            start = lens[s] - new[s]
            first = start // BT * BT
            rows = []
            for i, x in enumerate((st["k"], st["v"])):
                old = st["tails"][s, i, :, :start - first].double()
                rows.append(torch.cat([old, x[s, :new[s]].transpose(0, 1).double()], 1))         # [H, tokens, d]
            whole = (lens[s] - first) // BT
            for b in range(whole):
                page = int(st["table"][s, first // BT + b])
                for i, o in ((0, ko), (1, vo)):
                    x = rows[i][:, b * BT:(b + 1) * BT].reshape(H, -1)
                    sc = (x.abs().amax(1) / top)
                    z = x / torch.where(sc > 0, sc.float().double(), torch.ones_like(sc))[:, None]
                    if c["format"] == "int8":
                        z = torch.round(z)
                    else:
                        up = torch.searchsorted(grid, z.contiguous()).clamp(1, grid.numel() - 1)
                        lo, hi = grid[up - 1], grid[up]
                        tie = (z - lo == hi - z) & ((up - 1) % 2 == (grid.numel() // 2) % 2)     # the even one of the two
                        z = torch.where((z - lo < hi - z) | tie, lo, hi)
                    pool["codes"][page, :, i * BT * d:(i + 1) * BT * d] = z[:, o]
                    pool["scales"][page, :, i] = sc
            left = lens[s] % BT
            if left:
                for i in range(2):
                    tails[s, i, :, :left] = rows[i][:, whole * BT:]
        return {"codes": pool["codes"] if c["format"] == "e4m3" else None, "scales": pool["scales"], "tails": tails}
    out = torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda")
    g = c["q_heads"] // H
    kind = torch.int8 if c["format"] == "int8" else torch.float8_e4m3fn
    n = BT * d
    for s in range(c["batch"]):
        full, left = lens[s] // BT, lens[s] % BT
        if not lens[s]:
            continue
        u = st["pool"][st["table"][s, :full].long()]
        scale = u[..., 2 * n:2 * n + 8].contiguous().view(torch.float32).double()
        kv = []
        for i, o in ((0, ko), (1, vo)):
            x = torch.empty((full, H, n), dtype=torch.float64, device="cuda")
            x[..., o] = u[..., i * n:(i + 1) * n].contiguous().view(kind).double() * scale[..., i, None]
            x = x.view(full, H, BT, d).permute(1, 0, 2, 3).reshape(H, full * BT, d)
            kv.append(torch.cat([x, st["tails"][s, i, :, :left].double()], 1))
        q = st["q"][s].double().view(H, g, d)
        w = torch.softmax(torch.einsum("hgd,htd->hgt", q, kv[0]) / math.sqrt(d), -1)
        out[s] = torch.einsum("hgt,htd->hgd", w, kv[1]).reshape(-1, d)
    return out
