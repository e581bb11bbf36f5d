"""Cases of the operators on a chunk of new tokens: storing it in a 16-bit paged cache with the position rotation applied
on the way, attention of the chunk over that cache, and the verification of drafted tokens.

``run`` computes an operator either in its plain form (elementary torch operations in 32 bits, 64 for angles and for sums
that a choice depends on) or, with ``own`` set, through the framework's entry points.  ``exact`` is the definition in 64
bits, one sequence after another.

Layout of the cache (both forms use the same bytes): ``[page][K|V][kv_head][16 tokens][d]``; inside a tile, 16-byte chunk
``c`` of token ``t`` is stored at chunk ``c XOR (t mod 8)`` of its row (complete groups of eight chunks only).
"""
import math

import torch

own = False

BT = 16                      # tokens of a page
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
CODE = {"f16": 0, "bf16": 1, "f32": 2}
HALVES, ADJACENT = 0, 1      # which elements of a head a rotation pairs: i with i + half, or 2 i with 2 i + 1


# ---------------------------------------------------------------- cases

def listed():
    return [
        # eight drafted tokens of one user of a grouped-query model with a long history: latency counts
        dict(name="attn one user", op="attn", batch=1, new_min=8, new_max=8, start_min=8183, start_max=8183, q_heads=32, kv_heads=8, d=128,
             type="bf16", softcap=0.0, window=0, slopes=False, prefix=False),
        # up to four drafts and the token before them, for each of 64 users
        dict(name="attn drafts", op="attn", batch=64, new_min=1, new_max=5, start_min=1024, start_max=4096, q_heads=32, kv_heads=8, d=128,
             type="bf16", softcap=0.0, window=0, slopes=False, prefix=False),
        # single tokens of a multi-head model with small heads, from empty rows on
        dict(name="attn single tokens", op="attn", batch=128, new_min=0, new_max=1, start_min=0, start_max=2048, q_heads=16, kv_heads=16, d=64,
             type="f16", softcap=0.0, window=0, slopes=False, prefix=False),
        # a long prompt of the grouped-query model, all of it at once: the largest product of the set
        dict(name="attn prompt", op="attn", batch=1, new_min=8192, new_max=8192, start_min=0, start_max=0, q_heads=32, kv_heads=8, d=128,
             type="bf16", softcap=0.0, window=0, slopes=False, prefix=False),
        # chunks of prompts, 512 tokens a step, scores capped, a sliding window
        dict(name="attn capped window", op="attn", batch=4, new_min=385, new_max=512, start_min=0, start_max=8192, q_heads=16, kv_heads=8, d=128,
             type="bf16", softcap=50.0, window=4096, slopes=False, prefix=False),
        # ragged prompts of a multi-head model with heads of 80, a bias by distance, prefixes seen by all
        dict(name="attn biased prefix", op="attn", batch=8, new_min=1, new_max=640, start_min=0, start_max=640, q_heads=32, kv_heads=32, d=80,
             type="f16", softcap=0.0, window=0, slopes=True, prefix=True),
        # one decode step's keys and values of a large batch
        dict(name="append", op="write", batch=256, new_min=1, new_max=1, start_min=0, start_max=2048, q_heads=32, kv_heads=8, d=128, rotary=128,
             pairs=HALVES, axes=1, type="bf16"),
        # ragged prompts of the 7B shape
        dict(name="append prompts", op="write", batch=16, new_min=1, new_max=2048, start_min=0, start_max=0, q_heads=32, kv_heads=32, d=128,
             rotary=128, pairs=HALVES, axes=1, type="f16"),
        # images among the tokens: positions with three axes, half of a head rotated, adjacent pairs
        dict(name="append images", op="write", batch=2, new_min=577, new_max=1200, start_min=0, start_max=5000, q_heads=16, kv_heads=2, d=128,
             rotary=64, pairs=ADJACENT, axes=3, type="bf16"),
        # one user's drafts against the 7B shape's vocabulary
        dict(name="verify one user", op="verify", batch=1, drafts=4, vocab=32000, type="f32", given=True),
        # a batch's drafts against a large vocabulary
        dict(name="verify batch", op="verify", batch=128, drafts=5, vocab=128000, type="f32", given=True),
        # drafts that were looked up and have no probabilities of their own
        dict(name="verify looked up", op="verify", batch=48, drafts=10, vocab=50257, type="bf16", given=False),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, even over the logarithm."""
    return min(hi, max(lo, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    op = rng.choice(["attn", "attn", "attn", "attn", "write", "write", "verify", "verify"])
    if op == "verify":
        given, t = rng.random() < 0.6, rng.choice(["f32", "f32", "f16", "bf16"])
        vocab, drafts = _spread(rng, 2, 160000), rng.choice([1, 2, 3, 4, 5, 7, 8, 11, 16])
        most = (1 << 28) // (vocab * (drafts + 1))           # at most about 1 GiB of probabilities of each kind
        return dict(op=op, batch=_spread(rng, 1, max(1, min(256, most))), drafts=drafts, vocab=vocab, type=t, given=given)
    d, t = rng.choice([64, 80, 128]), rng.choice(["f16", "bf16"])
    hkv, g = rng.choice([1, 2, 5, 8, 32]), rng.choice([1, 1, 2, 3, 4, 7, 8, 12, 16])
    if op == "write":
        new = 1 if rng.random() < 0.4 else _spread(rng, 2, 4096)
        start = rng.choice([0, 16, 500, 4096, 100000])
        most = min((1 << 26) // (new * hkv * (g + 2) * d), (1 << 30) // ((new + start) * hkv * d))   # at most about 4 GiB of cache
        return dict(op=op, batch=_spread(rng, 1, max(1, min(256, most))), new_min=rng.choice([0, 1, new]) if new > 1 else 1, new_max=new,
                    start_min=0, start_max=start, q_heads=hkv * g, kv_heads=hkv, d=d,
                    rotary=rng.choice([d, d, d // 2, 16]), pairs=rng.choice([HALVES, ADJACENT]), axes=rng.choice([1, 1, 3]), type=t)
    new = rng.choice([1, _spread(rng, 2, 16), _spread(rng, 17, 2048)])
    start = _spread(rng, 1, 16384)
    most = min((1 << 31) // ((start + new) * hkv * g * new), (1 << 29) // ((start + new) * hkv * d * 2))
    while most < 1:
        start, new, hkv = start // 2, (new + 1) // 2, max(1, hkv // 2)
        most = min((1 << 31) // ((start + new) * hkv * g * new), (1 << 29) // ((start + new) * hkv * d * 2))
    return dict(op=op, batch=_spread(rng, 1, min(256, most)), new_min=rng.choice([0, 1, new]), new_max=new, start_min=rng.choice([0, start // 2, start]),
                start_max=start, q_heads=hkv * g, kv_heads=hkv, d=d, type=t, softcap=rng.choice([0.0, 0.0, 30.0, 50.0]),
                window=rng.choice([0, 0, 0, _spread(rng, 1, 8192)]), slopes=rng.random() < 0.25, prefix=rng.random() < 0.25)


def work(c):
    B = c["batch"]
    if c["op"] == "verify":
        rows = 2 if c["given"] else 1
        return {"bytes": float(B * c["vocab"] * rows * (4 if c["type"] == "f32" else 2)), "flops": 2.0 * B * c["vocab"] * rows}
    new, start = (c["new_min"] + c["new_max"]) / 2, (c["start_min"] + c["start_max"]) / 2
    q, kv = B * new * c["q_heads"] * c["d"], B * new * c["kv_heads"] * c["d"]
    if c["op"] == "write":
        return {"bytes": 2.0 * (2 * q + 4 * kv), "flops": 3.0 * (q + kv)}
    seen = min(start + new / 2, c["window"] or 1e30)
    read = min(start + new, (c["window"] or 1e30) + new)
    return {"bytes": 2.0 * (2 * q + 2 * B * read * c["kv_heads"] * c["d"]), "flops": 4.0 * seen * q}


# ---------------------------------------------------------------- the cache's layout

def _places(d):
    """[16, d]: where in a row of a tile element e of token t is stored."""
    t, e = torch.arange(BT, device="cuda")[:, None], torch.arange(d, device="cuda")[None]
    return torch.where(e // 64 < d // 64, (((e // 8) ^ (t % 8)) * 8 + e % 8), e.expand(BT, d))


class _Handle:
    """A handle of the framework that is released with the state that keeps it."""

    def __init__(self, made, free):
        self.h, self.free = made, free

    def __del__(self):
        try:
            self.free(self.h)
        except Exception:
            pass


# ---------------------------------------------------------------- inputs

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _ints(g, lo, hi, shape):
    return torch.randint(lo, hi + 1, shape, generator=g, device="cuda", dtype=torch.int32)


def _rows(g, shape, dtype):
    """Rows of q, K or V: normal, one entry in 100 eight times as large."""
    x = torch.randn(shape, generator=g, device="cuda", dtype=dtype)
    return torch.where(torch.rand(shape, generator=g, device="cuda", dtype=dtype) < 0.01, x * 8, x)


def prepare(c, seed):
    g = _gen(seed)
    st = {"case": c}
    B = c["batch"]
    if c["op"] == "verify":
        V, K, t = c["vocab"], c["drafts"], TYPES[c["type"]]
        # a model's probabilities: a few likely tokens; the draft's are near the target's
        logits = torch.randn((B, K + 1, V), generator=g, device="cuda").mul_(3.0)
        st["target"] = torch.softmax(logits, -1).to(t)
        near = torch.softmax(logits[:, :K].add_(torch.randn((B, K, V), generator=g, device="cuda")), -1)
        st["drafted"] = torch.multinomial(near.flatten(0, 1), 1, generator=g).view(B, K).int()
        st["draft"] = near.to(t) if c["given"] else None
        st["n"] = _ints(g, min(1, K - 1), K, (B,))
        st["u"] = torch.rand((B, K + 1), generator=g, device="cuda")
        st["lens"] = _ints(g, 100, 5000, (B,)) + st["n"] + 1
        st["tokens"] = torch.empty((B, K + 1), dtype=torch.int32, device="cuda")
        st["accepted"], st["lens_out"] = (torch.empty(B, dtype=torch.int32, device="cuda") for _ in range(2))
        return st
    t, H, Hq, d = TYPES[c["type"]], c["kv_heads"], c["q_heads"], c["d"]
    st["new"] = new = _ints(g, c["new_min"], c["new_max"], (B,))
    st["lens"] = lens = _ints(g, c["start_min"], c["start_max"], (B,)) + new
    st["T"], st["blocks"] = c["new_max"], max(1, (c["start_max"] + c["new_max"] + BT - 1) // BT)
    # the rows of all sequences stand one behind the other in buffers for the largest chunks; what is behind the last one belongs to nobody
    st["first"] = (torch.cumsum(new, 0) - new).int()
    st["rows"] = rows = B * c["new_max"] + 3
    n = B * st["blocks"] + 5
    st["n"] = n
    st["table"] = torch.randperm(n, generator=g, device="cuda")[:B * st["blocks"]].int().view(B, -1).contiguous()
    # q, K and V come out of one product: a token's row holds all three
    st["qkv"] = _rows(g, (rows, Hq + 2 * H, d), t)
    st["q"], st["k"], st["v"] = st["qkv"][:, :Hq], st["qkv"][:, Hq:Hq + H], st["qkv"][:, Hq + H:]
    if c["op"] == "write":
        st["pool"] = torch.zeros((n, 2, H, BT, d), dtype=t, device="cuda")
        st["freq"] = (10000.0 ** (-torch.arange(c["rotary"] // 2, device="cuda").double() * 2 / c["rotary"])).float()
        st["positions"], st["axis"] = None, None
        if c["axes"] > 1:
            st["positions"] = _ints(g, 0, 40000, (c["axes"], rows))
            st["axis"] = (torch.arange(c["rotary"] // 2, device="cuda") % c["axes"]).to(torch.uint8)
        st["q_out"] = torch.zeros((rows, Hq, d), dtype=t, device="cuda")
    else:
        st["pool"] = torch.cat([_rows(g, (min(8192, n - i), 2, H, BT, d), t) for i in range(0, n, 8192)])
        # what a page holds behind the last token is not read
        last, at = (lens.long() - 1).clamp(min=0), torch.arange(BT, device="cuda")
        page = st["table"].long()[torch.arange(B, device="cuda"), last // BT]
        behind = (at > (last % BT)[:, None])[:, None, None, :, None]
        st["pool"][page] = st["pool"][page].masked_fill(behind, float("nan"))
        st["slopes"] = torch.exp2(-8.0 * torch.arange(1, Hq + 1, device="cuda") / Hq).float() if c["slopes"] else None
        st["prefix"] = (lens * torch.rand(B, generator=g, device="cuda")).int() if c["prefix"] else None
        st["out"] = torch.zeros((rows, Hq, d), dtype=t, device="cuda")
    if own:
        from paper_2504_11816_b200 import binding as F
        st["h"] = _Handle(F.isv_chunk_create(q_heads=Hq, kv_heads=H, head_dim=d, dtype=CODE[c["type"]], max_seqs=B, max_ctas=0,
                                             rotary_dim=c.get("rotary", 0), rotary_pairs=c.get("pairs", 0), rotary_axes=c.get("axes", 1),
                                             scale=0.0, softcap=c.get("softcap", 0.0)), F.isv_chunk_free)
    return st


# ---------------------------------------------------------------- one pass

def run(st):
    return {"attn": _attn, "write": _write, "verify": _verify}[st["case"]["op"]](st)


def _padded(st):
    """Of token t of each sequence's chunk: its row (one behind the last where there is none), its position, whether it exists."""
    t = torch.arange(st["T"], device="cuda")
    there = t < st["new"][:, None]
    return torch.where(there, st["first"][:, None] + t, st["rows"]).long(), (st["lens"] - st["new"])[:, None] + t, there


def _attn(st):
    c = st["case"]
    if own:
        from paper_2504_11816_b200 import binding as F
        F.isv_chunk_attn(st["h"].h, st["pool"], st["n"], st["table"], st["blocks"], st["blocks"], st["lens"], st["new"], st["first"], st["rows"],
                         st["q"], st["q"].stride(0), st["slopes"], st["prefix"], c["window"], st["out"], None, c["batch"], st["T"],
                         torch.cuda.current_stream().cuda_stream)
        return st["out"]
    B, H, d, T = c["batch"], c["kv_heads"], c["d"], st["T"]
    G = c["q_heads"] // H
    row, pos, there = _padded(st)
    kv = st["pool"][st["table"].long()]                      # [B, blocks, 2, H, 16, d]
    kv = torch.gather(kv, -1, _places(d).expand(kv.shape)).permute(2, 0, 3, 1, 4, 5).reshape(2, B, H, -1, d).float()
    at = torch.arange(kv.shape[3], device="cuda")
    kv = kv.masked_fill_((at >= st["lens"][:, None])[:, None, :, None], 0.0)
    q = st["q"][row.clamp(max=st["rows"] - 1)].float().view(B, T, H, G, d).permute(0, 2, 3, 1, 4).reshape(B, H, G * T, d)
    s = torch.matmul(q, kv[0].transpose(2, 3)).view(B, H, G, T, -1).mul_(1 / math.sqrt(d))
    if c["softcap"]:
        s = s.div_(c["softcap"]).tanh_().mul_(c["softcap"])
    if st["slopes"] is not None:
        s -= st["slopes"].view(1, H, G, 1, 1) * (pos[..., None] - at).abs()[:, None, None].float()
    seen = at <= pos[..., None]
    if c["window"]:
        seen &= at > pos[..., None] - c["window"]
    if st["prefix"] is not None:
        seen |= at < st["prefix"][:, None, None]
    seen &= (at < st["lens"][:, None])[:, None]
    s.masked_fill_(~seen[:, None, None], float("-inf"))
    top = s.amax(-1, keepdim=True)
    e = s.sub_(torch.where(torch.isinf(top), torch.zeros_like(top), top)).exp_()
    total = e.sum(-1, keepdim=True)
    o = torch.matmul(e.view(B, H, G * T, -1), kv[1]).view(B, H, G, T, d) / torch.where(total > 0, total, torch.ones_like(total))
    out = torch.zeros((st["rows"] + 1,) + st["q"].shape[1:], dtype=st["q"].dtype, device="cuda")
    out[row] = o.permute(0, 3, 1, 2, 4).reshape(B, T, -1, d).to(out.dtype)
    return out[:-1]


def _rotated(c, x, angle):
    """x [..., heads, d] in fp32 turned by angle [..., pairs] (64 bits)."""
    cos, sin = angle.cos().float()[..., None, :], angle.sin().float()[..., None, :]
    r = c["rotary"]
    a, b = (x[..., :r // 2], x[..., r // 2:r]) if c["pairs"] == HALVES else (x[..., 0:r:2], x[..., 1:r:2])
    a, b = a * cos - b * sin, b * cos + a * sin
    both = torch.cat([a, b], -1) if c["pairs"] == HALVES else torch.stack([a, b], -1).flatten(-2)
    return torch.cat([both, x[..., r:]], -1)


def _write(st):
    c = st["case"]
    if own:
        from paper_2504_11816_b200 import binding as F
        F.isv_chunk_write(st["h"].h, st["pool"], st["n"], st["table"], st["blocks"], st["blocks"], st["lens"], st["new"], st["first"], st["rows"],
                          st["k"], st["v"], st["k"].stride(0), st["q"], st["q"].stride(0), st["q_out"], st["freq"], st["positions"], st["axis"], 1.0,
                          c["batch"], st["T"], torch.cuda.current_stream().cuda_stream)
        return {"pool": st["pool"], "q": st["q_out"]}
    row, pos, there = _padded(st)
    inside = row.clamp(max=st["rows"] - 1)
    if st["positions"] is None:
        angle = pos[..., None].double() * st["freq"].double()
    else:
        angle = st["positions"][:, inside][st["axis"].long()].permute(1, 2, 0).double() * st["freq"].double()
    k = _rotated(c, st["k"][inside].float(), angle).to(st["k"].dtype)
    places = _places(c["d"])[pos % BT]                       # [B, T, d]
    page, slot = torch.gather(st["table"].long(), 1, (pos // BT).clamp(max=st["blocks"] - 1))[there], (pos % BT)[there]
    for i, x in enumerate((k, st["v"][inside])):
        st["pool"][page, i, :, slot] = torch.zeros_like(x).scatter_(-1, places[:, :, None].expand(x.shape), x)[there]
    q = torch.zeros((st["rows"] + 1,) + st["q"].shape[1:], dtype=st["q"].dtype, device="cuda")
    q[row] = _rotated(c, st["q"][inside].float(), angle).to(q.dtype)
    return {"pool": st["pool"], "q": q[:-1]}


def _verify(st):
    c = st["case"]
    B, K, V = c["batch"], c["drafts"], c["vocab"]
    if own:
        from paper_2504_11816_b200 import binding as F
        F.isv_draft_verify(st["target"], None, B * (K + 1), st["draft"], V, CODE[c["type"]], st["drafted"], st["n"], st["u"], st["lens"], B, K,
                           st["tokens"], st["accepted"], st["lens_out"], None, torch.cuda.current_stream().cuda_stream)
        return {"tokens": st["tokens"], "accepted": st["accepted"], "lens": st["lens_out"]}
    x, n, row = st["drafted"].long(), st["n"].long(), torch.arange(B, device="cuda")
    p = torch.gather(st["target"][:, :K], 2, x[..., None])[..., 0].double()
    q = torch.gather(st["draft"], 2, x[..., None])[..., 0].double() if c["given"] else torch.ones_like(p)
    step = torch.arange(K, device="cuda")
    good = (st["u"][:, :K].double() * q < p) & (step < n[:, None])
    took = torch.cumprod(good.long(), 1).sum(1)
    refused = took < n
    left = st["target"][row, took].double()
    at = took.clamp(max=K - 1)
    if c["given"]:
        less = (left - st["draft"][row, at].double()).clamp(min=0)
    else:
        less = left.scatter(1, x[row, at][:, None], 0.0)
    left = torch.where((refused & (less.sum(1) > 0))[:, None], less, left)
    up = torch.cumsum(left, 1)
    above = up > st["u"][:, K].double()[:, None] * up[:, -1:]
    chosen = torch.where(above, torch.arange(V, device="cuda"), V).amin(1)
    tokens = torch.full((B, K + 1), -1, dtype=torch.int32, device="cuda")
    tokens[:, :K] = torch.where(step < took[:, None], st["drafted"], -1)
    tokens[row, took] = chosen.int()
    return {"tokens": tokens, "accepted": took.int(), "lens": (st["lens"] - n + took).int()}


# ---------------------------------------------------------------- the definition in 64 bits

def exact(c, seed):
    if c["op"] == "verify":
        return None                                          # whole numbers: nothing is rounded
    st = prepare(c, seed)
    H, G, d = c["kv_heads"], c["q_heads"] // c["kv_heads"], c["d"]
    lens, new, first = st["lens"].tolist(), st["new"].tolist(), st["first"].tolist()
    where = _places(d)
    if c["op"] == "write":
        if sum(new) > 1 << 17:
            return None
        pool = torch.zeros(st["pool"].shape, dtype=torch.float64, device="cuda")
        q_out = torch.zeros(st["q_out"].shape, dtype=torch.float64, device="cuda")
        half = c["rotary"] // 2
        one = torch.arange(half, device="cuda") if c["pairs"] == HALVES else 2 * torch.arange(half, device="cuda")
        two = one + (half if c["pairs"] == HALVES else 1)
        for s in range(c["batch"]):
            if not new[s]:
                continue
            rows = slice(first[s], first[s] + new[s])
            pos = torch.arange(lens[s] - new[s], lens[s], device="cuda")
            angle = (pos[:, None] if st["positions"] is None else st["positions"][:, rows].t()[:, st["axis"].long()]).double() * st["freq"].double()
            turn = torch.polar(torch.ones_like(angle), angle)[:, None]
            turned = []
            for x in (st["q"][rows], st["k"][rows]):
                y = x.double()
                z = torch.complex(y[..., one], y[..., two]) * turn
                y[..., one], y[..., two] = z.real, z.imag
                turned.append(y)
            q_out[rows] = turned[0]
            page, slot = st["table"][s].long()[pos // BT], pos % BT
            for i, x in enumerate((turned[1], st["v"][rows].double())):
                y = torch.empty_like(x)
                y.scatter_(-1, where[slot][:, None].expand(x.shape), x)
                pool[page, i, :, slot] = y
        return {"pool": pool, "q": q_out}
    out = torch.zeros(st["out"].shape, dtype=torch.float64, device="cuda")
    for s in range(c["batch"]):
        n = lens[s]
        if not new[s]:
            continue
        tiles = st["pool"][st["table"][s, :(n + BT - 1) // BT].long()]
        tiles = torch.gather(tiles, -1, where.expand(tiles.shape))
        k, v = (tiles[:, i].transpose(0, 1).reshape(H, -1, d)[:, :n].double() for i in range(2))
        at = torch.arange(n, device="cuda")
        step = max(1, (1 << 27) // (n * G * H))
        for t0 in range(0, new[s], step):
            t1 = min(new[s], t0 + step)
            rows = slice(first[s] + t0, first[s] + t1)
            pos = n - new[s] + torch.arange(t0, t1, device="cuda")
            x = torch.einsum("thgd,hnd->hgtn", st["q"][rows].double().view(t1 - t0, H, G, d), k) / math.sqrt(d)
            if c["softcap"]:
                x = c["softcap"] * torch.tanh(x / c["softcap"])
            far = pos[:, None] - at[None]
            if c["slopes"]:
                x = x - st["slopes"].double().view(H, G, 1, 1) * far.abs()
            hidden = far < 0
            if c["window"]:
                hidden = hidden | (far >= c["window"])
            if c["prefix"]:
                hidden = hidden & (at[None] >= int(st["prefix"][s]))
            x = x.masked_fill(hidden, float("-inf"))
            out[rows] = torch.einsum("hgtn,hnd->thgd", torch.softmax(x, -1), v).reshape(t1 - t0, -1, d)
    return out
