"""Operators around a step of an engine on the paged KV pool, as cases for measurement: block tables,
positions and slot maps from request lengths; rotary positions, alone and on the way into the pool;
ancestor masks of drafted tokens, and attention of such a tree over the cache.

``run`` makes the library's calls where ``own`` is true and computes the same in elementary torch
operations where it is not; ``exact`` computes it from the definition in 64 bits.
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


# ------------------------------------------------------------------------------------------
# cases


def _case(name, op, **kw):
    c = dict(op=op, requests=1, new_lo=1, new_hi=1, ctx_lo=0, ctx_hi=0, q_heads=32, kv_heads=8, dim=128,
             block=16, pool="bf16", io="bf16", layout=0, inner=0, layers=2, layer=1, window=0, words=1,
             rotary=128, interleaved=False, base=10000.0, scaling="none", tree=False, match=False,
             ragged=False)
    c.update(kw)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # a decoding step of 200 running requests: now and then one needs a block more
        _case("tables_single_tokens", "tables", requests=200, ctx_lo=100, ctx_hi=8000),
        # prompts whose prefix was matched are admitted: rows start with the matched blocks
        _case("tables_prompts", "tables", requests=96, new_lo=1500, new_hi=16001, ctx_lo=0, ctx_hi=60000,
              block=32, match=True),
        # the draft of 12 requests, 26 nodes each
        _case("masks_drafts", "masks", requests=12, new_lo=26, new_hi=26, ctx_lo=500, ctx_hi=4000),
        # wide drafts for a whole batch
        _case("masks_wide", "masks", requests=250, new_lo=300, new_hi=512, ctx_lo=500, ctx_hi=4000, words=8),
        # queries of a short chunk, half of each head rotated, interleaved pairs
        _case("rope_short_partial", "rope", new_lo=19, new_hi=19, ctx_lo=777, ctx_hi=777, rotary=64,
              interleaved=True),
        # the queries of a long prompt, positions scaled for a long context
        _case("rope_long", "rope", new_lo=40001, new_hi=40001, ctx_lo=90000, ctx_hi=90000, io="fp16",
              base=500000.0, scaling="parts"),
        # a decoding step of 64 requests: queries rotated, K rotated and V as it is into the pool
        _case("rope_append_single_tokens", "rope_append", requests=64, ctx_lo=200, ctx_hi=1500),
        # uncached rests of prompts into the 8-bit pool
        _case("rope_append_chunks_e4m3", "rope_append", requests=24, new_lo=700, new_hi=1500, ctx_lo=2000,
              ctx_hi=6001, q_heads=28, kv_heads=4, block=32, pool="e4m3", layout=1, base=1000000.0,
              scaling="linear"),
        # one user's draft: latency
        _case("tree_one", "attn_tree", new_lo=26, new_hi=26, ctx_lo=1999, ctx_hi=1999),
        # four drafted tokens each for 48 requests
        _case("tree_few_nodes", "attn_tree", requests=48, new_lo=4, new_hi=4, ctx_lo=1000, ctx_hi=8000),
        # drafts of 10 to 60 nodes for 32 requests
        _case("tree_drafts", "attn_tree", requests=32, new_lo=10, new_hi=60, ctx_lo=2000, ctx_hi=8000),
        # 64 nodes over long contexts of the 8-bit pool, 7 query heads share one
        _case("tree_long_e4m3", "attn_tree", requests=4, new_lo=64, new_hi=64, ctx_lo=60000, ctx_hi=131000,
              q_heads=28, kv_heads=4, block=32, pool="e4m3", layers=1, layer=0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["tables", "masks", "rope", "rope_append", "rope_append", "attn_tree", "attn_tree",
                     "attn_tree"])
    kv_heads, group = rng.choice([(1, 8), (2, 5), (4, 7), (8, 4), (8, 8), (8, 1), (4, 4)])
    pool = rng.choice(["bf16", "fp16", "e4m3", "e4m3"])
    io = pool if pool != "e4m3" else rng.choice(["bf16", "fp16"])
    if op in ("rope", "rope_append"):
        io = rng.choice(["bf16", "fp16", "fp32"])
    dim = rng.choice([64, 128])
    kw = dict(kv_heads=kv_heads, q_heads=kv_heads * group, dim=dim, block=rng.choice([8, 16, 24, 32, 64]),
              pool=pool, io=io, layout=rng.randrange(3), inner=rng.randrange(2), layers=2,
              layer=rng.randrange(2), rotary=rng.choice([dim, dim, dim // 2, 32]),
              interleaved=rng.random() < 0.4, base=rng.choice([10000.0, 500000.0, 1000000.0]),
              scaling=rng.choice(["none", "linear", "parts"]))
    if op == "tables":
        R = _log(rng, 1, 1000)
        new = rng.choice([1, 1, _log(rng, 1, 60), _log(rng, 1, 700000 // R)])
        ctx = _log(rng, 1, min(100000, 2000000 // R))
        return _case(None, op, requests=R, new_lo=max(1, int(new * rng.random())), new_hi=new,
                     ctx_lo=int(ctx * rng.random()), ctx_hi=ctx, match=rng.random() < 0.5,
                     ragged=rng.random() < 0.4, **kw)
    if op == "masks":
        words = rng.choice([1, 1, 2, 3, 5, 8])
        R = _log(rng, 1, 250)
        most = _log(rng, 1, 64 * words)
        return _case(None, op, requests=R, new_lo=max(1, int(most * rng.uniform(0.3, 1))), new_hi=most,
                     ctx_lo=0, ctx_hi=_log(rng, 1, 100000), words=words, **kw)
    if op == "rope":
        n = _log(rng, 1, 40000)
        return _case(None, op, new_lo=n, new_hi=n, ctx_lo=0, ctx_hi=_log(rng, 1, 1000000), **kw)
    if op == "rope_append":
        total = _log(rng, 16, 25000)
        R = min(total, _log(rng, 1, 100))
        per = max(1, total // R)
        ctx = _log(rng, 1, 4000)
        tree = per <= 64 and rng.random() < 0.3
        return _case(None, op, requests=R, new_lo=max(1, int(per * rng.uniform(0.3, 1.0))), new_hi=per,
                     ctx_lo=ctx // 2, ctx_hi=ctx, tree=tree, **kw)
    words = rng.choice([1, 1, 1, 2, 4])
    nodes = _log(rng, 2, rng.choice([8, 64, 64 * words]))
    R = _log(rng, 1, max(1, min(64, 2500 // nodes)))
    ctx = _log(rng, 16, min(100000, 300000 // R, 500000000 // (R * nodes * kv_heads * group)))
    return _case(None, op, requests=R, new_lo=max(1, int(nodes * rng.uniform(0.2, 1))), new_hi=nodes,
                 ctx_lo=int(ctx * rng.random()), ctx_hi=ctx, words=words,
                 window=rng.choice([0, 0, 0, _log(rng, 16, 4000)]), **kw)


def _spread(lo, hi, n, start):
    """n whole numbers between lo and hi, spread unevenly and always the same."""
    return [lo + int((hi - lo) * ((start + 0.618033988749895 * i) % 1.0) + 0.5) for i in range(n)]


def _lengths(c):
    """(new tokens, tokens in the cache before them) of every request."""
    R = c["requests"]
    new = _spread(c["new_lo"], c["new_hi"], R, 1.0 - 1e-9 if R == 1 else 0.9)
    ctx = _spread(c["ctx_lo"], c["ctx_hi"], R, 1.0 - 1e-9 if R == 1 else 0.37)
    if c["match"]:                                # whole blocks were matched
        ctx = [x // c["block"] * c["block"] for x in ctx]
    return new, ctx


def _up(a, b):
    return -(-a // b)


def work(case):
    c = case
    new, ctx = _lengths(c)
    n, R, H, D, T = sum(new), c["requests"], c["kv_heads"], c["dim"], c["block"]
    io = 4 if c["io"] == "fp32" else 2
    row = D + 1 if c["pool"] == "e4m3" else 2 * D          # bytes of one cached row
    if c["op"] == "tables":
        fresh = sum(_up(a + b, T) - _up(b, T) for a, b in zip(new, ctx))
        kept = sum(_up(b, T) for b in ctx) if c["match"] else sum(b % T != 0 for b in ctx)
        return {"bytes": R * (8 + 12) + 8 * fresh + (8 if c["match"] else 4) * kept + 12 * n, "flops": 0}
    if c["op"] == "masks":
        return {"bytes": 12 * R + n * (4 + 8 * c["words"] + 4), "flops": 0}
    if c["op"] == "rope":
        return {"bytes": n * (4 + 2 * c["q_heads"] * D * io), "flops": 0}
    if c["op"] == "rope_append":
        return {"bytes": n * (2 * c["q_heads"] * D * io + 2 * H * (D * io + row) + (4 if c["tree"] else 0)),
                "flops": 0}
    keys = pairs = 0
    w = c["window"]
    for a, b in zip(new, ctx):
        seen = min(b, w - 1) if w else b
        keys += a + seen
        pairs += a * seen + a                     # a node sees itself and a few above it
    return {"bytes": 2 * keys * H * row + n * (c["q_heads"] * (2 * D * io + 4) + 8 * c["words"]),
            "flops": 4 * pairs * c["q_heads"] * D}


# ------------------------------------------------------------------------------------------
# inputs


def _frequencies(c):
    """Radians per position of every rotated pair, and the factor on sine and cosine."""
    half = c["rotary"] // 2
    f = c["base"] ** (-torch.arange(half, dtype=torch.float64, device="cuda") / half)
    if c["scaling"] == "linear":
        return f / 4.0, 1.0
    if c["scaling"] == "parts":                   # slow pairs stretched 8 times, fast ones kept, a ramp between
        turns = 8192 * f / (2 * math.pi)
        keep = ((turns - 1) / (32 - 1)).clamp(0, 1)
        return f * (keep + (1 - keep) / 8.0), 0.1 * math.log(8.0) + 1.0
    return f, 1.0


def _parents(c, new, g):
    """Parent of every node in its request (-1: the request's last token), flat."""
    n = sum(new)
    first = torch.tensor([0] + new).cumsum(0)[:-1].repeat_interleave(torch.tensor(new)).cuda()
    i = torch.arange(n, device="cuda") - first
    u = torch.rand(n, device="cuda", generator=g, dtype=torch.float64)
    return torch.where(i == 0, -1, (u * i).long().clamp(max=i - 1)).to(torch.int32), first


def _ancestors(parent, first, new):
    """[n][most] truth values: whether node j of the request is node i or above it."""
    n, most = parent.numel(), max(new)
    at = torch.arange(n, device=parent.device)
    seen = torch.zeros(n, most, dtype=torch.bool, device=parent.device)
    up = at
    while True:
        seen[at, up - first[at]] = True
        above = parent[up].long()
        there = above >= 0
        if not bool(there.any()):
            return seen
        at, up = at[there], first[at[there]] + above[there]


def _packed(seen, words):
    """Truth values as bits of 64-bit words, the lowest first."""
    full = torch.zeros(seen.shape[0], 64 * words, dtype=torch.int64, device=seen.device)
    full[:, :seen.shape[1]] = seen
    return (full.view(-1, words, 64) << torch.arange(64, device=seen.device)).sum(-1)


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    new, ctx = _lengths(c)
    kv = [a + b for a, b in zip(new, ctx)]
    R, H, D, T, L = c["requests"], c["kv_heads"], c["dim"], c["block"], c["layers"]
    n = sum(new)
    s = {"c": c, "tokens": n, "max_new": max(new)}
    ints = dict(dtype=torch.int32, device="cuda")

    def normal(count, dtype, spread=1.0):
        t = torch.empty(count, dtype=dtype, device="cuda")
        for part in t.view(-1).split(1 << 28):
            part.copy_(torch.randn(part.numel(), dtype=torch.float16, device="cuda", generator=g).mul_(spread).clamp_(-448, 448))
        return t

    if c["op"] == "tables":
        s["held"], s["new"] = torch.tensor(ctx, **ints), torch.tensor(new, **ints)
        need = [_up(k, T) for k in kv]
        have = [_up(k, T) for k in ctx]
        blocks = sum(need) + 5
        s["blocks"] = blocks
        ids = torch.randperm(blocks, device="cuda", generator=g).to(torch.int32)
        # the free list is a ring that the running engine has gone round before
        fresh = sum(need) - sum(have)
        ring = fresh + 3
        free = ids[:ring]
        s["head"] = torch.tensor([5 * ring + ring // 2], dtype=torch.int64, device="cuda")
        s["tail"] = s["head"] + ring - 1
        s["free"] = free.contiguous().view(torch.uint32)
        s["head_out"] = torch.zeros_like(s["head"])
        other = torch.randint(0, blocks, (sum(have) + 1,), device="cuda", generator=g, dtype=torch.int32)
        s["match_off"] = torch.tensor([0] + have, dtype=torch.int64).cumsum(0).cuda()
        s["match"] = other.view(torch.uint32)
        if c["ragged"]:
            s["blk_off"] = torch.tensor([0] + need, dtype=torch.int64).cumsum(0).cuda()
            start = s["blk_off"][:-1]
            table = torch.full((sum(need),), -1, **ints)
        else:
            s["blk_off"] = None
            start = torch.arange(R, device="cuda") * max(need)
            table = torch.full((R * max(need),), -1, **ints)
        if not c["match"]:                        # rows that were begun earlier
            h = torch.tensor(have, device="cuda")
            e = torch.arange(sum(have), device="cuda")
            r = torch.repeat_interleave(torch.arange(R, device="cuda"), h)
            table[start[r] + e - s["match_off"][r]] = other[:sum(have)]
        s["table"] = (table if c["ragged"] else table.view(R, -1)).view(torch.uint32)
        s["tok_off"] = torch.zeros(R + 1, dtype=torch.int64, device="cuda")
        s["kv_len"] = torch.zeros(R, **ints)
        s["pos"] = torch.zeros(n, **ints)
        s["slots"] = torch.zeros(n, dtype=torch.int64, device="cuda")
        return s

    s["tok_off"] = torch.tensor([0] + new, dtype=torch.int64).cumsum(0).cuda()
    s["kv_len"] = torch.tensor(kv, **ints)
    parent, first = _parents(c, new, g)
    if c["op"] == "masks":
        s["parent"] = parent
        return s
    if c["op"] in ("rope", "rope_append"):
        s["inv_freq"], s["factor"] = _frequencies(c)
    if c["op"] == "rope":
        start = torch.tensor(ctx, device="cuda").repeat_interleave(torch.tensor(new, device="cuda"))
        s["pos"] = (start + torch.arange(n, device="cuda") - first).to(torch.int32)
        s["x"] = normal(n * c["q_heads"] * D, TYPES[c["io"]]).view(n, c["q_heads"], D)
        return s

    need = [_up(k, T) for k in kv]
    blocks = sum(need) + 3
    s["blocks"] = blocks
    elems = blocks * L * 2 * H * T * D
    if c["pool"] == "e4m3":
        s["pool"] = normal(elems, torch.float8_e4m3fn, 80.0).view(torch.uint8)
        s["scales"] = torch.randint(119, 122, (elems // D,), dtype=torch.uint8, device="cuda", generator=g)
    else:
        s["pool"] = normal(elems, TYPES[c["pool"]])
        s["scales"] = None
    ids = torch.randperm(blocks, device="cuda", generator=g).cpu()
    table = torch.full((R, max(need)), -1, dtype=torch.int64)      # "no block" behind the last one
    at = 0
    for r, k in enumerate(need):
        table[r, :k] = ids[at:at + k]
        at += k
    s["table"] = table.to(torch.int32).cuda().view(torch.uint32)
    io = TYPES[c["io"]]
    seen = _ancestors(parent, first, new) if c["op"] == "attn_tree" or c["tree"] else None
    if c["op"] == "rope_append":
        # Q, K and V stand beside one another in one projection's output, as they leave it
        Hq = c["q_heads"]
        qkv = normal(n * (Hq + 2 * H) * D, io).view(n, Hq + 2 * H, D)
        s["q"], s["k"], s["v"] = qkv[:, :Hq], qkv[:, Hq:Hq + H], qkv[:, Hq + H:]
        s["pos"] = None
        if c["tree"]:                             # nodes of a draft stand at their depth
            start = torch.tensor(ctx, device="cuda").repeat_interleave(torch.tensor(new, device="cuda"))
            s["pos"] = (start + seen.sum(-1) - 1).to(torch.int32)
    else:
        s["q"] = normal(n * c["q_heads"] * D, io, 2.0).view(n, c["q_heads"], D)
        s["mask"] = _packed(seen, c["words"]).view(torch.uint64)
    return s


# ------------------------------------------------------------------------------------------
# the framework's calls


def _library(s):
    from paper_2504_03648_b200 import binding as aibx

    c = s["c"]
    size = 1 if c["pool"] == "e4m3" else 2
    lay = aibx.KVLayout(c["layout"], c["layers"], c["kv_heads"], c["block"], c["dim"], size, s["blocks"])
    kind = {"bf16": aibx.TYPE_BF16, "fp16": aibx.TYPE_FP16, "e4m3": aibx.TYPE_E4M3}[c["pool"]]
    cache = aibx.KVCache(s["pool"], lay, kind, scales=s["scales"], inner=c["inner"], layer=c["layer"])
    batch = aibx.KVBatch(s["table"], s["tok_off"], s["kv_len"], s["tokens"], max_new=s["max_new"])
    return aibx, cache, batch


def _run_own(s):
    from paper_2504_03648_b200 import binding as aibx

    c, op = s["c"], s["c"]["op"]
    if op == "tables":
        aibx.kv_tables(s["held"], s["new"], c["block"], s["blocks"], s["free"], s["head"], s["tail"],
                       s["table"], s["tok_off"], s["kv_len"], s["tokens"], pos=s["pos"], slots=s["slots"],
                       head_out=s["head_out"], blk_off=s["blk_off"],
                       match_ids=s["match"] if c["match"] else None,
                       match_off=s["match_off"] if c["match"] else None)
        return {"table": s["table"].view(torch.int32), "tok_off": s["tok_off"], "kv_len": s["kv_len"],
                "pos": s["pos"], "slots": s["slots"], "head": s["head_out"]}
    if op == "masks":
        mask = torch.empty(s["tokens"], c["words"], dtype=torch.uint64, device="cuda")
        pos = torch.empty(s["tokens"], dtype=torch.int32, device="cuda")
        aibx.tree_masks(s["parent"], s["tok_off"], s["kv_len"], mask, pos=pos)
        return {"mask": mask.view(torch.int64), "pos": pos}
    if op in ("rope", "rope_append"):
        rope = aibx.Rope(s["inv_freq"], interleaved=c["interleaved"], factor=s["factor"])
    if op == "rope":
        y = torch.empty_like(s["x"])
        aibx.rope(rope, s["pos"], s["x"], y)
        return {"y": y}
    _, cache, batch = _library(s)
    if op == "rope_append":
        q = torch.empty(s["q"].shape, dtype=s["q"].dtype, device="cuda")
        aibx.rope_append(cache, batch, rope, s["k"], s["v"], q=s["q"], q_out=q, pos=s["pos"])
        return {"q": q, **_pool_out(s)}
    out = torch.empty(s["q"].shape, dtype=s["q"].dtype, device="cuda")
    lse = torch.empty(out.shape[:2], dtype=torch.float32, device="cuda")
    aibx.attn_tree(cache, batch, s["mask"], s["q"], out, lse=lse, window=c["window"])
    return {"out": out, "lse": lse}


# ------------------------------------------------------------------------------------------
# the plain form


def _pool_out(s):
    """The pool after writing: 8-bit rows and scale bytes as the numbers they are."""
    if s["scales"] is None:
        return {"pool": s["pool"]}
    return {"pool": s["pool"].view(torch.float8_e4m3fn), "scales": s["scales"].view(torch.float8_e8m0fnu)}


def _canonical(t, c, blocks, D):
    """The layer's part of a pool as [K/V][block][head][slot][D], a view whatever the layout."""
    H, T, L = c["kv_heads"], c["block"], c["layers"]
    two = (T, H) if c["inner"] else (H, T)
    if c["layout"] == 0:
        v = t.view(blocks, L, 2, *two, D)[:, c["layer"]].transpose(0, 1)
    elif c["layout"] == 1:
        v = t.view(L, blocks, 2, *two, D)[c["layer"]].transpose(0, 1)
    else:
        v = t.view(L, 2, blocks, *two, D)[c["layer"]]
    return v.transpose(2, 3) if c["inner"] else v


def _tables(s):
    c, T = s["c"], s["c"]["block"]
    h, n = s["held"].long(), s["new"].long()
    R, dev = h.numel(), h.device
    off = torch.zeros(R + 1, dtype=torch.int64, device=dev)
    off[1:] = n.cumsum(0)
    had, need = (h + T - 1) // T, (h + n + T - 1) // T
    fresh = need - had
    base = fresh.cumsum(0) - fresh
    start = s["blk_off"][:-1] if c["ragged"] else torch.arange(R, device=dev) * s["table"].shape[1]
    free, flat = s["free"].view(torch.int32), s["table"].view(torch.int32).view(-1)
    if c["match"]:
        e = torch.arange(s["match"].numel() - 1, device=dev)
        r = torch.searchsorted(s["match_off"], e, right=True) - 1
        flat[start[r] + e - s["match_off"][r]] = s["match"].view(torch.int32)[e]
    i = torch.arange(s["tokens"], device=dev)
    r = torch.searchsorted(off, i, right=True) - 1
    pos = h[r] + i - off[r]
    blk = pos // T
    opens = blk >= had[r]                                           # in a block that is new
    where = (s["head"] + base[r] + blk - had[r]) % free.numel()
    at = start[r] + blk
    flat[at[opens]] = free[where[opens]]
    slots = flat[at].long() * T + pos % T
    return {"table": s["table"].view(torch.int32), "tok_off": off, "kv_len": (h + n).to(torch.int32),
            "pos": pos.to(torch.int32), "slots": slots, "head": s["head"] + fresh.sum()}


def _masks(s):
    words, off, n = s["c"]["words"], s["tok_off"], s["tokens"]
    dev = off.device
    i = torch.arange(n, device=dev)
    r = torch.searchsorted(off, i, right=True) - 1
    first, j = off[r], i - off[r]
    up = torch.where(s["parent"] >= 0, first + s["parent"], n)      # node n: above all roots
    seen = torch.zeros(n + 1, 64 * words, dtype=torch.bool, device=dev)
    seen[i, j] = True
    up = torch.cat([up, torch.full((1,), n, device=dev)])
    for _ in range((64 * words).bit_length()):                      # twice as far up each time
        seen = seen | seen[up]
        up = up[up]
    mask = (seen[:n].view(n, words, 64).long() << torch.arange(64, device=dev)).sum(-1)
    base = s["kv_len"].long() - (off[1:] - off[:-1])
    return {"mask": mask, "pos": (base[r] + seen[:n].sum(-1) - 1).to(torch.int32)}


def _rotated(s, x, pos):
    """Rows [n][heads][D] rotated in 32 bits; the angles are reduced in 64."""
    c = s["c"]
    rd = c["rotary"]
    a = pos.double()[:, None] * s["inv_freq"]
    a = a - torch.round(a / (2 * math.pi)) * (2 * math.pi)
    cos, sin = (a.cos() * s["factor"]).float()[:, None], (a.sin() * s["factor"]).float()[:, None]
    x = x.float()
    part = x[..., :rd]
    if c["interleaved"]:
        x1, x2 = part[..., 0::2], part[..., 1::2]
        y = torch.stack([x1 * cos - x2 * sin, x2 * cos + x1 * sin], -1).flatten(-2)
    else:
        x1, x2 = part[..., :rd // 2], part[..., rd // 2:]
        y = torch.cat([x1 * cos - x2 * sin, x2 * cos + x1 * sin], -1)
    return torch.cat([y, x[..., rd:]], -1)


def _power(byte):
    return (byte.to(torch.int32) << 23).view(torch.float32)


def _rope(s):
    return {"y": _rotated(s, s["x"], s["pos"]).to(s["x"].dtype)}


def _rope_append(s):
    c, T, off = s["c"], s["c"]["block"], s["tok_off"]
    i = torch.arange(s["tokens"], device="cuda")
    r = torch.searchsorted(off, i, right=True) - 1
    at = s["kv_len"][r] - (off[r + 1] - i)
    blk, slot = s["table"].view(torch.int32)[r, at // T].long(), at % T
    pos = at if s["pos"] is None else s["pos"]
    q = _rotated(s, s["q"], pos).to(s["q"].dtype)
    x = torch.stack([_rotated(s, s["k"], pos), s["v"].float()])     # [2][n][H][D]
    if c["pool"] != "e4m3":
        _canonical(s["pool"], c, s["blocks"], c["dim"])[:, blk, :, slot] = x.to(s["pool"].dtype).transpose(0, 1)
        return {"q": q, **_pool_out(s)}
    a = torch.where(torch.isfinite(x), x.abs(), 0.0).amax(-1)
    m, e = torch.frexp(a)                                           # a = m * 2^e, 0.5 <= m < 1
    byte = (e - 9 + (m > 0.875)).clamp(-126, 127) + 127             # 448 = 0.875 * 2^9
    byte = torch.where(a > 0, byte, 127)
    y = (x * _power(254 - byte).unsqueeze(-1)).to(torch.float8_e4m3fn)
    _canonical(s["pool"], c, s["blocks"], c["dim"])[:, blk, :, slot] = y.view(torch.uint8).transpose(0, 1)
    _canonical(s["scales"], c, s["blocks"], 1)[:, blk, :, slot] = byte.to(torch.uint8).unsqueeze(-1).transpose(0, 1)
    return {"q": q, **_pool_out(s)}


def _attn_tree(s):
    c, T = s["c"], s["c"]["block"]
    R, H, G, D = c["requests"], c["kv_heads"], c["q_heads"] // c["kv_heads"], c["dim"]
    off, n, N, W = s["tok_off"], s["tokens"], s["max_new"], c["words"]
    i = torch.arange(n, device="cuda")
    r = torch.searchsorted(off, i, right=True) - 1
    j = i - off[r]
    q = torch.zeros(R, N, H, G, D, device="cuda")
    q[r, j] = s["q"].float().view(n, H, G, D)
    bits = torch.zeros(R, N, W, dtype=torch.int64, device="cuda")
    bits[r, j] = s["mask"].view(torch.int64)
    seen = ((bits[..., None] >> torch.arange(64, device="cuda")) & 1).bool().view(R, N, 64 * W)
    table = s["table"].view(torch.int32).long().clamp(min=0)
    L = table.shape[1] * T
    x = _canonical(s["pool"], c, s["blocks"], D)[:, table]          # [2][R][blocks][H][T][D]
    if c["pool"] == "e4m3":
        x = x.view(torch.float8_e4m3fn).float().mul_(_power(_canonical(s["scales"], c, s["blocks"], 1)[:, table]))
    x = x.float().transpose(2, 3).reshape(2, R, H, L, D)
    p = torch.matmul(q.permute(0, 2, 3, 1, 4).reshape(R, H, G * N, D), x[0].transpose(-1, -2))
    p = p.mul_(1.0 / math.sqrt(D)).view(R, H, G, N, L)
    key = torch.arange(L, device="cuda")
    base = s["kv_len"].long() - (off[1:] - off[:-1])
    node = key - base[:, None]                                      # [R][L]
    ok = torch.gather(seen, 2, node.clamp(0, 64 * W - 1)[:, None].expand(R, N, L))
    ok = ok & (node >= 0)[:, None] & (key < s["kv_len"][:, None])[:, None]
    cached = (node < 0)[:, None].expand(R, N, L)
    if c["window"]:
        here = base[:, None] + (seen.sum(-1) - 1).clamp(min=0)
        cached = cached & (key > here[..., None] - c["window"])
    ok = ok | cached
    p.masked_fill_(~ok[:, None, None], -math.inf)
    m = p.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    p.sub_(m).exp_()
    z = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(R, H, G * N, L), x[1]).view(R, H, G, N, D) / torch.where(z > 0, z, 1.0)
    o = o.permute(0, 3, 1, 2, 4)[r, j].reshape(n, H * G, D)
    lse = (m + z.log())[..., 0].permute(0, 3, 1, 2)[r, j].reshape(n, H * G)
    return {"out": o.to(TYPES[c["io"]]), "lse": lse}


def run(state):
    if own:
        return _run_own(state)
    return {"tables": _tables, "masks": _masks, "rope": _rope, "rope_append": _rope_append,
            "attn_tree": _attn_tree}[state["c"]["op"]](state)


# ------------------------------------------------------------------------------------------
# the definition in 64 bits, request by request


def _rows(c, blocks, D, kv, ids, head):
    """Places of one head's rows of the listed blocks, in order: [len(ids) * T][D], straight from offsets."""
    H, T, L = c["kv_heads"], c["block"], c["layers"]
    per = H * T * D
    base = {0: (ids * L + c["layer"]) * 2 * per + kv * per,
            1: (c["layer"] * blocks + ids) * 2 * per + kv * per,
            2: ((c["layer"] * 2 + kv) * blocks + ids) * per}[c["layout"]]
    slot = torch.arange(T, device="cuda")
    row = (slot * H + head) * D if c["inner"] else (head * T + slot) * D
    at = base[:, None, None] + row[None, :, None] + torch.arange(D, device="cuda")
    return at.reshape(-1, D)


def _two(e):
    """2^e of whole numbers, exactly."""
    return torch.tensor([2.0 ** i for i in range(-300, 300)], dtype=torch.float64, device="cuda")[e.long() + 300]


def _row_values(s, kv, ids, head):
    c = s["c"]
    x = s["pool"][_rows(c, s["blocks"], c["dim"], kv, ids, head)]
    if c["pool"] != "e4m3":
        return x.double()
    b = x.long()
    mant, ex = (b & 7).double(), (b >> 3) & 15
    mag = torch.where(ex == 0, mant * 2.0 ** -9, (1 + mant / 8) * _two(ex - 7))
    sc = s["scales"][_rows(c, s["blocks"], 1, kv, ids, head)]
    return torch.where(b >= 128, -mag, mag) * _two(sc.long() - 127)


def _turned(s, x, pos):
    """Rows [n][D] times the rotation's factor as complex numbers."""
    c = s["c"]
    rd = c["rotary"]
    pairs = x[:, :rd].reshape(-1, rd // 2, 2) if c["interleaved"] else x[:, :rd].reshape(-1, 2, rd // 2).transpose(1, 2)
    z = torch.view_as_complex(pairs.contiguous())
    turn = torch.polar(torch.full_like(s["inv_freq"], s["factor"]).expand(pos.numel(), -1), pos.double()[:, None] * s["inv_freq"])
    y = torch.view_as_real(z * turn)
    y = y.reshape(-1, rd) if c["interleaved"] else y.transpose(1, 2).reshape(-1, rd)
    return torch.cat([y, x[:, rd:]], -1)


def _exact_tables(s):
    c, T = s["c"], s["c"]["block"]
    held, new = s["held"].tolist(), s["new"].tolist()
    free, head = s["free"].view(torch.int32).tolist(), int(s["head"])
    table = s["table"].view(torch.int32).view(-1).tolist()
    match, moff = s["match"].view(torch.int32).tolist(), s["match_off"].tolist()
    start = s["blk_off"].tolist() if c["ragged"] else [r * s["table"].shape[1] for r in range(len(held))]
    off, pos, slots = [0], [], []
    for r, (h, n) in enumerate(zip(held, new)):
        row = start[r]
        had = _up(h, T)
        if c["match"]:
            table[row:row + had] = match[moff[r]:moff[r] + had]
        for b in range(had, _up(h + n, T)):
            table[row + b] = free[head % len(free)]
            head += 1
        pos += range(h, h + n)
        slots += [table[row + p // T] * T + p % T for p in range(h, h + n)]
        off.append(off[-1] + n)
    whole = dict(device="cuda")
    return {"table": torch.tensor(table, dtype=torch.int32, **whole).view(s["table"].shape),
            "tok_off": torch.tensor(off, **whole),
            "kv_len": torch.tensor([h + n for h, n in zip(held, new)], dtype=torch.int32, **whole),
            "pos": torch.tensor(pos, dtype=torch.int32, **whole), "slots": torch.tensor(slots, **whole),
            "head": torch.tensor([head], **whole)}


def _exact_masks(s):
    words = s["c"]["words"]
    parent, off, kv = s["parent"].tolist(), s["tok_off"].tolist(), s["kv_len"].tolist()
    rows, pos = [], []
    for r in range(len(kv)):
        bits, depth = [], []
        for i in range(off[r], off[r + 1]):
            p = parent[i]
            bits.append((1 << (i - off[r])) | (bits[p] if p >= 0 else 0))
            depth.append(depth[p] + 1 if p >= 0 else 0)
        base = kv[r] - len(bits)
        pos += [base + d for d in depth]
        for b in bits:
            parts = [(b >> (64 * w)) & (2 ** 64 - 1) for w in range(words)]
            rows.append([x - 2 ** 64 if x >= 2 ** 63 else x for x in parts])
    return {"mask": torch.tensor(rows, dtype=torch.int64, device="cuda"),
            "pos": torch.tensor(pos, dtype=torch.int32, device="cuda")}


def exact(case, seed):
    c = case
    s = prepare(c, seed)
    if c["op"] == "tables":
        return _exact_tables(s)
    if c["op"] == "masks":
        return _exact_masks(s)
    new, ctx = _lengths(c)
    H, G, D, T = c["kv_heads"], c["q_heads"] // c["kv_heads"], c["dim"], c["block"]
    if c["op"] == "rope":
        y = torch.stack([_turned(s, s["x"][:, h].double(), s["pos"]) for h in range(c["q_heads"])], 1)
        return {"y": y}
    table = s["table"].view(torch.int32).long()
    out = torch.zeros(s["tokens"], H * G, D, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["tokens"], H * G, dtype=torch.float64, device="cuda")
    if c["op"] == "rope_append":
        pool = s["pool"] if c["pool"] != "e4m3" else s["pool"].view(torch.float8_e4m3fn)
        pool = pool.double()
        scales = None if s["scales"] is None else _two(s["scales"].long() - 127)
    at = 0
    for r, (n, base) in enumerate(zip(new, ctx)):
        length = base + n
        ids = table[r, :_up(length, T)]
        if c["op"] == "rope_append":
            pos = torch.arange(base, length, device="cuda") if s["pos"] is None else s["pos"][at:at + n]
            for h in range(H * G):
                out[at:at + n, h] = _turned(s, s["q"][at:at + n, h].double(), pos)
            for h in range(H):
                for w, name in enumerate("kv"):
                    x = s[name][at:at + n, h].double()
                    if w == 0:
                        x = _turned(s, x, pos)
                    to = _rows(c, s["blocks"], D, w, ids, h)[base:length]
                    if c["pool"] == "e4m3":
                        a = x.abs().amax(-1)
                        e = torch.ceil(torch.log2(torch.where(a > 0, a, 448.0) / 448.0)).long()
                        e = torch.where(448 * _two(e - 1) >= a, e - 1, e)       # a logarithm may miss a whole number
                        e = torch.where(448 * _two(e) < a, e + 1, e)
                        e = torch.where(a > 0, e, 0)
                        y = x / _two(e)[:, None]
                        low = torch.floor(torch.log2(torch.where(y == 0, 1.0, y.abs()))).long()
                        low = torch.where(_two(low) > y.abs(), low - 1, low)
                        low = torch.where(_two(low + 1) <= y.abs(), low + 1, low).clamp(min=-6)
                        step = _two(low - 3)
                        x = torch.round(y / step) * step
                        scales[_rows(c, s["blocks"], 1, w, ids, h)[base:length, 0]] = _two(e)
                    pool[to] = x
            at += n
            continue
        node = torch.arange(length, device="cuda") - base
        words = s["mask"].view(torch.int64)[at:at + n]
        bit = (words[:, node.clamp(min=0) // 64] >> (node.clamp(min=0) % 64)) & 1
        ok = torch.where(node < 0, 1, bit).bool()
        if c["window"]:
            depth = (bit * (node >= 0)).sum(-1) - 1
            ok &= (node >= 0) | (node > depth[:, None] - c["window"])
        for h in range(H):
            k, v = _row_values(s, 0, ids, h)[:length], _row_values(s, 1, ids, h)[:length]
            for g in range(h * G, (h + 1) * G):
                z = s["q"][at:at + n, g].double() @ k.T / math.sqrt(D)
                z = torch.where(ok, z, -math.inf)
                lse[at:at + n, g] = torch.logsumexp(z, -1)
                out[at:at + n, g] = torch.softmax(z, -1) @ v
        at += n
    if c["op"] == "rope_append":
        return {"q": out, "pool": pool} if scales is None else {"q": out, "pool": pool, "scales": scales}
    return {"out": out, "lse": lse}
