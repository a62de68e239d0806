"""GPU tests of the token-wise calls as a serving engine runs them together: prompts in chunks, single
tokens, blocks that move, captured graphs, several streams, pools full of stale bytes, batches with
holes."""
import numpy as np
import pytest
import torch

from paged_ref import DTYPE, NO_BLOCK, Batch, Shape, attention, pool_values, tolerance
from paper_2504_03648_b200 import binding as aibx
from test_gpu_paged import KIND, POOLS, check_attention, dev, kv_layout, make_batch, make_cache, make_pool

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _clean_status():
    aibx.status_fetch()
    yield


def run(cache, batch, q, **kw):
    out = torch.empty_like(q)
    lse = torch.empty(q.shape[:2], device="cuda")
    aibx.attn_paged(cache, batch, q, out, lse=lse, **kw)
    return out, lse


def same(a, b):
    return all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(a, b))


@pytest.mark.parametrize("pool,io", POOLS)
def test_prompts_in_chunks_then_tokens_then_other_blocks(pool, io):
    """Write, attend, write more, attend; then every block moves elsewhere (rows and scale bytes by
    the block copies) and the last step gives the same bits from the new places."""
    s = Shape(H=2, D=64, T=16, layout=1, pool=pool, blocks=80)
    rng = np.random.default_rng(9)
    total = [150, 37, 260]
    b_all = Batch(rng, s, total, total)
    x = {n: torch.from_numpy(rng.normal(size=(sum(total), h, s.D))).to(DTYPE[io]) for n, h in (("q", 8), ("k", 2), ("v", 2))}
    p, sc = make_pool(rng, s)
    cache = make_cache(s, p, sc)
    done, last = [0, 0, 0], None
    for step in ([100, 5, 200], [49, 0, 59], [1, 31, 0], [0, 1, 1]):
        b = Batch.__new__(Batch)
        b.new, b.length = step, [d + n for d, n in zip(done, step)]
        b.table, b.blk_off = b_all.table, None
        b.tok_off = np.concatenate([[0], np.cumsum(step)]).astype(np.int64)
        b.kv_len, b.n_tokens = np.array(b.length, dtype=np.int32), sum(step)
        rows = np.concatenate([np.arange(d, d + n) + o for d, n, o in zip(done, step, b_all.tok_off)])
        batch = make_batch(b)
        aibx.kv_append(cache, batch, x["k"][rows].cuda(), x["v"][rows].cuda())
        got = run(cache, batch, x["q"][rows].cuda())
        host = cache._keep[0].cpu()
        values = pool_values(s, host.view(torch.float8_e4m3fn) if pool == "e4m3" else host,
                             None if sc is None else cache._keep[1].cpu().numpy())
        want, wl, mag, slack = attention(s, b, values, x["q"][rows].double().numpy(), s.D ** -0.5, True, 0)
        err = np.abs(got[0].double().cpu().numpy() - want)
        assert (err <= tolerance(s, io, want, mag, slack)).all()
        done, last = b.length, (b, rows, got)
    # the blocks go to other places of another pool
    b, rows, got = last
    used = b_all.table[b_all.table != NO_BLOCK]
    to = rng.permutation(s.blocks)[:len(used)].astype(np.uint32)
    lay = kv_layout(s)
    buf = torch.zeros(len(used) * lay.block_bytes, dtype=torch.uint8, device="cuda")
    aibx.kv_gather(cache._keep[0], lay, dev(used), len(used), buf)
    p2, sc2 = make_pool(rng, s)
    other = make_cache(s, p2, sc2)
    aibx.kv_scatter(other._keep[0], lay, dev(to), len(used), buf)
    if sc is not None:
        slay = aibx.KVLayout(s.layout, s.layers, s.H, s.T, 1, 1, s.blocks)
        sbuf = torch.zeros(len(used) * slay.block_bytes, dtype=torch.uint8, device="cuda")
        aibx.kv_gather(cache._keep[1], slay, dev(used), len(used), sbuf)
        aibx.kv_scatter(other._keep[1], slay, dev(to), len(used), sbuf)
    where = {int(f): int(t) for f, t in zip(used, to)}
    moved = Batch.__new__(Batch)
    moved.__dict__.update(b.__dict__)
    moved.table = np.array([[where.get(int(e), NO_BLOCK) for e in r] for r in b.table], dtype=np.uint32)
    assert same(run(other, make_batch(moved), x["q"][rows].cuda()), got)
    assert aibx.status_fetch() == (0, 0)


def test_matched_blocks_are_a_table():
    """The block ids that prefix matching leaves, completed with fresh blocks for the unmatched rest, are
    a ragged block table as they stand."""
    import oracle
    T, P = 16, 2
    rng = np.random.default_rng(4)
    s = Shape(H=2, D=64, T=T, blocks=64, pool="bf16")
    tokens = rng.integers(0, 1000, (2, 96)).astype(np.int32)
    tokens[1, :64] = tokens[0, :64]                             # four shared blocks
    tok_off = np.array([0, 96, 192], dtype=np.int64)
    blk_off = oracle.block_offsets(tok_off, T)
    keys = torch.empty(12, dtype=torch.uint64, device="cuda")
    aibx.hash_blocks(dev(tokens.reshape(-1)), dev(tok_off), dev(blk_off), T, 0, keys)
    index = aibx.Index(64, P)
    first = torch.arange(20, 26).to(torch.int32).cuda().view(torch.uint32)      # request 0's blocks
    index.insert(keys[:6], dev(np.full(6, 1, dtype=np.uint64)), first)
    ids = torch.empty(12, dtype=torch.uint32, device="cuda")
    length = torch.empty(2 * P, dtype=torch.uint32, device="cuda")
    any_len = torch.empty(2, dtype=torch.uint32, device="cuda")
    index.match_prefix(keys, dev(blk_off), length, any_len, ids)
    assert any_len.cpu().tolist() == [6, 4]
    table = ids.view(torch.int32)
    table[10:] = torch.tensor([40, 41], dtype=torch.int32)      # request 1: two blocks of its own
    x = {n: torch.from_numpy(rng.normal(size=(96, h, 64))).bfloat16().cuda() for n, h in (("q", 4), ("k", 2), ("v", 2))}
    pool, _ = make_pool(rng, s)
    cache = make_cache(s, pool, None)

    def batch(new, lens):
        off = np.concatenate([[0], np.cumsum(new)]).astype(np.int64)
        return aibx.KVBatch(table.view(torch.uint32), dev(off), dev(np.array(lens, dtype=np.int32)), int(sum(new)),
                            blk_off=dev(blk_off))

    aibx.kv_append(cache, batch([96, 0], [96, 0]), x["k"], x["v"])           # request 0 fills the blocks
    tail = slice(64, 96)                                                     # request 1 computes its rest only
    aibx.kv_append(cache, batch([0, 32], [96, 96]), x["k"][tail] * 2, x["v"][tail] * 2)
    got, _ = run(cache, batch([0, 32], [96, 96]), x["q"][tail].contiguous())
    k, v = [torch.cat([x[n][:64], x[n][tail] * 2]).double().cpu().repeat_interleave(2, 1) for n in "kv"]
    z = torch.einsum("qhd,khd->hqk", x["q"][tail].double().cpu(), k) / 8
    z.masked_fill_(torch.arange(96)[None, None] > torch.arange(64, 96)[None, :, None], -np.inf)
    w = torch.softmax(z, -1)
    want, mag = torch.einsum("hqk,khd->qhd", w, v), torch.einsum("hqk,khd->qhd", w, v.abs())
    # weights and result rounded to bf16 (2^-8 each), scores and sums far below that
    assert ((got.double().cpu() - want).abs() <= (2.0 ** -8 + 2.0 ** -14) * mag + 2.0 ** -8 * want.abs()).all()
    assert aibx.status_fetch() == (0, 0)


@pytest.mark.parametrize("pool,io", POOLS)
@pytest.mark.parametrize("new", [1, 70])
def test_stale_slots_do_not_matter(pool, io, new):
    """Every slot that no visible position names holds NaN or infinities (and, in an e4m3 pool, NaN
    scale bytes): the same bits as from a clean pool."""
    s = Shape(H=2, D=64 if pool == "fp16" else 128, T=16, pool=pool, blocks=90)
    rng = np.random.default_rng(8)
    lens = [new + c for c in (0, 5, 130, 300)]
    b = Batch(rng, s, [new] * 4, lens)
    p, sc = make_pool(rng, s)
    q = torch.from_numpy(rng.normal(size=(b.n_tokens, 8, s.D))).to(DTYPE[io]).cuda()
    for window in (0, 20):
        live = np.zeros(s.rows, dtype=bool)
        for r, L in enumerate(lens):
            for pos in range(max(0, L - new - window + 1) if window else 0, L):
                for kv in range(2):
                    for h in range(s.H):
                        live[s.row(b.entry(s, r, pos), kv, h, pos % s.T)] = True
        bad, bsc = p.clone(), None if sc is None else sc.copy()
        stale = torch.from_numpy(~live)
        if pool == "e4m3":
            bad.view(torch.uint8)[stale] = 0x7f
            bsc[~live] = 255
        else:
            bad[stale] = float("nan")
            bad[stale.nonzero()[::2, 0]] = float("inf")
        want = run(make_cache(s, p, sc), make_batch(b), q, window=window)
        got = run(make_cache(s, bad, bsc), make_batch(b), q, window=window)
        assert torch.isfinite(got[0]).all() and same(got, want)


@pytest.mark.parametrize("pool,io", POOLS)
@pytest.mark.parametrize("new", [1, 40])
def test_missing_blocks_and_short_tables(pool, io, new):
    s = Shape(H=1, D=64, T=8, pool=pool, blocks=200)
    rng = np.random.default_rng(11)
    lens = [200, 333, new + 2, 150]
    b = Batch(rng, s, [new] * 4, lens, pad=1)
    b.table[0, 3:9] = NO_BLOCK                                  # a hole
    b.table[1, :] = NO_BLOCK                                    # nothing there at all: empty rows
    st, out, lse = check_attention(s, b, io, G=2)
    assert st == (0, 0)
    assert (lse[new:2 * new] == -np.inf).all() and (out[new:2 * new] == 0).all()
    b.table[2, 0] = s.blocks + 7                                # out of range
    st, _, _ = check_attention(s, b, io, G=2)
    assert st[0] == aibx.ERR_RANGE and st[1] >= 1
    b = Batch(rng, s, [new, new], [300, 200], width=20)         # tables end at position 160
    st, _, _ = check_attention(s, b, io, G=2)
    assert st[0] == aibx.ERR_RANGE and st[1] >= 2


@pytest.mark.parametrize("pool,io", POOLS)
@pytest.mark.parametrize("new", [3, 90])
def test_rows_before_the_first_position(pool, io, new):
    """kv_len below the tokens of the call: rows at negative positions see nothing (causal), or all."""
    s = Shape(H=2, D=128, T=16, pool=pool, blocks=20)
    b = Batch(np.random.default_rng(2), s, [new] * 3, [0, 2, new - 1])
    for causal in (True, False):
        st, out, _ = check_attention(s, b, io, G=3, causal=causal)
        assert st == (0, 0) and (out[:new] == 0).all()


def test_more_tokens_than_promised_is_reported():
    s = Shape(H=1, D=64, T=16, blocks=30)
    b = Batch(np.random.default_rng(1), s, [1, 40], [20, 60])
    pool, _ = make_pool(np.random.default_rng(1), s)
    q = torch.ones(41, 2, 64, dtype=torch.bfloat16, device="cuda")
    run(make_cache(s, pool, None), make_batch(b, max_new=1), q)
    st = aibx.status_fetch()
    assert st == (aibx.ERR_RANGE, 1)


@pytest.mark.parametrize("pool,io", [("bf16", "bf16"), ("e4m3", "fp16")])
@pytest.mark.parametrize("new,G", [(1, 4), (20, 2)])
def test_more_requests_than_threads(pool, io, new, G):
    R = 1500
    s = Shape(H=1, D=64, T=8, pool=pool, blocks=R * 5, layers=1, layer=0)
    rng = np.random.default_rng(R)
    lens = rng.integers(new, 40, R)
    ns = [new if i % 7 else 0 for i in range(R)]
    b = Batch(rng, s, ns, [int(x) for x in lens], ragged=True)
    st, _, _ = check_attention(s, b, io, G=G, max_new=new)
    assert st == (0, 0)


@pytest.mark.parametrize("pool,io", POOLS)
@pytest.mark.parametrize("new", [1, 33])
def test_scores_that_keep_growing(pool, io, new):
    """Keys whose scores rise along the sequence, far past what the running maximum allows without being
    moved, and then fall again."""
    s = Shape(H=1, D=64, T=16, pool=pool, blocks=80, layers=1, layer=0)
    L = 900
    b = Batch(np.random.default_rng(3), s, [new], [L])

    def change(pool_, scales):
        for pos in range(L):
            i = s.row(b.entry(s, 0, pos), 0, 0, pos % s.T)
            up = (pos if pos < 600 else 1200 - pos) / 30.0
            if pool == "e4m3":
                pool_[i] = torch.full((64,), float(min(up * 4, 448))).to(torch.float8_e4m3fn)
                scales[i] = 127 - 3 + (pos % 3)
            else:
                pool_[i] = up / 2
        return pool_, scales

    st, _, _ = check_attention(s, b, io, G=4, change=change, spread=1.5)
    assert st == (0, 0)


@pytest.mark.parametrize("new", [1, 100])
def test_nan_in_what_a_row_sees_reaches_it(new):
    s = Shape(H=2, D=64, T=16, blocks=40)
    rng = np.random.default_rng(6)
    b = Batch(rng, s, [new], [new + 200])
    for kv in range(2):
        pool, _ = make_pool(rng, s)
        pool[s.row(b.entry(s, 0, 77), kv, 0, 77 % 16), 5] = float("nan")
        q = torch.from_numpy(rng.normal(size=(new, 4, 64))).bfloat16().cuda()
        out, lse = run(make_cache(s, pool, None), make_batch(b), q)
        hit = out[:, :2] if kv == 0 else out[:, :2, 5]
        assert torch.isnan(hit).all() and torch.isfinite(out[:, 2:]).all()
        assert torch.isnan(lse[:, :2]).all() == (kv == 0) and torch.isfinite(lse[:, 2:]).all()


@pytest.mark.parametrize("pool,io", [("bf16", "bf16"), ("e4m3", "bf16")])
def test_captured_and_replayed(pool, io):
    """One graph of a decoding step (write, attend) and of a chunk, replayed as lengths and tokens change,
    gives the bits of the eager calls; two graphs that share a workspace run one after the other."""
    s = Shape(H=2, D=128, T=16, pool=pool, blocks=120)
    rng = np.random.default_rng(12)
    p, sc = make_pool(rng, s)
    some = Shape(H=2, D=128, T=16, pool=pool, blocks=100)      # the others wait to be handed out
    cases = []
    for new, lens in ((1, [100, 311, 40]), (50, [70, 200, 50])):
        b = Batch(rng, some, [new] * 3, lens, spare=6)
        k, v = (torch.empty(b.n_tokens, 2, 128, dtype=DTYPE[io], device="cuda") for _ in range(2))
        q = torch.empty(b.n_tokens, 8, 128, dtype=DTYPE[io], device="cuda")
        cases.append((b, make_batch(b), q, k, v, torch.empty_like(q)))
    cache, eager = make_cache(s, p, sc), make_cache(s, p, sc)
    ws = torch.empty(max(aibx.attn_workspace_bytes(cache, c[1], c[2]) for c in cases), dtype=torch.uint8, device="cuda")

    def step(cache, c, out):
        aibx.kv_append(cache, c[1], c[3], c[4])
        aibx.attn_paged(cache, c[1], c[2], out, workspace=ws)

    for c in cases:
        for x in c[2:5]:
            x.normal_()
        step(cache, c, c[5])
    torch.cuda.synchronize()
    graphs = []
    for c in cases:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step(cache, c, c[5])
        graphs.append(g)
    cache._keep[0].copy_(eager._keep[0])
    if sc is not None:
        cache._keep[1].copy_(eager._keep[1])
    for turn in range(4):
        for c, g in zip(cases, graphs):
            for x in c[2:5]:
                x.normal_()
            ids, length = c[1]._keep[0].view(torch.int32), c[1]._keep[2]
            length += turn % 2
            for r in range(3):                              # a block for the token that was added
                need = (int(length[r]) + 15) // 16
                if int(ids[r, need - 1]) == -1:
                    ids[r, need - 1] = 100 + 3 * cases.index(c) + r
            g.replay()
            want = torch.empty_like(c[5])
            step(eager, c, want)
            assert torch.equal(c[5].view(torch.int16), want.view(torch.int16)), turn
    assert torch.equal(cache._keep[0].view(torch.uint8), eager._keep[0].view(torch.uint8))
    assert aibx.status_fetch() == (0, 0)


def test_streams_side_by_side():
    s = Shape(H=2, D=128, T=16, pool="bf16", blocks=160)
    rng = np.random.default_rng(13)
    pool, _ = make_pool(rng, s)
    cache = make_cache(s, pool, None)
    jobs = []
    for new, lens in ((1, [400, 600]), (90, [500, 300]), (1, [90, 100, 110]), (30, [40, 200])):
        b = Batch(rng, s, [new] * len(lens), lens)
        q = torch.randn(b.n_tokens, 8, 128, device="cuda").bfloat16()
        batch = make_batch(b)
        jobs.append((batch, q, run(cache, batch, q), torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(10):
        got = []
        for batch, q, _, st in jobs:
            with torch.cuda.stream(st):
                got.append(run(cache, batch, q))
        torch.cuda.synchronize()
        for g, (_, _, want, _) in zip(got, jobs):
            assert same(g, want)
    assert aibx.status_fetch() == (0, 0)


@pytest.mark.parametrize("pool,io", [("bf16", "bf16"), ("e4m3", "fp16")])
def test_strided_queries_and_outputs(pool, io):
    s = Shape(H=2, D=64, T=16, pool=pool, blocks=60)
    rng = np.random.default_rng(14)
    p, sc = make_pool(rng, s)
    cache = make_cache(s, p, sc)
    for new in (1, 60):
        b = Batch(rng, s, [new, new], [new + 70, new + 9])
        batch = make_batch(b)
        qkv = torch.randn(b.n_tokens, 10, 64, device="cuda").to(DTYPE[io])
        want, _ = run(cache, batch, qkv[:, :6].contiguous())
        wide = torch.full((6, b.n_tokens, 72), 7.0, dtype=DTYPE[io], device="cuda")
        aibx.attn_paged(cache, batch, qkv[:, :6], wide[..., :64].transpose(0, 1))
        assert torch.equal(wide[..., :64].transpose(0, 1), want) and (wide[..., 64:] == 7.0).all()


def test_pool_past_32_bit_offsets():
    """Rows beyond 4 GB from the pool's start, and beyond 2^31 rows' worth of bytes: the same bits as from a
    small pool."""
    big = Shape(H=8, D=128, T=16, layers=2, layer=1, blocks=45000, layout=2)      # 5.9 GB
    small = Shape(H=8, D=128, T=16, layers=1, layer=0, blocks=64, layout=2)
    rng = np.random.default_rng(15)
    pool = torch.empty(big.rows * 128, dtype=torch.bfloat16, device="cuda")
    cb = aibx.KVCache(pool, kv_layout(big), aibx.TYPE_BF16, layer=1)
    cs = aibx.KVCache(torch.empty(small.rows * 128, dtype=torch.bfloat16, device="cuda"), kv_layout(small),
                      aibx.TYPE_BF16)
    for new, lens in ((64, [300, 200]), (1, [301, 201])):
        b = Batch(np.random.default_rng(0), small, lens if new > 1 else [1, 1], lens)
        far = Batch.__new__(Batch)
        far.__dict__.update(b.__dict__)
        far.table = np.where(b.table == NO_BLOCK, NO_BLOCK, b.table + 44000).astype(np.uint32)
        k, v = (torch.randn(b.n_tokens, 8, 128, device="cuda").bfloat16() for _ in range(2))
        for c, x in ((cb, far), (cs, b)):
            aibx.kv_append(c, make_batch(x), k, v)
        back = [[torch.empty_like(k) for _ in range(2)] for _ in range(2)]
        aibx.kv_read(cb, make_batch(far), *back[0])
        assert torch.equal(back[0][0], k) and torch.equal(back[0][1], v)
        q = torch.randn(b.n_tokens, 32, 128, device="cuda").bfloat16()
        assert same(run(cb, make_batch(far), q), run(cs, make_batch(b), q))
    assert aibx.status_fetch() == (0, 0)


def test_other_devices_tensors_are_refused():
    s = Shape(H=1, D=64, T=16, blocks=8)
    pool, _ = make_pool(np.random.default_rng(0), s)
    b = Batch(np.random.default_rng(0), s, [2], [9])
    cache, batch = make_cache(s, pool, None), make_batch(b)
    x = torch.zeros(2, 1, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        aibx.kv_append(cache, batch, x, x)
    with pytest.raises(ValueError):
        aibx.attn_paged(cache, batch, x.cuda(), x)
    with pytest.raises(ValueError):
        aibx.attn_paged(cache, batch, x.cuda()[:1], x.cuda()[:1])
    with pytest.raises(ValueError):
        aibx.KVCache(pool[:-1].cuda(), kv_layout(s), aibx.TYPE_BF16)
