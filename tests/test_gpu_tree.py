"""GPU tests of attention of drafted trees against a plain 64-bit reference."""
import numpy as np
import pytest
import torch

from paged_ref import DTYPE, NO_BLOCK, Batch, Shape, pool_values
from paper_2504_03648_b200 import binding as aibx
from steps_ref import ancestors, pack, random_tree, tree_attention, tree_tolerance
from test_gpu_paged import POOLS, dev, make_batch, make_cache, make_pool

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _clean_status():
    aibx.status_fetch()
    yield


def trees(rng, b, roots=1):
    return [ancestors(random_tree(rng, n, roots)) for n in b.new]


def check_tree(s, b, io="bf16", G=4, window=0, seed=0, spread=1.0, max_new=None, change=None, sets=None, words=1,
               scale=None, junk=0, workspace=None):
    rng = np.random.default_rng(seed)
    pool, scales = make_pool(rng, s)
    if change is not None:
        pool, scales = change(pool, scales)
    sets = trees(rng, b) if sets is None else sets
    Hq = s.H * G
    q = torch.from_numpy(rng.normal(size=(b.n_tokens, Hq, s.D)) * spread).to(DTYPE[io])
    mask = np.full((b.n_tokens, words), junk, dtype=np.uint64)      # bits of nodes that are not there
    for r, n in enumerate(b.new):
        keep = np.array([(0xFFFFFFFFFFFFFFFF << max(0, min(64, n - 64 * w))) & 0xFFFFFFFFFFFFFFFF for w in range(words)], dtype=np.uint64)
        at = slice(int(b.tok_off[r]), int(b.tok_off[r + 1]))
        mask[at] = (mask[at] & keep) | pack(sets[r], words)
    cache, batch = make_cache(s, pool, scales), make_batch(b, max_new)
    out = torch.full((b.n_tokens, Hq, s.D), 7.0, dtype=DTYPE[io], device="cuda")
    ls = torch.full((b.n_tokens, Hq), 7.0, device="cuda")
    scale = s.D ** -0.5 if scale is None else scale
    aibx.attn_tree(cache, batch, dev(mask), q.cuda(), out, lse=ls, scale=scale, window=window, workspace=workspace)
    status = aibx.status_fetch()
    got = out.double().cpu().numpy()
    want, wl, mag, slack = tree_attention(s, b, pool_values(s, pool, scales), q.double().numpy(), scale, sets, window)
    n = int(b.tok_off[-1])
    assert (got[n:] == 7.0).all()
    tol = tree_tolerance(s, io, want[:n], mag[:n], slack[:n])
    err = np.abs(got[:n] - want[:n])
    assert np.isfinite(got[:n]).all()
    assert (err <= tol).all(), (float((err / tol).max()), np.argwhere(err > tol)[:5])
    gl = ls.double().cpu().numpy()
    assert (gl[n:] == 7.0).all()
    empty = np.isinf(wl[:n])
    assert (gl[:n][empty] == -np.inf).all() and (got[:n][empty] == 0).all()
    lt = slack[:n] + 2.0 ** -14 + 2.0 ** -22 * np.abs(np.where(empty, 0, wl[:n]))
    assert (np.abs(gl[:n] - wl[:n])[~empty] <= lt[~empty]).all()
    return status, out, ls


def shape_for(lens, **kw):
    T = kw.get("T", 16)
    return Shape(blocks=sum(-(-max(x, 0) // T) for x in lens) + 2, **kw)


@pytest.mark.parametrize("pool,io", POOLS)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("layout,inner,T", [(0, 0, 16), (1, 1, 8), (2, 0, 24), (2, 1, 256)])
@pytest.mark.parametrize("new", [[1, 3, 4, 0, 2], [26, 0, 17, 5, 32], [64, 33, 40, 1, 0]])
def test_tree(new, layout, inner, T, D, pool, io):
    """Few rows, up to a block, more."""
    lens = [n + c for n, c in zip(new, (0, 40, 300, 1, 95))]
    s = shape_for(lens, H=2, D=D, T=T, layout=layout, inner=inner, pool=pool)
    b = Batch(np.random.default_rng(T), s, new, lens, pad=3, ragged=T == 24)
    st, _, _ = check_tree(s, b, io, G=4, seed=D + T, spread=2.0, junk=0xFFFFFFFFFFFFFFFF)
    assert st == (0, 0)


@pytest.mark.parametrize("G", [1, 3, 7, 16, 40, 128])
@pytest.mark.parametrize("window", [0, 3, 70, 200])
@pytest.mark.parametrize("pool,io", [("bf16", "bf16"), ("e4m3", "bf16")])
def test_tree_one_request(G, window, pool, io):
    """One request alone, whatever its length: several steps cut between pieces, blocks of rows."""
    for n, c in ((1, 0), (2, 131), (16, 1000), (40 if G < 40 else 5, 400), (130 if G < 4 else 9, 77)):
        s = shape_for([n + c], H=1, D=128, T=16, layout=1, pool=pool)
        b = Batch(np.random.default_rng(G), s, [n], [n + c])
        st, _, _ = check_tree(s, b, io, G=G, window=window, seed=window, max_new=0, words=3)
        assert st == (0, 0)


@pytest.mark.parametrize("words,n", [(1, 64), (2, 65), (2, 128), (3, 150), (8, 512)])
@pytest.mark.parametrize("ctx", [0, 7, 128, 333])
def test_tree_many_nodes(words, n, ctx):
    """Masks of several words, at any place in a tile."""
    s = shape_for([n + ctx, 3 + ctx], H=1, D=64, T=8)
    b = Batch(np.random.default_rng(n), s, [n, 3], [n + ctx, 3 + ctx])
    st, _, _ = check_tree(s, b, G=2, words=words, seed=n + ctx)
    assert st == (0, 0)


@pytest.mark.parametrize("pool,io", [("bf16", "bf16"), ("e4m3", "fp16")])
@pytest.mark.parametrize("G,n", [(1, 5), (4, 20), (4, 50)])
def test_rows_that_see_nothing(G, n, pool, io):
    """Masks of any kind: empty, not of itself, all; no cached tokens, so that rows are left empty."""
    rng = np.random.default_rng(G)
    new, lens = [n, n, n], [n, n + 30, n]
    s = shape_for(lens, H=2, D=128, T=16, pool=pool)
    b = Batch(rng, s, new, lens)
    sets = [[set() if i % 3 == 0 else set(rng.choice(n, rng.integers(1, n), replace=False).tolist()) for i in range(n)],
            [set() for i in range(n)], [set(range(n)) for i in range(n)]]
    st, out, lse = check_tree(s, b, io, G=G, sets=sets, seed=n)
    assert st == (0, 0) and bool((lse[:n][::3] == -float("inf")).all())


@pytest.mark.parametrize("G,n", [(2, 5), (4, 20), (4, 60)])
@pytest.mark.parametrize("window", [0, 40])
def test_missing_blocks(G, n, window):
    """Blocks that are not there, bad ids, a table that ends early."""
    lens = [n + 200, n + 60, n + 90]
    s = shape_for(lens, H=2, D=64, T=8)
    b = Batch(np.random.default_rng(n), s, [n] * 3, lens, width=-(-(n + 150) // 8))
    b.table[0, 3] = NO_BLOCK
    b.table[1, 7] = s.blocks + 3
    b.table[2, -(-(n + 90) // 8) - 1] = NO_BLOCK
    st, _, _ = check_tree(s, b, G=G, window=window, seed=n)
    assert st[0] == aibx.ERR_RANGE and st[1] >= 2 - (window > 0)


@pytest.mark.parametrize("G", [2, 4, 8])
def test_a_chain_is_causal_attention(G):
    """The mask of a chain gives attn_paged's result, to the roundings of two orders of sums."""
    new = [20, 7, 33]
    lens = [n + c for n, c in zip(new, (500, 0, 131))]
    s = shape_for(lens, H=2, D=128, T=16)
    rng = np.random.default_rng(3)
    b = Batch(rng, s, new, lens)
    pool, _ = make_pool(rng, s)
    cache, batch = make_cache(s, pool, None), make_batch(b)
    q = torch.from_numpy(rng.normal(size=(b.n_tokens, 2 * G, 128))).bfloat16().cuda()
    mask = dev(np.concatenate([pack([set(range(i + 1)) for i in range(n)], 1) for n in new]))
    a, c = torch.empty_like(q), torch.empty_like(q)
    aibx.attn_paged(cache, batch, q, a)
    aibx.attn_tree(cache, batch, mask, q, c)
    _, _, mag, slack = tree_attention(s, b, pool_values(s, pool, None), q.double().cpu().numpy(), 128 ** -0.5,
                                      [[set(range(i + 1)) for i in range(n)] for n in new], 0)
    tol = 2 * tree_tolerance(s, "bf16", a.double().cpu().numpy(), mag, slack)
    assert (np.abs(a.double().cpu().numpy() - c.double().cpu().numpy()) <= tol).all()


def test_hidden_nodes_may_hold_anything_in_k():
    """NaN and infinite K of nodes that a row does not see do not reach it; those that it sees do."""
    n = 20
    s = shape_for([n + 50], H=1, D=64, T=16)
    rng = np.random.default_rng(5)
    b = Batch(rng, s, [n], [n + 50])
    pool, _ = make_pool(rng, s)
    for j, x in ((4, float("nan")), (9, float("inf")), (11, float("-inf"))):
        pool[s.row(b.entry(s, 0, 50 + j), 0, 0, (50 + j) % 16)] = x
    sets = [{i} if i in (4, 9, 11) else {i} | {j for j in range(i) if j not in (4, 9, 11)} for i in range(n)]
    cache, batch = make_cache(s, pool, None), make_batch(b)
    for G in (1, 4, 8):
        q = torch.from_numpy(rng.normal(size=(n, G, 64))).bfloat16().cuda()
        out = torch.empty_like(q)
        aibx.attn_tree(cache, batch, dev(pack(sets, 1)), q, out)
        bad = torch.isnan(out).all(-1).all(-1).cpu().numpy()
        assert list(np.flatnonzero(bad)) == [4, 9, 11]
        clean = pool.clone()
        for j in (4, 9, 11):
            clean[s.row(b.entry(s, 0, 50 + j), 0, 0, (50 + j) % 16)] = 0.0
        want = torch.empty_like(q)
        aibx.attn_tree(make_cache(s, clean, None), batch, dev(pack(sets, 1)), q, want)
        rest = torch.from_numpy(~bad).cuda()
        assert torch.equal(out[rest], want[rest])


def test_stale_slots_do_not_matter():
    """What lies behind kv_len in the last block, and in blocks of others, is never read into a result."""
    def spoil(pool, scales):
        at = np.array([s.row(blk, kv, h, t) for blk in range(s.blocks) for kv in range(2) for h in range(s.H)
                       for t in range(s.T) if (blk, t) not in used])
        pool[at] = float("nan")
        return pool, scales

    for new in ([3, 2], [25, 11], [50, 20]):
        lens = [n + c for n, c in zip(new, (21, 130))]
        s = shape_for(lens, H=2, D=128, T=16)
        b = Batch(np.random.default_rng(6), s, new, lens)
        used = {(b.entry(s, r, j), j % s.T) for r in range(2) for j in range(lens[r])}
        st, _, _ = check_tree(s, b, G=4, change=spoil)
        assert st == (0, 0)


def test_scales_far_apart():
    """e4m3 rows whose scale bytes differ widely, in the cache and among the nodes."""
    def change(pool, scales):
        rng = np.random.default_rng(2)
        scales = scales.copy()
        far = rng.random(len(scales)) < 0.1
        scales[far] = rng.integers(100, 135, int(far.sum()))
        return pool, scales

    for new in ([3, 4], [30, 25], [60, 45]):
        lens = [n + c for n, c in zip(new, (300, 140))]
        s = shape_for(lens, H=2, D=128, T=16, pool="e4m3")
        b = Batch(np.random.default_rng(6), s, new, lens)
        st, _, _ = check_tree(s, b, G=4, change=change, scale=2.0 ** -12, words=1)
        assert st == (0, 0)


def test_more_nodes_than_bits():
    """RANGE for the request; the other's rows are right."""
    new = [70, 9]
    lens = [n + 40 for n in new]
    s = shape_for(lens, H=1, D=64, T=16)
    b = Batch(np.random.default_rng(7), s, new, lens)
    sets = [[{j for j in x if j < 64} for x in t] for t in trees(np.random.default_rng(0), b)]
    st, _, _ = check_tree(s, b, G=4, sets=sets)
    assert st[0] == aibx.ERR_RANGE


def test_negative_positions_and_empty_requests():
    """More nodes than cached and new tokens together (kv_len < n), requests without tokens."""
    new, lens = [6, 0, 20, 3], [4, 9, 12, 0]
    s = shape_for(lens, H=2, D=64, T=8)
    b = Batch(np.random.default_rng(8), s, new, lens)
    for G in (1, 4):
        st, _, _ = check_tree(s, b, G=G, seed=G, sets=[[set(range(i + 1)) for i in range(n)] for n in new])
        assert st == (0, 0)


def test_far_positions():
    """Cached tokens near the last position that can be told, all but a window of them without a block."""
    T, ctx, n = 256, 2 ** 31 - 2 - 9, 9
    s = Shape(H=1, D=64, T=T, blocks=4, layers=1, layer=0)
    rng = np.random.default_rng(10)
    pool, _ = make_pool(rng, s)
    cache = make_cache(s, pool, None)
    entries = -(-(ctx + n) // T)
    table = torch.full((1, entries), -1, dtype=torch.int32, device="cuda")
    table[0, -2:] = torch.tensor([2, 1], dtype=torch.int32, device="cuda")
    batch = aibx.KVBatch(table.view(torch.uint32), dev(np.array([0, n])), dev(np.array([ctx + n], dtype=np.int32)), n, max_new=n)
    sets = ancestors(random_tree(rng, n))
    for G in (1, 4, 16):
        q = torch.from_numpy(rng.normal(size=(n, G, 64))).bfloat16()
        out = torch.empty(n, G, 64, dtype=torch.bfloat16, device="cuda")
        aibx.attn_tree(cache, batch, dev(pack(sets, 1)), q.cuda(), out, window=200)
        small = Batch(rng, s, [n], [2 * T - 2])                # the same last two blocks, seen from near
        small.table = np.array([[2, 1]], dtype=np.uint32)
        assert (ctx + n) % T == T - 2
        want, _, mag, slack = tree_attention(s, small, pool_values(s, pool, None), q.double().numpy(), 64 ** -0.5, [sets], 200)
        assert (np.abs(out.double().cpu().numpy() - want) <= tree_tolerance(s, "bf16", want, mag, slack)).all()
    assert aibx.status_fetch() == (0, 0)


@pytest.mark.parametrize("pool,io", [("bf16", "bf16"), ("e4m3", "fp16")])
def test_same_bits_every_time_captured_and_beside_itself(pool, io):
    """Two calls, a replayed one, and calls on several streams with workspaces of their own."""
    rng = np.random.default_rng(11)
    new = [int(x) for x in rng.integers(1, 40, 12)]
    lens = [n + int(c) for n, c in zip(new, rng.integers(0, 900, 12))]
    s = shape_for(lens, H=4, D=128, T=16, pool=pool)
    b = Batch(rng, s, new, lens)
    p, sc = make_pool(rng, s)
    cache, batch = make_cache(s, p, sc), make_batch(b)
    q = torch.from_numpy(rng.normal(size=(b.n_tokens, 16, 128))).to(DTYPE[io]).cuda()
    mask = dev(np.concatenate([pack(t, 1) for t in trees(rng, b)]))
    size = aibx.attn_tree_workspace_bytes(cache, batch, q)
    streams = [torch.cuda.Stream() for _ in range(3)]
    outs = [torch.empty_like(q) for _ in range(5)]
    ws = [torch.full((size,), 255, dtype=torch.uint8, device="cuda") for _ in range(5)]
    aibx.attn_tree(cache, batch, mask, q, outs[0], workspace=ws[0])
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=streams[0]):
        aibx.attn_tree(cache, batch, mask, q, outs[1], workspace=ws[1])
    for _ in range(3):
        graph.replay()
    for k in range(3):
        streams[k].wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(streams[k]):
            for _ in range(3):
                aibx.attn_tree(cache, batch, mask, q, outs[2 + k], workspace=ws[2 + k])
    torch.cuda.synchronize()
    for o in outs[1:]:
        assert torch.equal(o, outs[0])
    assert aibx.status_fetch() == (0, 0)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("io", ["bf16", "fp16"])
@pytest.mark.parametrize("new", [[2, 5], [9, 16]])
def test_queries_of_wide_range(new, io, D):
    """Over e4m3 an element of a query may lose what is below 2^-17 of the query's largest: a score is off by at
    most that times the sum of a key's magnitudes, beside what slack counts.  A query with an infinity gives
    NaN, and leaves the others alone."""
    rng = np.random.default_rng(D + len(io))
    lens = [n + c for n, c in zip(new, (300, 77))]
    s = shape_for(lens, H=2, D=D, T=16, pool="e4m3")
    b = Batch(rng, s, new, lens)
    pool, scales = make_pool(rng, s)
    sets = trees(rng, b)
    q = torch.from_numpy(rng.normal(size=(b.n_tokens, 8, D)) * 2.0 ** -rng.uniform(0, 12, (b.n_tokens, 8, D))).to(DTYPE[io])
    q[1, 3, 5] = float("inf")
    out = torch.empty(q.shape, dtype=q.dtype, device="cuda")
    aibx.attn_tree(make_cache(s, pool, scales), make_batch(b, max(new)), dev(pack([x for one in sets for x in one], 1)), q.cuda(), out)
    got = out.double().cpu().numpy()
    assert np.isnan(got[1, 3]).all()
    q[1, 3, 5] = 0.0
    values, qd, scale = pool_values(s, pool, scales), q.double().numpy(), D ** -0.5
    want, _, mag, slack = tree_attention(s, b, values, qd, scale, sets, 0)
    slack = slack + scale * 2.0 ** -17 * np.abs(qd).max(-1) * np.abs(values).sum(-1).max()
    tol = tree_tolerance(s, io, want, mag, slack)
    fine = np.ones(got.shape[:2], dtype=bool)
    fine[1, 3] = False
    assert (np.abs(got - want) <= tol)[fine].all()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("new", [[1, 2], [2, 5], [9, 16], [40, 30]])
def test_queries_near_the_ends_of_their_type(new, D):
    """Queries of 2^124, and of 2^-112, whose scores are ordinary numbers."""
    lens = [n + c for n, c in zip(new, (300, 77))]
    s = shape_for(lens, H=2, D=D, T=16, pool="e4m3")
    for e in (122, -114):
        b = Batch(np.random.default_rng(6), s, new, lens)
        st, _, _ = check_tree(s, b, "bf16", G=4, seed=D, spread=2.0 ** e, scale=2.0 ** (min(-e, 112) - 4))
        assert st == (0, 0)
