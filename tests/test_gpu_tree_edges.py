"""GPU tests of attention of drafted trees where one row's numbers could reach another's, and where queries,
weights and scores are at the edge of the types that hold them."""
import numpy as np
import pytest
import torch

from paged_ref import DTYPE, Batch, pool_values, tolerance
from paper_2504_03648_b200 import binding as aibx
from steps_ref import ancestors, pack, random_tree, tree_attention, tree_tolerance
from test_gpu_paged import dev, make_batch, make_cache, make_pool
from test_gpu_tree import shape_for

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _clean_status():
    aibx.status_fetch()
    yield


def dense(s, b, values, q, scale, sets):
    """steps_ref.tree_attention without a window, a request and KV head at a time."""
    n, Hq, D = q.shape
    G = Hq // s.H
    out, lse = np.full((n, Hq, D), np.nan), np.full((n, Hq), np.nan)
    mag, slack = np.zeros_like(out), np.zeros_like(lse)
    for r, k in enumerate(b.new):
        at, base = slice(int(b.tok_off[r]), int(b.tok_off[r + 1])), b.length[r] - k
        seen = np.zeros((k, b.length[r]), dtype=bool)
        seen[:, :base] = True
        for i, nodes in enumerate(sets[r]):
            seen[i, [base + j for j in nodes]] = True
        for h in range(s.H):
            rows = [s.row(b.entry(s, r, j), 0, h, j % s.T) for j in range(b.length[r])]
            K, V = values[rows], values[[s.row(b.entry(s, r, j), 1, h, j % s.T) for j in range(b.length[r])]]
            for g in range(h * G, h * G + G):
                z = np.where(seen, scale * (q[at, g] @ K.T), -np.inf)
                m = z.max(-1, keepdims=True)
                w = np.exp(z - m)
                t = w.sum(-1, keepdims=True)
                lse[at, g] = (m + np.log(t))[:, 0]
                out[at, g], mag[at, g] = (w / t) @ V, (w / t) @ np.abs(V)
                most = np.where(seen, np.abs(K).max(-1), 0).max(-1)
                slack[at, g] = scale * (D + 4) * 2.0 ** -24 * most * np.abs(q[at, g]).sum(-1) + 4 * 2.0 ** -24 * np.abs(m[:, 0])
    return out, lse, mag, slack


def call(s, b, pool, scales, q, sets, scale, words=1):
    out = torch.empty(q.shape, dtype=q.dtype, device="cuda")
    lse = torch.empty(q.shape[:2], device="cuda")
    mask = dev(np.concatenate([pack(x, words) for x in sets]))
    aibx.attn_tree(make_cache(s, pool, scales), make_batch(b), mask, q.cuda(), out, lse=lse, scale=scale)
    assert aibx.status_fetch() == (0, 0)
    return out.double().cpu().numpy(), lse.double().cpu().numpy()


# rows of one KV head: 24, 48, 120
@pytest.mark.parametrize("n,G", [(3, 8), (12, 4), (30, 4)])
@pytest.mark.parametrize("pool", ["fp16", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
def test_an_infinite_query_beside_scores_that_grow(D, pool, n, G):
    """Every 128 keys hold one whose score is 8 above all before it, for every row, and is infinite for one: the
    others' running maximum has to follow all the same, or their weights (e^8 from one to the next) leave fp16."""
    rng = np.random.default_rng(n + D)
    ctx = 40 * 128 + 5                            # (8 heads of 41 tiles: several to a CTA)
    s = shape_for([n + ctx], H=8, D=D, T=16, pool=pool)
    b = Batch(rng, s, [n], [n + ctx])
    kv, _ = make_pool(rng, s)
    scale = D ** -0.5
    line = np.where(rng.random(D) < 0.5, -1.0, 1.0)
    line[5] = 1.0
    for h in range(s.H):
        for t in range(41):
            j = 128 * t + (64 + 7 * h) % 128 if t < 40 else 128 * t
            kv[s.row(b.entry(s, 0, j), 0, h, j % s.T)] = torch.from_numpy(line * 8 * t / (scale * D)).to(DTYPE[pool])
    sets = [ancestors(random_tree(rng, n))]
    q = torch.from_numpy(line + 0.1 * rng.normal(size=(n, s.H * G, D))).to(DTYPE[pool])
    fine = np.ones((n, s.H * G), dtype=bool)
    fine[1, 1::G] = False                         # a row of every KV head
    q[1, 1::G, 5] = float("inf")
    got, gl = call(s, b, kv, None, q, sets, scale)
    assert np.isnan(got[~fine]).all()
    q[1, 1::G, 5] = 0.0
    want, wl, mag, slack = dense(s, b, pool_values(s, kv, None), q.double().numpy(), scale, sets)
    assert np.isfinite(got[fine]).all()
    assert (np.abs(got - want) <= tree_tolerance(s, pool, want, mag, slack))[fine].all()
    assert (np.abs(gl - wl) <= slack + 2.0 ** -14 + 2.0 ** -22 * np.abs(wl))[fine].all()


@pytest.mark.parametrize("window", [1, 5, 30])
@pytest.mark.parametrize("G", [1, 4, 8])
def test_a_chain_longer_than_the_window(G, window):
    """With the bits of ancestors `window` and more nodes up cleared it is attn_paged with that window, to the
    roundings of two orders of sums."""
    new = [20, 4, 33]
    lens = [n + c for n, c in zip(new, (200, 0, 131))]
    s = shape_for(lens, H=2, D=128, T=16)
    rng = np.random.default_rng(G + window)
    b = Batch(rng, s, new, lens)
    pool, _ = make_pool(rng, s)
    sets = [[set(range(max(0, i - window + 1), i + 1)) for i in range(n)] for n in new]
    q = torch.from_numpy(rng.normal(size=(b.n_tokens, 2 * G, 128))).bfloat16().cuda()
    cache, batch = make_cache(s, pool, None), make_batch(b)
    x, y = torch.empty_like(q), torch.empty_like(q)
    aibx.attn_paged(cache, batch, q, x, window=window)
    aibx.attn_tree(cache, batch, dev(np.concatenate([pack(t, 1) for t in sets])), q, y, window=window)
    _, _, mag, slack = tree_attention(s, b, pool_values(s, pool, None), q.double().cpu().numpy(), 128 ** -0.5, sets, window)
    x, y = x.double().cpu().numpy(), y.double().cpu().numpy()
    assert (np.abs(x - y) <= 2 * tree_tolerance(s, "bf16", x, mag, slack)).all()


# ------------------------------------------------------------------------------------------
# over e4m3


@pytest.mark.parametrize("new,G", [([3, 2], 2), ([12, 5], 2), ([20, 9], 3), ([40, 33], 4)])
@pytest.mark.parametrize("io", ["bf16", "fp16"])
@pytest.mark.parametrize("D", [64, 128])
def test_queries_with_an_element_far_above_the_others(D, io, new, G):
    """One element 2^15 times the others, where all keys are zero.  Elements of a query may lose what is below
    2^-24 of its largest: a score is off by at most that times the sum of a key's magnitudes."""
    rng = np.random.default_rng(D + len(new))
    lens = [n + c for n, c in zip(new, (300, 77))]
    s = shape_for(lens, H=2, D=D, T=16, pool="e4m3")
    b = Batch(rng, s, new, lens)
    pool, scales = make_pool(rng, s)
    pool.view(torch.uint8).view(s.rows, D)[:, 5] = 0
    sets = [ancestors(random_tree(rng, n)) for n in new]
    q = torch.from_numpy(rng.normal(size=(b.n_tokens, 2 * G, D)))
    q[..., 5] = 2.0 ** 15
    q = q.to(DTYPE[io])
    scale = 3 * D ** -0.5
    got, gl = call(s, b, pool, scales, q, sets, scale)
    values, qd = pool_values(s, pool, scales), q.double().numpy()
    far = scale * 2.0 ** -24 * 2.0 ** 15 * np.abs(values).sum(-1).max()
    qd[..., 5] = 0.0                              # (that product is zero: no part of any sum)
    want, wl, mag, slack = dense(s, b, values, qd, scale, sets)
    slack = slack + far
    assert (np.abs(got - want) <= tree_tolerance(s, io, want, mag, slack)).all()
    assert (np.abs(gl - wl) <= slack + 2.0 ** -14 + 2.0 ** -22 * np.abs(wl)).all()


@pytest.mark.parametrize("new,G", [([3, 2], 2), ([12, 5], 2), ([20, 9], 3), ([40, 33], 4)])
@pytest.mark.parametrize("e", [-118, -121, -124, -126])
@pytest.mark.parametrize("D", [64, 128])
def test_the_smallest_queries(D, e, new, G):
    """bf16 queries about 2^e, subnormal ones among them, and a scale that makes ordinary scores of them: they lose
    nothing that larger ones keep."""
    rng = np.random.default_rng(D - e)
    lens = [n + c for n, c in zip(new, (300, 77))]
    s = shape_for(lens, H=2, D=D, T=16, pool="e4m3")
    b = Batch(rng, s, new, lens)
    pool, scales = make_pool(rng, s)
    sets = [ancestors(random_tree(rng, n)) for n in new]
    q = torch.from_numpy((rng.normal(size=(b.n_tokens, 2 * G, D)) * 2.0 ** e).astype(np.float32)).bfloat16()
    assert int((q != 0).sum()) > 0.9 * q.numel()
    scale = 2.0 ** (-e - 1)
    got, gl = call(s, b, pool, scales, q, sets, scale)
    want, wl, mag, slack = dense(s, b, pool_values(s, pool, scales), q.double().numpy(), scale, sets)
    assert (np.abs(got - want) <= tree_tolerance(s, "bf16", want, mag, slack)).all()
    assert (np.abs(gl - wl) <= slack + 2.0 ** -14 + 2.0 ** -22 * np.abs(wl)).all()


@pytest.mark.parametrize("n,G", [(8, 1), (16, 1), (24, 2), (50, 1), (64, 2)])
@pytest.mark.parametrize("io", ["bf16", "fp16"])
@pytest.mark.parametrize("D", [64, 128])
def test_weights_whose_values_cancel(D, io, n, G):
    """Every node sees two, whose V are 1 and -1 and whose weights are nearly the same: what is left of their
    difference shows how many bits the weights have.  11, as attn_paged's over the same pool."""
    rng = np.random.default_rng(n + D)
    new = [n] * 6
    s = shape_for(new, H=2, D=D, T=16, pool="e4m3")
    b = Batch(rng, s, new, new)
    pool, scales = make_pool(rng, s)
    at = np.array([[s.row(b.entry(s, r, j), 1, h, j % s.T) for j in range(n)] for r in range(6) for h in range(2)])
    rows = pool.view(torch.uint8).view(s.rows, D)
    rows[at[:, ::2].reshape(-1)] = 0x38           # 1
    rows[at[:, 1::2].reshape(-1)] = 0xB8          # -1
    scales[at] = 127
    sets = [[{2 * int(rng.integers(0, n // 2)), 2 * int(rng.integers(0, n // 2)) + 1} for _ in range(n)] for _ in range(6)]
    q = torch.from_numpy(rng.normal(size=(b.n_tokens, 2 * G, D))).to(DTYPE[io])
    scale = 0.2 * D ** -0.5
    got, _ = call(s, b, pool, scales, q, sets, scale)
    want, _, mag, slack = dense(s, b, pool_values(s, pool, scales), q.double().numpy(), scale, sets)
    assert (np.abs(got - want) <= tolerance(s, io, want, mag, slack)).all()
