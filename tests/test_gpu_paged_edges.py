"""GPU tests of the paged token and attention calls where numbers, lengths and bounds are at their
edges: scales far apart, rows of zeros, scale bytes at the ends of their range, positions near 2^31,
more tokens than promised, many short segments."""
import numpy as np
import pytest
import torch

from paged_ref import DTYPE, HALF_STEP, Batch, Shape, attention, pool_values, tolerance
from paper_2504_03648_b200 import binding as aibx
from test_gpu_paged import POOLS, check_attention, dev, make_batch, make_cache, make_pool

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
def test_many_short_segments(pool, io):
    """Chunks of one to three tiles, several to a CTA: every warp of a CTA has to move from segment to
    segment with the others.  Right, and the same bits every time."""
    R = 700
    s = Shape(H=2, D=64, T=16, pool=pool, blocks=R * 12, layers=1, layer=0)
    rng = np.random.default_rng(21)
    new = [int(x) for x in rng.integers(20, 40, R)]
    b = Batch(rng, s, new, [n + int(c) for n, c in zip(new, rng.integers(0, 140, R))])
    p, sc = make_pool(rng, s)
    cache, batch = make_cache(s, p, sc), make_batch(b)
    q = torch.from_numpy(rng.normal(size=(b.n_tokens, 2, s.D))).to(DTYPE[io])
    want = run(cache, batch, q.cuda())
    for _ in range(20):
        assert same(run(cache, batch, q.cuda()), want)
    few = Batch.__new__(Batch)                                  # the plain form of some of them
    few.__dict__.update(b.__dict__)
    pick = list(range(0, R, 29))
    few.new, few.length = [b.new[r] for r in pick], [b.length[r] for r in pick]
    few.table = b.table[pick]
    few.tok_off = np.concatenate([[0], np.cumsum(few.new)]).astype(np.int64)
    few.n_tokens = int(few.tok_off[-1])
    rows = np.concatenate([np.arange(b.tok_off[r], b.tok_off[r + 1]) for r in pick])
    out, lse, mag, slack = attention(s, few, pool_values(s, p, sc), q[rows].double().numpy(), s.D ** -0.5, True, 0)
    assert (np.abs(want[0][rows].double().cpu().numpy() - out) <= tolerance(s, io, out, mag, slack)).all()
    assert aibx.status_fetch() == (0, 0)


# (tokens, bound, query heads per KV head): the row kernel alone, with rows to spare or not; both
# kernels; the tile kernel alone for one request
@pytest.mark.parametrize("new,bound,G", [([1, 3, 2, 1], 1, 2), ([1, 9, 1], 1, 8), ([200, 1, 30, 101], 100, 4),
                                         ([1, 2, 20], 1, 17), ([41], 40, 2), ([6, 5, 3], 4, 4), ([2], 1, 4)])
@pytest.mark.parametrize("pool,io", [("bf16", "bf16"), ("e4m3", "fp16")])
def test_every_request_past_the_bound_is_reported(new, bound, G, pool, io):
    s = Shape(H=1, D=64, T=16, pool=pool, blocks=60)
    rng = np.random.default_rng(22)
    b = Batch(rng, s, new, [n + 30 for n in new])
    p, sc = make_pool(rng, s)
    q = torch.from_numpy(rng.normal(size=(b.n_tokens, G, 64))).to(DTYPE[io]).cuda()
    run(make_cache(s, p, sc), make_batch(b, max_new=bound), q)
    assert aibx.status_fetch() == (aibx.ERR_RANGE, sum(n > bound for n in new))
    run(make_cache(s, p, sc), make_batch(b, max_new=max(new)), q)
    assert aibx.status_fetch() == (0, 0)


def of_v(s, x, per_row):
    """The V rows of a pool of layout 0 (a view: [blocks, layers, rows, per_row])."""
    return x.reshape(s.blocks, s.layers, 2, s.H * s.T, per_row)[:, :, 1]


@pytest.mark.parametrize("byte", [200, 253, 254])
@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("D", [64, 128])
def test_largest_v_scales(byte, new, D):
    """V rows of up to 2^(byte - 127), alone and beside the power below: weights, sums and lse."""
    s = Shape(H=2, D=D, T=16, pool="e4m3", blocks=60)
    b = Batch(np.random.default_rng(23), s, [new, new], [new + 5, new + 300])

    for lower in (0, 1):
        def change(pool, scales):
            v = of_v(s, pool, D)
            v[:] = (v.float() / 512).to(torch.float8_e4m3fn)        # magnitudes below 1: the values are finite
            of_v(s, scales, 1)[:] = byte
            of_v(s, scales, 1)[:, :, ::3] = byte - lower
            return pool, scales

        st, out, _ = check_attention(s, b, "bf16", G=4, change=change)
        assert st == (0, 0) and (out != 0).any(-1).all()
