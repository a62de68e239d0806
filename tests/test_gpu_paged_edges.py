"""GPU tests of the paged token and attention calls where numbers, lengths and bounds are at their
edges: scales far apart, rows of zeros, scale bytes at the ends of their range, positions near 2^31,
more tokens than promised, many short segments."""
import numpy as np
import pytest
import torch

from paged_ref import DTYPE, HALF_STEP, Batch, Shape, attention, pool_values, tolerance
from paper_2504_03648_b200 import binding as aibx
from test_gpu_paged import POOLS, check_attention, dev, expected_append, make_batch, make_cache, make_pool

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


# ------------------------------------------------------------------------------------------
# e4m3 rows whose scales are far apart

def definition(values, rows_k, rows_v, q, scale, first):
    """Causal attention of one (request, KV head) in 64 bits, and what the roundings may add to the
    output: q [n][G][D] at positions first .., rows of K and of V for positions 0 .."""
    k, v = values[rows_k], values[rows_v]
    z = scale * np.einsum("ngd,kd->ngk", q, k)
    z[:, :, :][np.broadcast_to(np.arange(len(k))[None, None] > first + np.arange(len(q))[:, None, None], z.shape)] = -np.inf
    m = z.max(-1, keepdims=True)
    w = np.exp(z - m)
    t = w.sum(-1, keepdims=True)
    w /= t
    out, lse = w @ v, (m + np.log(t))[..., 0]
    mag = w @ np.abs(v)
    # A score: fp32 products and sums of D terms; queries are fp16, within 2^-25 of their row's largest.
    slack = scale * (q.shape[-1] + 4) * 2.0 ** -24 * np.abs(q).sum(-1) * np.abs(k).max() + 2.0 ** -22 * np.abs(m[..., 0])
    # A weight: fp16 (2^-11), or below 2^-14 on a grid of 2^-24, in units 2^7 below the largest 2^(t + b)
    # and of keys whose b is at most 4 below the largest: 2^-25 * 2^-7 * 2^4 of the largest weight each.
    grid = 2.0 ** -28 * w.max(-1, keepdims=True) * np.abs(v).sum(0)
    return out, lse, (2.0 ** -11 + 2 * slack[..., None] + 2.0 ** -20) * mag + grid, slack


def check_scales(s, b, pool, scales, q, io, G):
    """Every request of b against the definition; q: [n_tokens][H * G][D] on the host."""
    cache, batch = make_cache(s, pool, scales), make_batch(b)
    out, lse = run(cache, batch, q.cuda())
    values = pool_values(s, pool, scales)
    out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    for r, n in enumerate(b.new):
        L, o = b.length[r], int(b.tok_off[r])
        for h in range(s.H):
            rows = [np.array([s.row(b.entry(s, r, p), kv, h, p % s.T) for p in range(L)]) for kv in range(2)]
            heads = slice(h * G, h * G + G)
            want, wl, tol, slack = definition(values, *rows, q[o:o + n, heads].double().numpy(), s.D ** -0.5, L - n)
            # the result is rounded once; 2^-25 below fp16's normal numbers, 2^-134 below bf16's
            tol = tol + HALF_STEP[io] * np.abs(want) + (2.0 ** -25 if io == "fp16" else 2.0 ** -133)
            err = np.abs(out[o:o + n, heads] - want)
            assert (err <= tol).all(), (r, h, float((err / tol).max()), float(err.max() / np.abs(want).max()))
            assert (np.abs(lse[o:o + n, heads] - wl) <= slack + 2.0 ** -14 + 2.0 ** -22 * np.abs(wl)).all()
    assert aibx.status_fetch() == (0, 0)


def null_key_pool(rng, s, b, q, lead, size, where, G):
    """A pool written by append: V of magnitude `size`, and at position where(length) a key that leads the
    others' scores by about `lead`, with a V of zeros."""
    cache = make_cache(s, torch.zeros(s.rows, s.D).to(torch.float8_e4m3fn), np.full(s.rows, 127, dtype=np.uint8))
    total = sum(b.length)
    whole = Batch.__new__(Batch)
    whole.__dict__.update(b.__dict__)
    whole.new = b.length
    whole.tok_off = np.concatenate([[0], np.cumsum(b.length)]).astype(np.int64)
    whole.n_tokens = total
    k = rng.normal(size=(total, s.H, s.D)) * 0.3
    v = rng.normal(size=(total, s.H, s.D)) * size
    u = np.ones(s.D)
    for r, L in enumerate(b.length):
        i = int(whole.tok_off[r]) + where(L)
        k[i] = u * (lead / (s.D ** -0.5 * s.D))
        v[i] = 0.0
    k, v = (torch.from_numpy(x).float().cuda() for x in (k, v))
    aibx.kv_append(cache, make_batch(whole), k, v)
    return cache._keep[0].cpu().view(torch.float8_e4m3fn).view(s.rows, s.D), cache._keep[1].cpu().numpy()


def near_ones(rng, n, heads, D, io):
    """Queries whose product with a row of ones is about D."""
    return torch.from_numpy(1.0 + 0.1 * rng.normal(size=(n, heads, D))).to(DTYPE[io])


WHERE = {"first": lambda L: 0, "middle": lambda L: L // 2, "late": lambda L: max(0, L - 45)}


@pytest.mark.parametrize("size", [3.0, 1.0, 0.1, 0.01, 0.001, 1e-5])
@pytest.mark.parametrize("lead", [3.0, 6.0, 8.0, 14.0])
@pytest.mark.parametrize("where", list(WHERE))
def test_a_leading_row_of_zeros_few_rows(size, lead, where):
    for D, io, new, G in ((128, "bf16", 1, 8), (64, "fp16", 1, 4), (128, "fp16", 3, 5)):
        s = Shape(H=2, D=D, T=16, pool="e4m3", blocks=340, layers=1, layer=0)
        rng = np.random.default_rng(24)
        b = Batch(rng, s, [new, new], [1000, 4003])
        q = near_ones(rng, b.n_tokens, 2 * G, D, io)
        pool, scales = null_key_pool(rng, s, b, q, lead, size, WHERE[where], G)
        assert (scales == 127).any()
        check_scales(s, b, pool, scales, q, io, G)


def spread_pool(rng, s, kind):
    """Pools as others may write them: bytes far apart, one byte for all, bytes larger than the rows need."""
    pool = torch.from_numpy(rng.normal(size=(s.rows, s.D)) * 100).clamp(-448, 448).to(torch.float8_e4m3fn)
    scales = rng.integers(118, 123, s.rows).astype(np.uint8)
    v = of_v(s, scales, 1)
    if kind == "spread of 40":
        v[:] = rng.integers(90, 131, v.shape)
    elif kind == "whole range":
        v[:] = rng.integers(0, 240, v.shape)
    elif kind == "lowest":
        v[:] = rng.integers(0, 30, v.shape)
    elif kind == "one byte":                                # elements around e4m3's least
        v[:] = 127
        x = of_v(s, pool, s.D)
        x[:] = (x.float() / 8192).to(torch.float8_e4m3fn)
    elif kind == "loose":                                    # one row in 50: 2^17 larger a scale than it needs
        x = of_v(s, pool, s.D)
        loose = torch.from_numpy(rng.random(tuple(x.shape[:3])) < 0.02)
        x[loose] = (x[loose].float().sign() * 2.0 ** -9).to(torch.float8_e4m3fn)
        v[:] = np.where(loose.numpy()[..., None], 127, 104)
    return pool, scales


KINDS = ["spread of 40", "whole range", "lowest", "one byte", "loose"]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("D,io,new,G", [(128, "bf16", 1, 8), (64, "fp16", 1, 4), (128, "fp16", 3, 5), (64, "bf16", 2, 8)])
def test_scales_far_apart_few_rows(kind, D, io, new, G):
    s = Shape(H=2, D=D, T=16, pool="e4m3", blocks=120, layers=1, layer=0)
    rng = np.random.default_rng(25)
    b = Batch(rng, s, [new] * 3, [200, 37, 1500])
    pool, scales = spread_pool(rng, s, kind)
    q = torch.from_numpy(rng.normal(size=(b.n_tokens, 2 * G, D)) * 2).to(DTYPE[io])
    if kind == "whole range" and io == "fp16":
        of_v(s, scales, 1)[:] = rng.integers(0, 130, of_v(s, scales, 1).shape)     # results that fp16 can hold
    check_scales(s, b, pool, scales, q, io, G)


@pytest.mark.parametrize("new", [1, 3, 40])
@pytest.mark.parametrize("kv", [0, 1])
def test_nan_scale_of_a_visible_row(new, kv):
    """Scale byte 255: NaN for the heads that see the row; of V it leaves lse alone."""
    s = Shape(H=2, D=64, T=16, pool="e4m3", blocks=40)
    rng = np.random.default_rng(26)
    b = Batch(rng, s, [new], [new + 200])
    pool, scales = make_pool(rng, s)
    scales[s.row(b.entry(s, 0, 77), kv, 0, 77 % 16)] = 255
    q = torch.from_numpy(rng.normal(size=(new, 4, 64))).bfloat16().cuda()
    out, lse = run(make_cache(s, pool, scales), make_batch(b), q)
    assert torch.isnan(out[:, :2]).all() and torch.isfinite(out[:, 2:]).all()
    assert torch.isnan(lse[:, :2]).all() == (kv == 0) and torch.isfinite(lse[:, 2:]).all()
    if kv == 1:
        assert torch.isfinite(lse).all()


@pytest.mark.parametrize("size", [3.0, 1.0, 0.1, 0.01, 0.001, 1e-5])
@pytest.mark.parametrize("lead", [3.0, 6.0, 8.0, 14.0])
@pytest.mark.parametrize("where", list(WHERE))
def test_a_leading_row_of_zeros_chunks(size, lead, where):
    for D, io, new, G in ((128, "bf16", 40, 3), (64, "fp16", 150, 1), (128, "fp16", 9, 40)):
        s = Shape(H=2, D=D, T=16, pool="e4m3", blocks=340, layers=1, layer=0)
        rng = np.random.default_rng(27)
        b = Batch(rng, s, [new, new], [1000, 4003])
        q = near_ones(rng, b.n_tokens, 2 * G, D, io)
        pool, scales = null_key_pool(rng, s, b, q, lead, size, WHERE[where], G)
        check_scales(s, b, pool, scales, q, io, G)


@pytest.mark.parametrize("size", [1.0, 0.1, 0.001])
@pytest.mark.parametrize("new", [1, 30])
def test_a_leading_row_of_zeros_in_a_long_context(size, new):
    """One key of V = 0 that leads 130,000 others by a factor of 10^5, in the first tile of the line."""
    s = Shape(H=1, D=64, T=64, pool="e4m3", blocks=2050, layers=1, layer=0)
    rng = np.random.default_rng(28)
    b = Batch(rng, s, [new], [130001])
    q = near_ones(rng, new, 2, 64, "fp16")
    pool, scales = null_key_pool(rng, s, b, q, 11.5, size, WHERE["first"], 2)
    check_scales(s, b, pool, scales, q, "fp16", 2)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("D,io,new,G", [(128, "bf16", 40, 3), (64, "fp16", 150, 1), (128, "fp16", 5, 100), (64, "bf16", 300, 1)])
def test_scales_far_apart_chunks(kind, D, io, new, G):
    s = Shape(H=2, D=D, T=16, pool="e4m3", blocks=160, layers=1, layer=0)
    rng = np.random.default_rng(29)
    b = Batch(rng, s, [new] * 3, [new + 160, new, 1500])
    pool, scales = spread_pool(rng, s, kind)
    q = torch.from_numpy(rng.normal(size=(b.n_tokens, 2 * G, D)) * 2).to(DTYPE[io])
    if kind == "whole range" and io == "fp16":
        of_v(s, scales, 1)[:] = rng.integers(0, 130, of_v(s, scales, 1).shape)     # results that fp16 can hold
    check_scales(s, b, pool, scales, q, io, G)


def of_k(s, x, per_row):
    return x.reshape(s.blocks, s.layers, 2, s.H * s.T, per_row)[:, :, 0]


def key_tolerance(values, rows_k, rows_v, q, scale, first):
    """As definition(), with the error of every score on its own: products and sums of that key's D
    terms, and queries within 2^-25 of their row's largest element."""
    k, v = values[rows_k], values[rows_v]
    z = scale * np.einsum("ngd,kd->ngk", q, k)
    z[np.broadcast_to(np.arange(len(k))[None, None] > first + np.arange(len(q))[:, None, None], z.shape)] = -np.inf
    m = z.max(-1, keepdims=True)
    w = np.exp(z - m)
    w /= w.sum(-1, keepdims=True)
    err = scale * ((q.shape[-1] + 4) * 2.0 ** -24 * np.einsum("ngd,kd->ngk", np.abs(q), np.abs(k))
                   + 2.0 ** -25 * np.abs(q).max(-1, keepdims=True) * np.where(q == 0, 0, 1).max(-1, keepdims=True)
                   * np.einsum("ngd,kd->ngk", np.where(q == 0, 0.0, 1.0), np.abs(k))) + 2.0 ** -22 * np.abs(m)
    mag = w @ np.abs(v)
    out = w @ v
    # e^err - 1 <= 2 err for what moves a weight, once in it and once, on average, in the sum
    moved = (w * err) @ np.abs(v) + (w * err).sum(-1, keepdims=True) * np.abs(out)
    return 2 * moved + (2.0 ** -11 + 2.0 ** -20) * mag + 2.0 ** -28 * w.max(-1, keepdims=True) * np.abs(v).sum(0)


@pytest.mark.parametrize("kind", ["a zero row with a large byte", "large rows beside the query", "rows 2^30 below"])
@pytest.mark.parametrize("D,io,new,G", [(128, "bf16", 40, 3), (64, "fp16", 150, 1), (128, "fp16", 1, 8), (64, "bf16", 300, 1)])
def test_key_scales_far_apart(kind, D, io, new, G):
    """K rows whose scales say nothing about their scores must not take bits from the others."""
    s = Shape(H=2, D=D, T=16, pool="e4m3", blocks=160, layers=1, layer=0)
    rng = np.random.default_rng(31)
    b = Batch(rng, s, [new] * 2, [new + 160, 1500])
    pool, scales = make_pool(rng, s)
    q = torch.from_numpy(rng.normal(size=(b.n_tokens, 2 * G, D)) * 2).to(DTYPE[io])
    q[..., D // 2:] = 0
    k, kb = of_k(s, pool, D), of_k(s, scales, 1)
    odd = rng.random(kb.shape[:3]) < 0.05
    if kind == "a zero row with a large byte":
        k.view(torch.uint8)[torch.from_numpy(odd)] = 0
        kb[odd] = 200
    elif kind == "large rows beside the query":
        x = k[torch.from_numpy(odd)].float()
        x[:, :D // 2] = 0                                       # scores of 0
        k[torch.from_numpy(odd)] = x.to(torch.float8_e4m3fn)
        kb[odd] = 150
    else:                                                       # scores of about 0, in the place of 0
        kb[odd] = 90
    cache, batch = make_cache(s, pool, scales), make_batch(b)
    out, lse = run(cache, batch, q.cuda())
    values = pool_values(s, pool, scales)
    out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    for r, n in enumerate(b.new):
        L, o = b.length[r], int(b.tok_off[r])
        for h in range(2):
            rows = [np.array([s.row(b.entry(s, r, p), kv, h, p % s.T) for p in range(L)]) for kv in range(2)]
            heads = slice(h * G, h * G + G)
            qq = q[o:o + n, heads].double().numpy()
            want, wl, _, _ = definition(values, *rows, qq, s.D ** -0.5, L - n)
            tol = key_tolerance(values, *rows, qq, s.D ** -0.5, L - n) + HALF_STEP[io] * np.abs(want)
            err = np.abs(out[o:o + n, heads] - want)
            assert (err <= tol).all(), (r, h, float((err / tol).max()), float(err.max() / np.abs(want).max()))
            assert (np.abs(lse[o:o + n, heads] - wl) <= 2.0 ** -12).all()
    assert aibx.status_fetch() == (0, 0)


# ------------------------------------------------------------------------------------------
# positions at the end of their range

@pytest.mark.parametrize("pool,io", POOLS)
@pytest.mark.parametrize("new", [1, 70])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("back", [0, 1, 40])
def test_positions_up_to_the_last_of_31_bits(pool, io, new, D, back):
    """A sequence of 2^31 - 1 tokens (or a few less) seen through a window: written, read back, attended
    to, with a missing block among the last ones."""
    T, L, n, window, G = 8, 2 ** 31 - 1 - back, 1000, 600, 4
    s = Shape(H=1, D=D, T=T, pool=pool, blocks=140, layers=1, layer=0)
    rng = np.random.default_rng(32)
    p, sc = make_pool(rng, s)
    cache = make_cache(s, p, sc)
    entries = -(-L // T)
    used = 130                                                  # blocks of the last positions
    table = torch.full((1, entries), -1, dtype=torch.int32, device="cuda")
    ids = rng.permutation(s.blocks)[:used].astype(np.int32)
    table[0, entries - used:] = dev(ids)
    k, v = (torch.from_numpy(rng.normal(size=(n, 1, D))).to(DTYPE[io]).cuda() for _ in range(2))

    def batch(m):
        return aibx.KVBatch(table.view(torch.uint32), dev(np.array([0, m], dtype=np.int64)),
                            dev(np.array([L], dtype=np.int32)), m, max_new=m)

    aibx.kv_append(cache, batch(n), k, v)
    back_k, back_v = torch.empty_like(k, dtype=torch.float32), torch.empty_like(v, dtype=torch.float32)
    aibx.kv_read(cache, batch(n), back_k, back_v)
    if pool != "e4m3":
        assert torch.equal(back_k, k.float()) and torch.equal(back_v, v.float())
    hole = entries - 1 if back == 40 else entries - 2           # not the only block of the last row
    table[0, hole] = -1
    q = torch.from_numpy(rng.normal(size=(new, G, D)) * 2).to(DTYPE[io])
    out, lse = run(cache, batch(new), q.cuda(), window=window)
    assert aibx.status_fetch() == (0, 0)
    pos = np.arange(L - n, L)
    kk, vv = (x.double().cpu().numpy()[:, 0] for x in (back_k, back_v))
    row = np.arange(L - new, L)[:, None, None]
    seen = (pos <= row) & (pos > row - window) & (pos // T != hole)
    z = np.where(seen, D ** -0.5 * np.einsum("ngd,kd->ngk", q.double().numpy(), kk), -np.inf)
    m = z.max(-1, keepdims=True)
    w = np.exp(z - m)
    t = w.sum(-1, keepdims=True)
    w /= t
    want, wl, mag = w @ vv, (m + np.log(t))[..., 0], w @ np.abs(vv)
    slack = D ** -0.5 * (D + 4) * 2.0 ** -24 * np.abs(kk).max() * np.abs(q.double().numpy()).sum(-1) + 2.0 ** -22 * np.abs(m[..., 0])
    # weights rounded to the operands' type (fp16 below 2^-14 of the largest: 2^-25 of it), scores, the result
    tol = (HALF_STEP["fp16" if pool == "e4m3" else io] + 2 * slack[..., None] + 2.0 ** -20) * mag \
        + 2.0 ** -25 * w.max(-1, keepdims=True) * np.abs(vv).sum(0) + HALF_STEP[io] * np.abs(want)
    assert (np.abs(out.double().cpu().numpy() - want) <= tol).all()
    assert (np.abs(lse.double().cpu().numpy() - wl) <= slack + 2.0 ** -14 + 2.0 ** -22 * np.abs(wl)).all()


def test_every_position_of_31_bits_is_counted():
    """No window: 2^31 - 1 positions that all hold one of two rows."""
    T, L = 65536, 2 ** 31 - 1
    s = Shape(H=1, D=64, T=T, pool="bf16", blocks=2, layers=1, layer=0)
    pool = torch.zeros(s.rows, 64, dtype=torch.bfloat16)
    for kv in range(2):
        for blk in range(2):
            at = s.row(blk, kv, 0, 0)
            pool[at:at + T] = float(blk) if kv else 0.0         # equal scores, V = 0 or 1
    cache = make_cache(s, pool, None)
    table = torch.zeros(1, L // T + 1, dtype=torch.int32, device="cuda")
    table[0, 3::4] = 1                                          # a quarter of the positions
    for new in (1, 20):
        batch = aibx.KVBatch(table.view(torch.uint32), dev(np.array([0, new], dtype=np.int64)),
                             dev(np.array([L], dtype=np.int32)), new, max_new=new)
        q = torch.ones(new, 2, 64, dtype=torch.bfloat16, device="cuda")
        out, lse = run(cache, batch, q)
        # a sum of 2^31 ones: fp32 sums of 2^7 per step and thread, a few thousand steps, 148 pieces
        assert ((out.float() - 0.25).abs() <= 2.0 ** -8).all()
        assert ((lse - 31 * np.log(2.0)).abs() <= 2.0 ** -8).all()
    assert aibx.status_fetch() == (0, 0)


@pytest.mark.parametrize("every", [1, 20])
@pytest.mark.parametrize("D,io,new,G", [(128, "bf16", 40, 3), (64, "fp16", 150, 1), (128, "fp16", 1, 8)])
def test_zero_keys_at_the_largest_scale(every, D, io, new, G):
    """K rows of zeros with byte 254 have scores of 0, whatever the queries are."""
    s = Shape(H=2, D=D, T=16, pool="e4m3", blocks=40, layers=1, layer=0)
    rng = np.random.default_rng(33)
    b = Batch(rng, s, [new], [new + 300])
    pool, scales = make_pool(rng, s)
    k, kb = of_k(s, pool, D).view(torch.uint8), of_k(s, scales, 1)
    k[:, :, ::every] = 0
    kb[:, :, ::every] = 254
    q = torch.from_numpy(rng.normal(size=(b.n_tokens, 2 * G, D)) * (50 if every == 1 else 2)).to(DTYPE[io])
    cache, batch = make_cache(s, pool, scales), make_batch(b)
    out, lse = run(cache, batch, q.cuda())
    values = pool_values(s, pool, scales)
    for h in range(2):
        rows = [np.array([s.row(b.entry(s, 0, p), kv, h, p % s.T) for p in range(new + 300)]) for kv in range(2)]
        heads = slice(h * G, h * G + G)
        qq = q[:, heads].double().numpy()
        want, wl, _, _ = definition(values, *rows, qq, D ** -0.5, 300)
        tol = key_tolerance(values, *rows, qq, D ** -0.5, 300) + HALF_STEP[io] * np.abs(want)
        assert (np.abs(out[:, heads].double().cpu().numpy() - want) <= tol).all()
        assert (np.abs(lse[:, heads].double().cpu().numpy() - wl) <= 2.0 ** -12).all()
    assert aibx.status_fetch() == (0, 0)


# ------------------------------------------------------------------------------------------
# batches of many requests, few of them with tokens

@pytest.mark.parametrize("pool,io", [("bf16", "bf16"), ("e4m3", "fp16")])
@pytest.mark.parametrize("every,pad", [(64, 0), (64, 40), (33, 3), (31, 1), (1000, 0)])
def test_few_of_many_requests_have_tokens(pool, io, every, pad):
    s = Shape(H=1, D=64, T=8, pool=pool, blocks=140, layers=1, layer=0)
    rng = np.random.default_rng(34)
    new = [0] * 4097
    for i, r in enumerate(range(every // 2, 4097, every)):
        new[r] = 1 + (i % 3 == 0)
    b = Batch(rng, s, new, [n + 5 if n else 0 for n in new], pad=pad)
    p, sc = make_pool(rng, s)
    cache, batch = make_cache(s, p, sc), make_batch(b)
    k, v = (torch.from_numpy(rng.normal(size=(b.n_tokens, 1, 64))).to(DTYPE[io]) for _ in range(2))
    aibx.kv_append(cache, batch, k.cuda(), v.cuda())
    want, want_s = expected_append(s, b, p, sc, k, v)
    assert torch.equal(cache._keep[0].cpu().view(torch.uint8).view(-1), want.view(torch.uint8).view(-1))
    if sc is not None:
        assert np.array_equal(cache._keep[1].cpu().numpy(), want_s)
    back = [torch.full((b.n_tokens, 1, 64), 7.0, device="cuda") for _ in range(2)]
    aibx.kv_read(cache, batch, *back)
    values = pool_values(s, want, want_s)
    ref = np.full((2, b.n_tokens, 1, 64), 7.0)
    for i, r, pos in b.tokens():
        for kv in range(2):
            ref[kv, i, 0] = values[s.row(b.entry(s, r, pos), kv, 0, pos % 8)]
    assert all(torch.equal(x.cpu(), torch.from_numpy(y).float()) for x, y in zip(back, ref))
    q = torch.from_numpy(rng.normal(size=(b.n_tokens, 2, 64))).to(DTYPE[io])
    out, _ = run(cache, batch, q.cuda())
    n = int(b.tok_off[-1])
    full, _, mag, slack = attention(s, b, values, q.double().numpy(), 64 ** -0.5, True, 0)
    assert (np.abs(out.double().cpu().numpy() - full)[:n] <= tolerance(s, io, full[:n], mag[:n], slack[:n])).all()
    assert aibx.status_fetch() == (0, 0)


@pytest.mark.parametrize("D", [64, 128])
def test_scales_far_apart_captured_and_side_by_side(D):
    """Pools of every kind at once, on several streams, eager and from graphs: the same bits."""
    jobs = []
    for i, (kind, new, lens) in enumerate([("spread of 40", 1, [900, 40, 300]), ("loose", 90, [700, 350]), ("one byte", 3, [500, 800]),
                                           ("whole range", 260, [300, 1200]), (None, 120, [1000])]):
        s = Shape(H=2, D=D, T=16, pool="e4m3", blocks=160, layers=1, layer=0)
        rng = np.random.default_rng(40 + i)
        pool, scales = spread_pool(rng, s, kind) if kind else make_pool(rng, s)
        b = Batch(rng, s, [new] * len(lens), lens)
        cache, batch = make_cache(s, pool, scales), make_batch(b)
        q = torch.from_numpy(rng.normal(size=(b.n_tokens, 8, D))).bfloat16().cuda()
        ws = torch.empty(aibx.attn_workspace_bytes(cache, batch, q), dtype=torch.uint8, device="cuda")
        out = torch.empty_like(q)
        want = run(cache, batch, q)[0]
        g, st = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        with torch.cuda.graph(g):
            aibx.attn_paged(cache, batch, q, out, workspace=ws)
        jobs.append((cache, batch, q, want, st, g, out, ws))    # (a graph's workspace lives as long as it does)
    torch.cuda.synchronize()
    for turn in range(6):
        got = []
        for cache, batch, q, _, st, g, _, _ in jobs:
            with torch.cuda.stream(st):
                got.append(run(cache, batch, q)[0])
                g.replay()
        torch.cuda.synchronize()
        for x, (_, _, _, want, _, _, out, _) in zip(got, jobs):
            assert torch.equal(x.view(torch.int16), want.view(torch.int16)), turn
            assert torch.equal(out.view(torch.int16), want.view(torch.int16)), turn
    assert aibx.status_fetch() == (0, 0)
