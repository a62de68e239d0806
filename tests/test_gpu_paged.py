"""GPU tests of the token-wise calls on a paged pool: append, read and attention against a plain
64-bit reference, at the sizes, layouts and masks where they can go wrong."""
import itertools

import numpy as np
import pytest
import torch

from paged_ref import (DTYPE, HALF_STEP, NO_BLOCK, Batch, Shape, attention, pool_values, quantise,
                       tolerance)
from paper_2504_03648_b200 import binding as aibx

pytestmark = pytest.mark.gpu
KIND = {"bf16": aibx.TYPE_BF16, "fp16": aibx.TYPE_FP16, "e4m3": aibx.TYPE_E4M3}


@pytest.fixture(autouse=True)
def _clean_status():
    aibx.status_fetch()
    yield


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def kv_layout(s):
    return aibx.KVLayout(s.layout, s.layers, s.H, s.T, s.D, s.elem, s.blocks)


def make_pool(rng, s, spread=1.0):
    """(host pool, host scales or None) with random content."""
    if s.pool == "e4m3":
        x = torch.from_numpy(rng.normal(size=(s.rows, s.D)) * 100 * spread).clamp(-448, 448)
        return x.to(torch.float8_e4m3fn), rng.integers(118, 123, s.rows).astype(np.uint8)
    return torch.from_numpy(rng.normal(size=(s.rows, s.D)) * spread).to(DTYPE[s.pool]), None


def make_cache(s, pool, scales):
    return aibx.KVCache(pool.view(torch.uint8).cuda() if s.pool == "e4m3" else pool.cuda(), kv_layout(s),
                        KIND[s.pool], scales=None if scales is None else dev(scales), inner=s.inner,
                        layer=s.layer)


def make_batch(b, max_new=None):
    return aibx.KVBatch(dev(b.table), dev(b.tok_off), dev(b.kv_len), b.n_tokens,
                        max_new=max(b.new + [0]) if max_new is None else max_new,
                        blk_off=None if b.blk_off is None else dev(b.blk_off))


# ------------------------------------------------------------------------------------------
# append and read

SHAPES = [Shape(), Shape(H=1, D=128, T=8, layout=1, inner=1, pool="e4m3"),
          Shape(H=3, D=64, T=24, layout=2, pool="e4m3"), Shape(H=4, D=128, T=32, layout=1, pool="fp16"),
          Shape(H=8, D=16, T=16, inner=1, pool="e4m3"), Shape(H=2, D=8, T=1, blocks=300, pool="bf16"),
          Shape(H=5, D=40, T=7, layout=2, inner=1, pool="fp16"), Shape(H=2, D=264, T=8, pool="bf16"),
          Shape(H=2, D=1024, T=8, layout=2, pool="e4m3"), Shape(H=1, D=320, T=16, layout=1, pool="e4m3")]


def expected_append(s, b, pool, scales, k, v):
    pool, scales = pool.clone(), None if scales is None else scales.copy()
    rows = pool.view(torch.uint8).view(s.rows, -1) if s.pool == "e4m3" else pool
    for i, r, p in b.tokens():
        blk = b.entry(s, r, p)
        if blk is None:
            continue
        for kv, x in enumerate((k, v)):
            for h in range(s.H):
                at = s.row(blk, kv, h, p % s.T)
                if s.pool == "e4m3":
                    y, byte = quantise(x[i, h].double().numpy())
                    rows[at] = torch.from_numpy(y)
                    scales[at] = byte
                else:
                    rows[at] = x[i, h].double().to(DTYPE[s.pool]) if x.dtype != torch.float32 else \
                        x[i, h].to(DTYPE[s.pool])
    return pool, scales


@pytest.mark.parametrize("io", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_append_then_read(shape, io):
    s = SHAPES[shape]
    rng = np.random.default_rng(100 * shape + len(io))
    most = s.blocks * s.T // 8
    new = [1, 0, min(5, most), min(37, most), 2]
    b = Batch(rng, s, new, [n + c for n, c in zip(new, (0, 3, 2 * s.T, 1, s.T - 2))], ragged=shape % 2 == 1,
              pad=3)
    pool, scales = make_pool(rng, s)
    x = [torch.from_numpy(rng.normal(size=(b.n_tokens, s.H, s.D)) * 10.0 ** rng.uniform(-6, 4, (b.n_tokens, 1, 1)))
         .to(DTYPE[io]) for _ in range(2)]
    x[0][0, 0] = 0.0                                       # a row without a scale of its own
    x[1][-4, 0, :2] = torch.tensor([448.0, -1.0]).to(DTYPE[io])
    cache, batch = make_cache(s, pool, scales), make_batch(b)
    # K and V side by side in one tensor, as a projection leaves them
    both = torch.cat([x[0], x[1]], dim=1).cuda()
    aibx.kv_append(cache, batch, both[:, :s.H], both[:, s.H:])
    want, want_s = expected_append(s, b, pool, scales, *x)
    got = cache._keep[0].cpu().view(torch.uint8)
    assert torch.equal(got.view(-1), want.view(torch.uint8).view(-1))
    if scales is not None:
        assert np.array_equal(cache._keep[1].cpu().numpy(), want_s)
    assert aibx.status_fetch() == (0, 0)
    # and back, into every type
    values = pool_values(s, want, want_s)
    for to in ("bf16", "fp16", "fp32"):
        k = torch.full((b.n_tokens, s.H, s.D), 7.0, dtype=DTYPE[to], device="cuda")
        v = torch.full_like(k, 7.0)
        aibx.kv_read(cache, batch, k, v)
        ref = np.full((2, b.n_tokens, s.H, s.D), 7.0)
        for i, r, p in b.tokens():
            for kv, h in itertools.product(range(2), range(s.H if p >= 0 else 0)):   # others stay as they are
                ref[kv, i, h] = values[s.row(b.entry(s, r, p), kv, h, p % s.T)]
        ref = torch.from_numpy(ref).float().to(DTYPE[to])    # cached values are exact in fp32
        assert torch.equal(k.cpu(), ref[0]) and torch.equal(v.cpu(), ref[1])
    assert aibx.status_fetch() == (0, 0)


@pytest.mark.parametrize("io", ["bf16", "fp16", "fp32"])
def test_append_quantises_every_value(io):
    """Rows around every border of the e4m3 grid and of the scale rule, NaN and infinities."""
    s = Shape(H=1, D=128, T=8, blocks=70, pool="e4m3", layers=1, layer=0)
    rng = np.random.default_rng(5)
    rows = []
    for k in range(-20, 15):
        top = 448.0 * 2.0 ** k
        rows += [top, np.nextafter(np.float32(top), np.float32(0)), np.nextafter(np.float32(top), np.float32(1e30))]
    fine = np.unique(np.concatenate([np.abs(quantise_grid()), (quantise_grid()[1:] + quantise_grid()[:-1]) / 2]))
    n = 400
    x = np.zeros((n, 1, 128))
    for i in range(n):
        if i < len(rows):
            x[i, 0, 0] = rows[i]
            x[i, 0, 1:] = rng.normal(size=127) * rows[i] / 4
        else:
            x[i, 0] = rng.choice(fine, 128) * rng.choice([-1, 1], 128) * 2.0 ** int(rng.integers(-6, 6))
    x = torch.from_numpy(x).to(DTYPE[io])
    x[7, 0, 3], x[8, 0, 4], x[9, 0, 5] = float("nan"), float("inf"), float("-inf")
    x[10] = float("nan")
    x[11, 0, :] = -0.0
    if io == "fp32":
        x[12, 0, :] = 1e-42                                 # subnormal: the lowest scale
        x[13, 0, 0] = 3.4e38
    b = Batch(rng, s, [n], [n])
    pool, scales = make_pool(rng, s)
    cache, batch = make_cache(s, pool, scales), make_batch(b)
    aibx.kv_append(cache, batch, x.cuda(), x.cuda())
    want, want_s = expected_append(s, b, pool, scales, x, x)
    got = cache._keep[0].cpu().view(torch.uint8).view(s.rows, -1)
    want = want.view(torch.uint8).view(s.rows, -1)
    nan = (want & 127) == 127
    assert torch.equal(nan, (got & 127) == 127)             # a NaN's sign is free
    assert torch.equal(got[~nan], want[~nan])
    assert np.array_equal(cache._keep[1].cpu().numpy(), want_s)


def quantise_grid():
    from paged_ref import E4M3
    return E4M3[:127]


def test_append_and_read_skip_what_is_not_there():
    s = Shape(H=2, D=64, T=8, blocks=12)
    rng = np.random.default_rng(3)
    b = Batch(rng, s, [20, 6, 4], [20, 30, 2], width=3)       # second: last tokens behind the table
    b.table[0, 1] = NO_BLOCK
    b.table[0, 2] = s.blocks                                  # out of range
    pool, _ = make_pool(rng, s)
    cache, batch = make_cache(s, pool, None), make_batch(b)
    x = torch.from_numpy(rng.normal(size=(b.n_tokens, 2, 64))).bfloat16()
    aibx.kv_append(cache, batch, x.cuda(), x.cuda())
    want, _ = expected_append(s, b, pool, None, x, x)
    assert torch.equal(cache._keep[0].cpu(), want)
    assert aibx.status_fetch() == (aibx.ERR_RANGE, 4 + 6)     # four of block 2, six behind the table
    k = torch.full((b.n_tokens, 2, 64), 7.0, device="cuda")
    aibx.kv_read(cache, batch, k, k.clone())
    seen = torch.tensor([b.entry(s, r, p) is not None for _, r, p in b.tokens()])
    assert torch.equal(k.cpu()[~seen], torch.full_like(k.cpu()[~seen], 7.0))
    assert not (k.cpu()[seen] == 7.0).all()


@pytest.mark.parametrize("shift", [1, 3])
def test_append_and_read_unaligned(shift):
    s = Shape(H=3, D=64, T=16, pool="e4m3")
    rng = np.random.default_rng(shift)
    b = Batch(rng, s, [33], [40])
    pool, scales = make_pool(rng, s)
    cache, batch = make_cache(s, pool, scales), make_batch(b)
    flat = torch.from_numpy(rng.normal(size=33 * 211 + 8)).half().cuda()
    k = torch.as_strided(flat, (33, 3, 64), (211, 67, 1), shift)
    v = torch.as_strided(flat, (33, 3, 64), (193, 64, 1), 0)
    aibx.kv_append(cache, batch, k, v)
    want, want_s = expected_append(s, b, pool, scales, k.cpu(), v.cpu())
    assert torch.equal(cache._keep[0].cpu().view(-1), want.view(torch.uint8).view(-1))
    assert np.array_equal(cache._keep[1].cpu().numpy(), want_s)
    out = torch.zeros(33 * 211 + 8, device="cuda")
    ko = torch.as_strided(out, (33, 3, 64), (211, 67, 1), shift)
    vo = torch.zeros(33, 3, 64, device="cuda")
    aibx.kv_read(cache, batch, ko, vo)
    values = pool_values(s, want, want_s)
    for i, r, p in b.tokens():
        for h in range(3):
            assert np.array_equal(ko[i, h].cpu().numpy(), values[s.row(b.entry(s, r, p), 0, h, p % s.T)].astype(np.float32))
            assert np.array_equal(vo[i, h].cpu().numpy(), values[s.row(b.entry(s, r, p), 1, h, p % s.T)].astype(np.float32))
    rest = torch.ones_like(out, dtype=torch.bool)
    torch.as_strided(rest, (33, 3, 64), (211, 67, 1), shift).fill_(False)
    assert (out[rest] == 0).all()


# ------------------------------------------------------------------------------------------
# attention

def check_attention(s, b, io="bf16", G=4, causal=True, window=0, seed=0, spread=1.0, max_new=None, scale=None,
                    change=None, lse=True):
    rng = np.random.default_rng(seed)
    pool, scales = make_pool(rng, s)
    if change is not None:
        pool, scales = change(pool, scales)
    Hq = s.H * G
    q = torch.from_numpy(rng.normal(size=(b.n_tokens, Hq, s.D)) * spread).to(DTYPE[io])
    cache, batch = make_cache(s, pool, scales), make_batch(b, max_new)
    out = torch.full((b.n_tokens, Hq, s.D), 7.0, dtype=DTYPE[io], device="cuda")
    ls = torch.full((b.n_tokens, Hq), 7.0, device="cuda") if lse else None
    scale = s.D ** -0.5 if scale is None else scale
    aibx.attn_paged(cache, batch, q.cuda(), out, lse=ls, scale=scale, causal=causal, window=window)
    status = aibx.status_fetch()
    got = out.double().cpu().numpy()
    want, wl, mag, slack = attention(s, b, pool_values(s, pool, scales), q.double().numpy(), scale, causal, window)
    n = int(b.tok_off[-1])
    assert (got[n:] == 7.0).all()                             # rows behind the last request
    tol = tolerance(s, io, want[:n], mag[:n], slack[:n])
    err = np.abs(got[:n] - want[:n])
    assert np.isfinite(got[:n]).all()
    assert (err <= tol).all(), (float((err / tol).max()), np.argwhere(err > tol)[:5])
    if lse:
        gl = ls.double().cpu().numpy()
        assert (gl[n:] == 7.0).all()
        empty = np.isinf(wl[:n])
        assert (gl[:n][empty] == -np.inf).all()
        # sums of up to thousands of weights in fp32: 2^-24 per term of a chain of at most 2^10
        lt = slack[:n] + 2.0 ** -14 + 2.0 ** -22 * np.abs(np.where(empty, 0, wl[:n]))
        assert (np.abs(gl[:n] - wl[:n])[~empty] <= lt[~empty]).all()
    return status, out, ls


POOLS = [("bf16", "bf16"), ("fp16", "fp16"), ("e4m3", "bf16"), ("e4m3", "fp16")]


@pytest.mark.parametrize("pool,io", POOLS)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("layout,inner,T", [(0, 0, 16), (1, 1, 8), (2, 0, 24), (0, 1, 48), (1, 0, 256), (2, 1, 64)])
def test_attention_single_tokens(pool, io, D, layout, inner, T):
    lens = [1, T, T + 1, 5 * T - 1, 0, 130, 333]
    s = Shape(H=2, D=D, T=T, layout=layout, inner=inner, pool=pool, blocks=sum(-(-x // T) for x in lens) + 2)
    b = Batch(np.random.default_rng(T), s, [1] * len(lens), lens, pad=2)
    st, _, _ = check_attention(s, b, io, G=4, seed=D + T, spread=2.0)
    assert st == (0, 0)


@pytest.mark.parametrize("G,new", [(1, [1, 16, 3, 0, 9]), (7, [1, 2, 1, 2, 1]), (16, [1, 1, 0, 1, 1]), (5, [3, 1, 2, 0, 1]),
                                   (8, [2, 2, 1, 0, 2])])
@pytest.mark.parametrize("causal,window", [(True, 0), (True, 5), (False, 0), (False, 70), (True, 64), (True, 200)])
@pytest.mark.parametrize("pool,io", [("bf16", "bf16"), ("e4m3", "fp16")])
def test_attention_few_rows(G, new, causal, window, pool, io):
    lens = [n + c for n, c in zip(new, (0, 100, 259, 40, 700))]
    s = Shape(H=3, D=64 if G == 5 else 128, T=16, layout=1, pool=pool, blocks=90)
    b = Batch(np.random.default_rng(G), s, new, lens, ragged=G == 7)
    st, _, _ = check_attention(s, b, io, G=G, causal=causal, window=window, seed=window)
    assert st == (0, 0)


@pytest.mark.parametrize("pool,io", POOLS)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("layout,inner,T", [(0, 0, 16), (1, 1, 8), (2, 0, 24), (2, 1, 256)])
def test_attention_chunks(pool, io, D, layout, inner, T):
    new = [17, 0, 64, 130, 5, 33]
    lens = [n + c for n, c in zip(new, (0, 40, 300, 1, 128, 95))]
    s = Shape(H=2, D=D, T=T, layout=layout, inner=inner, pool=pool, blocks=sum(-(-x // T) for x in lens) + 2)
    b = Batch(np.random.default_rng(T), s, new, lens, pad=3, ragged=T == 24)
    st, _, _ = check_attention(s, b, io, G=4, seed=D + T, spread=2.0)
    assert st == (0, 0)


@pytest.mark.parametrize("G", [1, 3, 7, 40, 128])
@pytest.mark.parametrize("causal,window", [(True, 0), (True, 5), (False, 0), (False, 70), (True, 200)])
@pytest.mark.parametrize("pool,io", [("bf16", "bf16"), ("e4m3", "bf16")])
def test_attention_one_chunk(G, causal, window, pool, io):
    """One request: the tile kernel alone, whatever its length."""
    for n, c in ((1, 0), (2, 131), (40, 400), (300 if G < 4 else 9, 77)):
        s = Shape(H=1, D=128, T=16, layout=1, pool=pool, blocks=90)
        b = Batch(np.random.default_rng(G), s, [n], [n + c])
        st, _, _ = check_attention(s, b, io, G=G, causal=causal, window=window, seed=window, max_new=0)
        assert st == (0, 0)
