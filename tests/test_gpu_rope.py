"""GPU tests of rotary positions, alone and on the way into the pool, against the 64-bit formula."""
import numpy as np
import pytest
import torch

from paged_ref import DTYPE, HALF_STEP, Batch, Shape, pool_values
from paper_2504_03648_b200 import binding as aibx
from steps_ref import LEAST, rotate, within
from test_gpu_paged import dev, make_batch, make_cache, make_pool

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _clean_status():
    aibx.status_fetch()
    yield


def frequencies(rd, base=10000.0):
    return base ** (-np.arange(rd // 2) / (rd // 2))


def rows(rng, n, heads, D, io, spread=1.0):
    return torch.from_numpy(rng.normal(size=(n, heads, D)) * spread).to(DTYPE[io])


@pytest.mark.parametrize("io", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("D,rd", [(64, 64), (128, 128), (128, 64), (128, 32), (96, 48), (80, 32), (72, 16), (256, 256), (512, 512), (16, 16), (40, 32)])
def test_rope(D, rd, interleaved, io):
    rng = np.random.default_rng(D + rd)
    n, heads = 37, 5
    x = rows(rng, n, heads, D, io)
    pos = np.concatenate([[0, 1, -1, 2 ** 31 - 1, -2 ** 31, 131072, 1000003], rng.integers(0, 200000, n - 7)]).astype(np.int32)
    f, factor = frequencies(rd), 1.25
    want, err = rotate(x.double().numpy(), pos, f, interleaved, factor)
    r = aibx.Rope(dev(f), interleaved=interleaved, factor=factor)
    y = torch.full_like(x, 7.0).cuda()
    aibx.rope(r, dev(pos), x.cuda(), y)
    got = y.double().cpu().numpy()
    assert np.array_equal(got[..., rd:], x.double().numpy()[..., rd:])
    assert within(got, want, err, io)
    inplace = x.cuda()
    aibx.rope(r, dev(pos), inplace, inplace)
    assert torch.equal(inplace, y)


@pytest.mark.parametrize("n,heads", [(1, 1), (1, 70), (3, 2), (700, 3), (5000, 1), (3001, 40)])
def test_rope_shapes_and_strides(n, heads):
    """Any number of tokens and heads; heads first, rows that are not aligned, rows between others' ones."""
    rng = np.random.default_rng(n)
    f = frequencies(64)
    r = aibx.Rope(dev(f), factor=1.0)
    pos = rng.integers(0, 9999, n).astype(np.int32)
    x = rows(rng, n, heads, 64, "bf16")
    want, err = rotate(x.double().numpy(), pos, f, False, 1.0)
    y = torch.empty_like(x).cuda()
    aibx.rope(r, dev(pos), x.cuda(), y)
    assert within(y.double().cpu().numpy(), want, err, "bf16")
    first = x.transpose(0, 1).contiguous().cuda().transpose(0, 1)
    other = torch.full((heads, n, 67), 7.0, dtype=torch.bfloat16, device="cuda")
    aibx.rope(r, dev(pos), first, other[..., 1:65].transpose(0, 1))
    assert torch.equal(other[..., 1:65].transpose(0, 1), y)
    assert (other[..., :1] == 7).all() and (other[..., 65:] == 7).all()


def test_rope_there_and_back():
    """Turned by p and then by -p a row is itself again, and the gradient of a rotation is the turn back."""
    rng = np.random.default_rng(2)
    n, heads, D = 50, 3, 128
    f = frequencies(D, 500000.0)
    r = aibx.Rope(dev(f))
    pos = dev(rng.integers(0, 100000, n).astype(np.int32))
    x = torch.from_numpy(rng.normal(size=(n, heads, D))).float().cuda()
    y, z = torch.empty_like(x), torch.empty_like(x)
    aibx.rope(r, pos, x, y)
    aibx.rope(r, -pos, y, z)
    size = (x[..., :64].abs() + x[..., 64:].abs()).repeat(1, 1, 2)
    assert ((z - x).abs() <= size * 2.0 ** -24 * 24).all()     # two rotations, each within 8, of terms up to sqrt 2 larger
    g = torch.from_numpy(rng.normal(size=(n, heads, D))).cuda()
    p = pos.double()
    xd = x.double().requires_grad_()
    a = p[:, None] * torch.from_numpy(f).cuda()
    c, s = a.cos()[:, None], a.sin()[:, None]
    out = torch.cat([xd[..., :64] * c - xd[..., 64:] * s, xd[..., 64:] * c + xd[..., :64] * s], -1)
    out.backward(g)
    back = torch.empty_like(x)
    gf = g.float()
    aibx.rope(r, -pos, gf, back)
    size = (gf[..., :64].abs() + gf[..., 64:].abs()).repeat(1, 1, 2)
    turns = (a.abs() / 6.28)[:, None].repeat(1, 1, 2)
    assert ((back.double() - xd.grad).abs() <= size * (9 * 2.0 ** -24 + 6.3 * turns * 2.0 ** -51)).all()
    # differences: the rotation is linear, so a step of any size gives the slope along it
    h = torch.from_numpy(rng.normal(size=(n, heads, D))).float().cuda()
    up, down = torch.empty_like(x), torch.empty_like(x)
    aibx.rope(r, pos, x + h, up)
    aibx.rope(r, pos, x - h, down)
    slope = ((up.double() - down.double()) / 2 * g).sum(-1)
    want = (h.double() * xd.grad).sum(-1)
    bound = ((x.abs() + h.abs()).double().amax(-1) * g.abs().sum(-1)) * 2.0 ** -24 * 40
    assert ((slope - want).abs() <= bound).all()


def test_rope_keeps_nan_and_infinity_to_their_pairs():
    f = frequencies(64)
    r = aibx.Rope(dev(f))
    x = torch.ones(4, 2, 64)
    x[1, 0, 3], x[2, 1, 40], x[3, 0, 63] = float("nan"), float("inf"), float("-inf")
    y = torch.empty_like(x).cuda()
    aibx.rope(r, dev(np.array([5, 6, 7, 8], dtype=np.int32)), x.cuda(), y)
    bad = ~torch.isfinite(y.cpu())
    want = torch.zeros_like(bad)
    want[1, 0, [3, 35]] = want[2, 1, [8, 40]] = want[3, 0, [31, 63]] = True
    assert torch.equal(bad, want)


# ------------------------------------------------------------------------------------------
# into the pool

SHAPES = [(Shape(), 64), (Shape(H=1, D=128, T=8, layout=1, inner=1, pool="e4m3"), 128),
          (Shape(H=3, D=64, T=24, layout=2, pool="e4m3"), 32), (Shape(H=4, D=128, T=32, layout=1, pool="fp16"), 64),
          (Shape(H=8, D=16, T=16, inner=1, pool="e4m3"), 16), (Shape(H=5, D=40, T=7, layout=2, inner=1, pool="fp16"), 32),
          (Shape(H=2, D=264, T=8, pool="bf16"), 128), (Shape(H=2, D=512, T=8, layout=2, pool="e4m3"), 512),
          (Shape(H=1, D=320, T=16, layout=1, pool="e4m3"), 320)]


def check_pool(s, b, got, got_s, before, before_s, k, kerr, v, io):
    """Rows of the batch's tokens hold k (off by kerr) and v, rounded once; all others are as before."""
    touched = np.zeros(s.rows, dtype=bool)
    values = pool_values(s, got, got_s)
    for i, r, p in b.tokens():
        blk = b.entry(s, r, p)
        if blk is None:
            continue
        for h in range(s.H):
            for kv, (x, e) in enumerate(((k[i, h], kerr[i, h]), (v[i, h], np.zeros(s.D)))):
                at = s.row(blk, kv, h, p % s.T)
                touched[at] = True
                if s.pool != "e4m3":
                    assert within(values[at], x, e, s.pool)
                    continue
                # the scale: the least power for a largest magnitude within its error
                a, ae = np.abs(x).max(), e[np.abs(x).argmax()]
                byte = int(got_s[at])
                if a > 0:
                    assert a - ae <= 448 * 2.0 ** (byte - 127) and (byte == 1 or a + ae > 448 * 2.0 ** (byte - 128))
                else:
                    assert byte == 127
                unit = 2.0 ** (byte - 127)
                assert (np.abs(values[at] - x) <= e + np.maximum(HALF_STEP["e4m3"] * (np.abs(x) + e), 2.0 ** -10 * unit)).all()
    same = ~touched
    raw, old = got.view(torch.uint8).view(s.rows, -1).numpy(), before.view(torch.uint8).view(s.rows, -1).numpy()
    assert np.array_equal(raw[same], old[same])
    if before_s is not None:
        assert np.array_equal(got_s[same], before_s[same])


@pytest.mark.parametrize("io", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_rope_append(shape, interleaved, io):
    s, rd = SHAPES[shape]
    rng = np.random.default_rng(100 * shape + len(io))
    most = s.blocks * s.T // 8
    new = [1, 0, min(5, most), min(37, most), 2]
    b = Batch(rng, s, new, [n + c for n, c in zip(new, (0, 3, 2 * s.T, 1, s.T - 2))], ragged=shape % 2 == 1, pad=3)
    Hq = 3 * s.H
    pool, scales = make_pool(rng, s)
    qkv = (torch.from_numpy(rng.normal(size=(b.n_tokens, Hq + 2 * s.H, s.D)) * 10.0 ** rng.uniform(-3, 3, (b.n_tokens, 1, 1)))).to(DTYPE[io])
    qkv[0, Hq] = 0.0
    f, factor = frequencies(rd, 1e6), 0.9
    cache, batch = make_cache(s, pool, scales), make_batch(b)
    d = qkv.cuda()
    q_out = torch.full((b.n_tokens, Hq, s.D), 7.0, dtype=d.dtype, device="cuda")
    r = aibx.Rope(dev(f), interleaved=interleaved, factor=factor)
    aibx.rope_append(cache, batch, r, d[:, Hq:Hq + s.H], d[:, Hq + s.H:], q=d[:, :Hq], q_out=q_out)
    at = np.zeros(b.n_tokens, dtype=np.int64)
    for i, _, p in b.tokens():
        at[i] = p
    x = qkv.double().numpy()
    turned, err = rotate(x, at, f, interleaved, factor)
    n = int(b.tok_off[-1])
    got = q_out.double().cpu().numpy()
    assert within(got[:n], turned[:n, :Hq], err[:n, :Hq], io) and (got[n:] == 7.0).all()
    p1, s1 = cache._keep[0].cpu(), None if scales is None else cache._keep[1].cpu().numpy()
    check_pool(s, b, p1 if scales is None else p1.view(torch.float8_e4m3fn), s1, pool, scales, turned[:, Hq:Hq + s.H],
               err[:, Hq:Hq + s.H], x[:, Hq + s.H:], io)
    # V's bytes are kv_append's, and so are those of a K that is not turned
    plain = make_cache(s, pool, scales)
    aibx.kv_append(plain, batch, d[:, Hq:Hq + s.H], d[:, Hq + s.H:])
    still = make_cache(s, pool, scales)
    aibx.rope_append(still, batch, aibx.Rope(dev(f), interleaved=interleaved), d[:, Hq:Hq + s.H], d[:, Hq + s.H:],
                     pos=torch.zeros(b.n_tokens, dtype=torch.int32, device="cuda"))
    assert torch.equal(still._keep[0], plain._keep[0])
    if scales is not None:
        assert torch.equal(still._keep[1], plain._keep[1])
    assert aibx.status_fetch() == (0, 0)


def test_rope_append_at_given_positions_in_place_and_unaligned():
    s = Shape(H=2, D=64, T=16, pool="bf16")
    rng = np.random.default_rng(8)
    b = Batch(rng, s, [9, 20], [30, 20], pad=1)
    pool, _ = make_pool(rng, s)
    cache, batch = make_cache(s, pool, None), make_batch(b)
    n, Hq = b.n_tokens, 4
    flat = torch.from_numpy(rng.normal(size=n * 600 + 3)).half().cuda()
    q = torch.as_strided(flat, (n, Hq, 64), (600, 65, 1), 3)
    k = torch.as_strided(flat, (n, 2, 64), (600, 70, 1), 301)
    v = torch.as_strided(flat, (n, 2, 64), (600, 64, 1), 460)
    pos = rng.integers(0, 5000, n).astype(np.int32)
    f = frequencies(64)
    x = flat.clone().cpu()
    old = [t.double().cpu().numpy().copy() for t in (q, k, v)]
    aibx.rope_append(cache, batch, aibx.Rope(dev(f)), k, v, q=q, q_out=q, pos=dev(pos))
    tq, eq = rotate(old[0], pos, f, False, 1.0)
    tk, ek = rotate(old[1], pos, f, False, 1.0)
    assert within(q.double().cpu().numpy()[:29], tq[:29], eq[:29], "fp16")
    check_pool(s, b, cache._keep[0].cpu(), None, pool, None, tk, ek, old[2], "fp16")
    rest = torch.ones(flat.numel(), dtype=torch.bool)
    torch.as_strided(rest, (29, Hq, 64), (600, 65, 1), 3).fill_(False)
    assert torch.equal(flat.cpu()[rest], x[rest])


def test_rope_append_skips_what_is_not_there():
    from paged_ref import NO_BLOCK
    s = Shape(H=2, D=64, T=8, blocks=12)
    rng = np.random.default_rng(3)
    b = Batch(rng, s, [20, 6, 4], [20, 30, 2], width=3)       # second: behind the table; third: negative positions
    b.table[0, 1] = NO_BLOCK
    b.table[0, 2] = s.blocks
    pool, _ = make_pool(rng, s)
    cache, batch = make_cache(s, pool, None), make_batch(b)
    x = torch.from_numpy(rng.normal(size=(b.n_tokens, 2, 64))).bfloat16()
    q = torch.empty(b.n_tokens, 2, 64, dtype=torch.bfloat16, device="cuda")
    f = frequencies(64)
    aibx.rope_append(cache, batch, aibx.Rope(dev(f)), x.cuda(), x.cuda(), q=x.cuda(), q_out=q)
    at = np.array([p for _, _, p in b.tokens()])
    turned, err = rotate(x.double().numpy(), at, f, False, 1.0)
    assert within(q.double().cpu().numpy(), turned, err, "bf16")   # queries have no slot to be missing
    check_pool(s, b, cache._keep[0].cpu(), None, pool, None, turned, err, x.double().numpy(), "bf16")
    assert aibx.status_fetch() == (aibx.ERR_RANGE, 4 + 6)


def test_rope_append_of_nan_and_infinity():
    """e4m3 rows take their scale from the finite elements; a pair with a NaN or infinity is NaN."""
    s = Shape(H=1, D=64, T=8, blocks=4, layers=1, layer=0, pool="e4m3")
    rng = np.random.default_rng(4)
    b = Batch(rng, s, [3], [3])
    pool, scales = make_pool(rng, s)
    cache, batch = make_cache(s, pool, scales), make_batch(b)
    x = torch.ones(3, 1, 64)
    x[0, 0, 3], x[1, 0, 40] = float("nan"), float("inf")
    aibx.rope_append(cache, batch, aibx.Rope(dev(frequencies(64))), x.cuda(), x.cuda(),
                     pos=torch.tensor([1, 2, 3], dtype=torch.int32, device="cuda"))
    got = pool_values(s, cache._keep[0].cpu().view(torch.float8_e4m3fn), cache._keep[1].cpu().numpy())
    for i, bad in enumerate(([3, 35], [8, 40], [])):
        k = got[s.row(b.entry(s, 0, i), 0, 0, i)]
        assert sorted(np.flatnonzero(np.isnan(k))) == bad
        assert np.abs(k[~np.isnan(k)]).max() <= np.sqrt(2) * (1 + 2.0 ** -4)


def test_rope_append_far_blocks():
    """Offsets past 2^32 bytes."""
    free = torch.cuda.mem_get_info()[0]
    s = Shape(H=8, D=128, T=64, layers=4, layer=3, blocks=10000, layout=1, pool="bf16")
    size = s.rows * s.D * 2
    assert size > 2 ** 32
    if free < size + 2 ** 30:
        pytest.skip("too little device memory")
    pool = torch.zeros(size // 2, dtype=torch.bfloat16, device="cuda")
    cache = aibx.KVCache(pool, aibx.KVLayout(1, 4, 8, 64, 128, 2, s.blocks), aibx.TYPE_BF16, layer=3)
    table = torch.tensor([[s.blocks - 1, 0]], dtype=torch.int32, device="cuda").view(torch.uint32)
    batch = aibx.KVBatch(table, dev(np.array([0, 2], dtype=np.int64)), dev(np.array([65], dtype=np.int32)), 2)
    x = torch.randn(2, 8, 128, device="cuda").bfloat16()
    f = frequencies(128)
    aibx.rope_append(cache, batch, aibx.Rope(dev(f)), x, x)
    want, err = rotate(x.double().cpu().numpy(), np.array([63, 64]), f, False, 1.0)
    rows_ = pool.view(s.rows, 128)
    for i, (blk, slot) in enumerate(((s.blocks - 1, 63), (0, 0))):
        at = [s.row(blk, 0, h, slot) for h in range(8)]
        assert within(rows_[at].double().cpu().numpy(), want[i], err[i], "bf16")
        at = [s.row(blk, 1, h, slot) for h in range(8)]
        assert torch.equal(rows_[at], x[i])
    assert int((pool != 0).sum()) <= 2 * 2 * 8 * 128
