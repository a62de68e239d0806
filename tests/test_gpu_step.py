"""GPU tests of the calls around a step together, as an engine makes them: prompts matched against the
index, tables grown, keys rotated into the pool, attention; then a drafted tree, eager and captured."""
import numpy as np
import pytest
import torch

from paged_ref import Batch, Shape, attention, pool_values, tolerance
from paper_2504_03648_b200 import binding as aibx
from steps_ref import ancestors, random_tree, rotate, tree_attention, tree_tolerance
from test_gpu_paged import dev, make_cache, make_pool

pytestmark = pytest.mark.gpu
T = 16


@pytest.fixture(autouse=True)
def _clean_status():
    aibx.status_fetch()
    yield


class Engine:
    """Requests of one layer: tables, a free list and rotated keys, all on the device."""

    def __init__(self, R, pool="bf16", H=2, G=4, D=64, width=24, seed=0):
        self.rng = np.random.default_rng(seed)
        self.R, self.H, self.G, self.D, self.width = R, H, G, D, width
        self.s = Shape(H=H, D=D, T=T, blocks=R * width + 5, layout=1, pool=pool)
        host, scales = make_pool(self.rng, self.s)
        self.cache = make_cache(self.s, host, scales)
        self.free = dev(self.rng.permutation(self.s.blocks).astype(np.uint32))
        self.head, self.tail = dev(np.zeros(1, dtype=np.int64)), dev(np.array([self.s.blocks], dtype=np.int64))
        self.table = torch.full((R, width), -1, dtype=torch.int32, device="cuda").view(torch.uint32)
        self.kv_len = torch.zeros(R, dtype=torch.int32, device="cuda")
        self.tok_off = torch.zeros(R + 1, dtype=torch.int64, device="cuda")
        f, self.factor = aibx.rope_frequencies(D, 10000.0, scaling="parts", scale=4.0, trained=256)
        self.f = f.numpy()
        self.rope = aibx.Rope(f.cuda(), factor=self.factor)

    def qkv(self, n):
        return torch.from_numpy(self.rng.normal(size=(n, (self.G + 2) * self.H, self.D))).bfloat16()

    def split(self, qkv):
        a, b = self.G * self.H, (self.G + 1) * self.H
        return qkv[:, :a], qkv[:, a:b], qkv[:, b:]

    def grow(self, held, new, n, pos=None, slots=None, **match):
        aibx.kv_tables(held, new, T, self.s.blocks, self.free, self.head, self.tail, self.table, self.tok_off,
                       self.kv_len, n, pos=pos, slots=slots, **match)

    def batch(self, n, max_new):
        return aibx.KVBatch(self.table, self.tok_off, self.kv_len, n, max_new=max_new)

    def values(self):
        p, sc = self.cache._keep
        return pool_values(self.s, p.cpu().view(torch.float8_e4m3fn) if sc is not None else p.cpu(),
                           None if sc is None else sc.cpu().numpy())

    def reference(self, new):
        """The requests as the reference sees them."""
        b = Batch.__new__(Batch)
        b.new, b.length, b.blk_off = list(new), self.kv_len.tolist(), None
        b.table = self.table.cpu().numpy()
        b.tok_off = np.concatenate([[0], np.cumsum(new)]).astype(np.int64)
        b.n_tokens, b.kv_len = int(b.tok_off[-1]), self.kv_len.cpu().numpy()
        return b


def near(got, want, tol):
    assert (np.abs(got.double().cpu().numpy() - want) <= tol).all()


def step(e, new, held=None, **match):
    """One step of new tokens in order; returns queries, their rotation and the attention's output."""
    n = sum(new)
    held = e.kv_len if held is None else held
    pos = torch.empty(n, dtype=torch.int32, device="cuda")
    slots = torch.empty(n, dtype=torch.int64, device="cuda")
    e.grow(held, dev(np.array(new, dtype=np.int32)), n, pos=pos, slots=slots, **match)
    x = e.qkv(n)
    q, k, v = e.split(x.cuda())
    turned = torch.empty(q.shape, dtype=q.dtype, device="cuda")
    batch = e.batch(n, max(new))
    aibx.rope_append(e.cache, batch, e.rope, k, v, q=q, q_out=turned)
    out = torch.empty(q.shape, dtype=q.dtype, device="cuda")
    aibx.attn_paged(e.cache, batch, turned, out)
    b = e.reference(new)
    at = np.array([p for _, _, p in b.tokens()])
    assert pos.tolist() == at.tolist()
    assert slots.tolist() == [b.entry(e.s, r, p) * T + p % T for _, r, p in b.tokens()]
    # the cached keys are the tokens' own, rotated for their positions
    values = e.values()
    want, err = rotate(e.split(x)[1].double().numpy(), at, e.f, False, e.factor)
    for i, r, p in b.tokens():
        for h in range(e.H):
            row = values[e.s.row(b.entry(e.s, r, p), 0, h, p % T)]
            step_ = 2.0 ** -4 if e.s.pool == "e4m3" else 2.0 ** -8
            least = np.abs(want[i, h]).max() * 2.0 ** -17 if e.s.pool == "e4m3" else 0.0   # 2^-10 of a scale above max / 448
            assert (np.abs(row - want[i, h]) <= err[i, h] + step_ * (np.abs(want[i, h]) + err[i, h]) + least).all()
    o, _, mag, slack = attention(e.s, b, values, turned.double().cpu().numpy(), e.D ** -0.5, True, 0)
    near(out, o, tolerance(e.s, "bf16", o, mag, slack))


@pytest.mark.parametrize("pool", ["bf16", "e4m3"])
def test_prompts_matched_then_steps(pool):
    """Prompts fill blocks and are published; prompts that share their beginnings are matched, take over those
    blocks in their tables, compute the rest, and go on token by token."""
    e = Engine(6, pool)
    rng = np.random.default_rng(5)
    shared = rng.integers(0, 1000, 100).astype(np.int32)
    prompts = [np.concatenate([shared[:k], rng.integers(0, 1000, m)]).astype(np.int32) for k, m in
               ((100, 9), (64, 30), (0, 40), (100, 1), (96, 0), (33, 50))]
    index = aibx.Index(1024, 1)

    def keys(seqs):
        off = np.concatenate([[0], np.cumsum([len(x) for x in seqs])]).astype(np.int64)
        blk = np.concatenate([[0], np.cumsum([len(x) // T for x in seqs])]).astype(np.int64)
        h = torch.empty(int(blk[-1]), dtype=torch.uint64, device="cuda")
        aibx.hash_blocks(dev(np.concatenate(seqs)), dev(off), dev(blk), T, 0, h)
        return h, dev(blk)

    # the first prompt of all, alone: nothing matches
    first = [len(prompts[0])] + [0] * 5
    step(e, first)
    h, blk = keys(prompts[:1])
    full = len(prompts[0]) // T
    index.insert(h, torch.ones(full, dtype=torch.int64, device="cuda").view(torch.uint64), e.table.view(torch.int32)[0, :full].contiguous().view(torch.uint32))
    # then the others, against what it left
    h, blk = keys(prompts)
    match_len = torch.empty(6, dtype=torch.uint32, device="cuda")
    any_len = torch.empty(6, dtype=torch.uint32, device="cuda")
    ids = torch.empty(h.numel(), dtype=torch.uint32, device="cuda")
    index.match_prefix(h, blk, match_len, any_len, ids)
    assert any_len.tolist() == [6, 4, 0, 6, 6, 2]
    lens = np.array([len(p) for p in prompts])
    held = np.minimum(np.array(any_len.tolist()) * T, lens - 1)   # one token at least is computed
    new = lens - held
    new[0], held[0] = 0, lens[0]                             # (the first runs on)
    # its own row lies in blocks past the matched ones: they come as matched ids, too
    own = e.table[0].clone()
    all_ids = [own[:-(-int(lens[0]) // T)]] + [ids[int(blk[r]):int(blk[r + 1])] for r in range(1, 6)]
    off = np.concatenate([[0], np.cumsum([len(x) for x in all_ids])]).astype(np.int64)
    step(e, new.tolist(), held=dev(held.astype(np.int32)), match_ids=torch.cat(all_ids), match_off=dev(off))
    rows = e.table.view(torch.int32).tolist()
    assert rows[3][:6] == rows[0][:6] and rows[1][:4] == rows[0][:4] and rows[1][4] != rows[0][4]
    for _ in range(3):
        step(e, [1] * 6)
    step(e, [1, 0, 3, 1, 0, 20])
    assert int(e.head) == sum(-(-int(x) // T) for x in e.kv_len.tolist()) - (4 + 6 + 6 + 2)
    assert aibx.status_fetch() == (0, 0)


@pytest.mark.parametrize("pool,nodes", [("bf16", [2, 1, 0, 2]), ("bf16", [26, 3, 0, 40]), ("e4m3", [10, 16, 1, 7]), ("e4m3", [30, 50, 0, 64])])
def test_drafts(pool, nodes):
    """Tables, masks, rotation by depth and attention of a drafted tree in one captured graph, replayed with
    other drafts of the same number of nodes in the same buffers."""
    e = Engine(4, pool, width=40)
    step(e, [200, 33, 7, 120])
    n, R = sum(nodes), 4
    before = e.kv_len.clone()
    head0 = e.head.clone()
    d = dict(parent=torch.empty(n, dtype=torch.int32, device="cuda"), x=torch.empty(n, (e.G + 2) * e.H, e.D, dtype=torch.bfloat16, device="cuda"),
             new=dev(np.array(nodes, dtype=np.int32)), mask=torch.empty(n, 1, dtype=torch.int64, device="cuda").view(torch.uint64),
             pos=torch.empty(n, dtype=torch.int32, device="cuda"))
    q, k, v = e.split(d["x"])
    turned, out = torch.empty_like(q.contiguous()), torch.empty_like(q.contiguous())
    lse = torch.empty(n, e.G * e.H, device="cuda")
    head = torch.empty_like(e.head)
    kv = torch.empty_like(e.kv_len)
    batch = aibx.KVBatch(e.table, e.tok_off, kv, n, max_new=max(nodes))
    ws = torch.empty(aibx.attn_tree_workspace_bytes(e.cache, batch, out), dtype=torch.uint8, device="cuda")

    def draft():
        aibx.kv_tables(before, d["new"], T, e.s.blocks, e.free, head0, e.tail, e.table, e.tok_off, kv, n, head_out=head)
        aibx.tree_masks(d["parent"], e.tok_off, kv, d["mask"], pos=d["pos"])
        aibx.rope_append(e.cache, batch, e.rope, k, v, q=q, q_out=turned, pos=d["pos"])
        aibx.attn_tree(e.cache, batch, d["mask"], turned, out, lse=lse, workspace=ws)

    stream = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        draft()
    for turn in range(3):
        trees = [random_tree(e.rng, m) for m in nodes]
        d["parent"].copy_(dev(np.array([p for t in trees for p in t], dtype=np.int32)))
        x = e.qkv(n)
        d["x"].copy_(x)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        e.kv_len = kv
        b = e.reference(nodes)
        sets = [ancestors(t) for t in trees]
        at = np.array([int(before[r]) + len(s) - 1 for r, t in enumerate(sets) for s in t])
        assert d["pos"].tolist() == at.tolist()
        want, err = rotate(e.split(x)[0].double().numpy(), at, e.f, False, e.factor)
        assert (np.abs(turned.double().cpu().numpy() - want) <= err + 2.0 ** -8 * (np.abs(want) + err)).all()
        o, _, mag, slack = tree_attention(e.s, b, e.values(), turned.double().cpu().numpy(), e.D ** -0.5, sets, 0)
        near(out, o, tree_tolerance(e.s, "bf16", o, mag, slack))
        first = out.clone()
        out.zero_()
        draft()                                              # the same, eager
        assert torch.equal(out, first)
    assert int(head) - int(head0) == sum(-(-(int(a) + m) // T) - -(-int(a) // T) for a, m in zip(before, nodes))
    assert aibx.status_fetch() == (0, 0)


def test_two_layers_on_two_streams():
    """Two layers' keys appended and read by attention at the same time, with workspaces of their own."""
    rng = np.random.default_rng(3)
    s = [Shape(H=4, D=128, T=16, layers=2, layer=i, blocks=200, pool="fp16") for i in range(2)]
    new = [int(x) for x in rng.integers(1, 30, 8)]
    lens = [m + int(c) for m, c in zip(new, rng.integers(0, 300, 8))]
    b = Batch(rng, s[0], new, lens)
    host, _ = make_pool(rng, s[0])
    pool = host.cuda()
    caches = [aibx.KVCache(pool, aibx.KVLayout(0, 2, 4, 16, 128, 2, 200), aibx.TYPE_FP16, layer=i) for i in range(2)]
    batch = aibx.KVBatch(dev(b.table), dev(b.tok_off), dev(b.kv_len), b.n_tokens, max_new=max(new))
    f, _ = aibx.rope_frequencies(128)
    rope = aibx.Rope(f.cuda(), interleaved=True)
    x = torch.from_numpy(rng.normal(size=(b.n_tokens, 16 + 8, 128))).half().cuda()
    sets = [[set(range(i + 1)) for i in range(m)] for m in new]
    from steps_ref import pack
    mask = dev(np.concatenate([pack(t, 1) for t in sets]))
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [torch.zeros(b.n_tokens, 16, 128, dtype=torch.float16, device="cuda") for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(4):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                q = torch.empty(b.n_tokens, 16, 128, dtype=torch.float16, device="cuda")
                aibx.rope_append(caches[i], batch, rope, x[:, 16:20], x[:, 20:], q=x[:, :16], q_out=q)
                aibx.attn_tree(caches[i], batch, mask, q, outs[i])
    torch.cuda.synchronize()
    turned, _ = rotate(x.double().cpu().numpy(), np.array([p for _, _, p in b.tokens()]), f.numpy(), True, 1.0)
    for i in range(2):
        o, _, mag, slack = tree_attention(s[i], b, pool_values(s[i], pool.cpu(), None), q.double().cpu().numpy(), 128 ** -0.5, sets, 0)
        near(outs[i], o, tree_tolerance(s[i], "fp16", o, mag, slack))
    assert np.abs(q.double().cpu().numpy() - turned[:, :16]).max() < 0.02
    assert aibx.status_fetch() == (0, 0)


def test_tensors_of_another_device_are_refused():
    e = Engine(2)
    x = torch.zeros(3, 2, 64, dtype=torch.bfloat16)
    pos = torch.zeros(3, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):
        aibx.rope(e.rope, pos, x, x)
    with pytest.raises(ValueError):
        aibx.rope(e.rope, pos.cpu(), x.cuda(), x.cuda())
    with pytest.raises(ValueError):
        aibx.tree_masks(pos, e.tok_off, e.kv_len, torch.zeros(3, 1, dtype=torch.int64).view(torch.uint64))
    with pytest.raises(ValueError):
        e.grow(e.kv_len.cpu(), e.kv_len, 3)
    with pytest.raises(ValueError):
        e.grow(e.kv_len, e.kv_len.cpu(), 3)
    with pytest.raises(ValueError):
        aibx.attn_tree(e.cache, e.batch(3, 3), torch.zeros(3, 1, dtype=torch.int64).view(torch.uint64), x.cuda(), x.cuda())
