"""GPU tests of block tables and ancestor masks against plain references: whole numbers, bit for bit."""
import numpy as np
import pytest
import torch

from paged_ref import NO_BLOCK
from paper_2504_03648_b200 import binding as aibx
from steps_ref import Ring, ancestors, pack, random_tree, tables

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _clean_status():
    aibx.status_fetch()
    yield


def dev(a, dtype=None):
    return torch.from_numpy(np.ascontiguousarray(a if dtype is None else np.asarray(a, dtype=dtype))).cuda()


class Step:
    """Random requests with rows, a ring that wraps, matched ids."""

    def __init__(self, seed, R, T, new, ctx, ragged=False, match=False, spare=2, short=0, pad=3, extra=0):
        rng = np.random.default_rng(seed)
        self.T, self.R, self.match, self.ragged = T, R, match, ragged
        self.held = rng.integers(0, ctx + 1, R)
        if match:
            self.held = self.held // T * T
            self.held[::3] = np.maximum(self.held[::3] - 1, 0)       # all but the last token matched
        self.new = np.broadcast_to(np.asarray(new if np.ndim(new) else rng.integers(0, new + 1, R)), (R,)).copy()
        had, need = -(-self.held // T), -(-(self.held + self.new) // T)
        fresh = int((need - had).sum())
        fresh += extra
        self.blocks = fresh + int(had.sum()) + 7
        cap = fresh + 3
        head = 10 * cap + cap // 2
        self.ring = Ring(rng.permutation(max(self.blocks, cap))[:cap], head, head + cap - 1 - short)
        self.match_rows = [rng.integers(0, self.blocks, h).astype(np.uint32) for h in had] if match else None
        widths = need + rng.integers(0, spare + 1, R) if ragged else np.full(R, max(list(need) + [0]) + spare)
        self.blk_off = np.concatenate([[0], np.cumsum(widths)]).astype(np.int64)
        self.flat = np.full(int(self.blk_off[-1]) + 1, 0xABCD, dtype=np.uint32)
        if not match:
            for r in range(R):
                self.flat[self.blk_off[r]:self.blk_off[r] + had[r]] = rng.integers(0, self.blocks, had[r])
        self.n = int(self.new.sum())
        self.rows = self.n + pad

    def want(self):
        flat = self.flat.copy()
        rows = [flat[self.blk_off[r]:self.blk_off[r + 1]] for r in range(self.R)]
        return (flat,) + tables(self.held, self.new, self.T, self.blocks, self.ring, rows, self.match_rows, self.rows)

    def run(self, in_place=False):
        d = {}
        d["held"], d["new"] = dev(self.held, np.int32), dev(self.new, np.int32)
        d["table"] = dev(self.flat)
        table = d["table"][:-1] if self.ragged else d["table"][:-1].view(self.R, -1)
        d["head"], d["tail"] = dev([self.ring.head], np.int64), dev([self.ring.tail], np.int64)
        d["head_out"] = d["head"] if in_place else dev([-1], np.int64)
        d["kv_len"] = d["held"] if in_place else torch.full((self.R,), -7, dtype=torch.int32, device="cuda")
        d["tok_off"] = torch.full((self.R + 1,), -7, dtype=torch.int64, device="cuda")
        d["pos"] = torch.full((self.rows,), -7, dtype=torch.int32, device="cuda")
        d["slots"] = torch.full((self.rows,), -7, dtype=torch.int64, device="cuda")
        match = {}
        if self.match:
            ids = np.concatenate(self.match_rows + [np.zeros(1, dtype=np.uint32)])
            match = dict(match_ids=dev(ids), match_off=dev(np.concatenate([[0], np.cumsum([len(x) for x in self.match_rows])]), np.int64))
        self.free = dev(self.ring.ids)
        self.call = lambda: aibx.kv_tables(
            d["held"], d["new"], self.T, self.blocks, self.free, d["head"], d["tail"], table, d["tok_off"], d["kv_len"],
            self.rows, pos=d["pos"], slots=d["slots"], head_out=d["head_out"],
            blk_off=dev(self.blk_off) if self.ragged else None, **match)
        self.call()
        return d

    def check(self, d, status=(0, 0)):
        flat, off, kv, pos, slots, head, missing, wrong = self.want()
        assert np.array_equal(d["table"].cpu().numpy(), flat)
        assert d["tok_off"].tolist() == off and d["kv_len"].tolist() == kv
        n = min(len(pos), self.rows)
        assert d["pos"].tolist() == pos[:n] + [-7] * (self.rows - n)
        assert d["slots"].tolist() == slots[:n] + [-7] * (self.rows - n)
        assert int(d["head_out"]) == head
        code, detail = aibx.status_fetch()
        assert code == status[0]
        assert (missing > 0) == (code == aibx.ERR_FULL) and (code != aibx.ERR_RANGE or wrong > 0)
        if code == aibx.ERR_FULL and not wrong:
            assert detail == missing


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("match,ragged", [(False, False), (True, False), (False, True), (True, True)])
@pytest.mark.parametrize("R,T,new,ctx", [(1, 16, [1], 0), (1, 16, [1], 40), (3, 8, 0, 50), (7, 16, 1, 70), (200, 16, 1, 300),
                                         (511, 1, 3, 9), (512, 24, 9, 30), (513, 32, 65, 200), (1500, 16, 2, 40),
                                         (5, 64, 5000, 3000), (1, 16, [30001], 100), (40, 7, 900, 900)])
def test_tables(R, T, new, ctx, match, ragged, in_place):
    s = Step(R * 31 + T, R, T, new, ctx, ragged=ragged, match=match)
    s.check(s.run(in_place))


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("short", [1, 5, 40])
def test_too_few_blocks(short, in_place):
    """The ring holds two more ids than are wanted, less `short`."""
    s = Step(short, 30, 16, 90, 100, short=short)
    s.check(s.run(in_place), status=(aibx.ERR_FULL if short > 2 else 0,))


def test_no_free_ids_at_all():
    s = Step(3, 20, 8, 30, 30)
    s.ring.tail = s.ring.head - 5                            # behind its head: nothing there
    s.check(s.run(), status=(aibx.ERR_FULL,))


def test_wrong_lengths_and_rows():
    s = Step(4, 12, 16, 20, 60, extra=30)
    s.held[2], s.new[5] = -3, -1
    s.new[7] = 16 * int(s.blk_off[1]) + 5                    # more blocks than its row has entries
    s.rows = int(np.maximum(s.new, 0).sum()) + 2
    s.check(s.run(), status=(aibx.ERR_RANGE,))


def test_lengths_past_the_last_position():
    s = Step(5, 3, 1024, [5, 40, 5], 60, extra=9)
    s.held[1] = 2 ** 31 - 20
    d = s.run()
    assert d["tok_off"].tolist() == [0, 5, 5, 10] and d["kv_len"].tolist()[1] == 2 ** 31 - 20
    assert aibx.status_fetch()[0] == aibx.ERR_RANGE


def test_bad_ids_and_missing_matches():
    s = Step(6, 9, 8, 20, 40, match=True, extra=9)
    s.match_rows[3] = s.match_rows[3][:len(s.match_rows[3]) // 2]
    s.ring.ids[:] = s.blocks + 1
    for m in s.match_rows[4:5]:
        m[:] = NO_BLOCK
    s.check(s.run(), status=(aibx.ERR_RANGE,))


def test_fewer_rows_than_tokens():
    s = Step(7, 9, 8, 20, 40, pad=-11)
    s.check(s.run(), status=(aibx.ERR_RANGE,))


def test_positions_and_slots_are_optional():
    s = Step(8, 20, 16, 30, 100)
    d = s.run()
    table = dev(s.flat)
    kv = torch.empty_like(d["kv_len"])
    aibx.kv_tables(d["held"], d["new"], s.T, s.blocks, s.free, d["head"], d["tail"], table[:-1].view(s.R, -1),
                   torch.empty_like(d["tok_off"]), kv, s.rows, head_out=torch.empty_like(d["head"]))
    assert torch.equal(table, d["table"]) and torch.equal(kv, d["kv_len"])
    aibx.status_fetch()


def test_a_captured_step_walks_on():
    """One captured call with its outputs in the place of its inputs: replayed, it is the next step each time."""
    T, R, steps = 8, 33, 40
    rng = np.random.default_rng(1)
    held0 = rng.integers(0, 30, R).astype(np.int32)
    rows = [[int(x) for x in rng.integers(500, 600, -(-h // T))] for h in held0]
    width = 12
    table = np.full((R, width), NO_BLOCK, dtype=np.uint32)
    for r, x in enumerate(rows):
        table[r, :len(x)] = x
    cap = 300
    ids = rng.permutation(400)[:cap].astype(np.uint32)
    new = rng.integers(0, 3, R).astype(np.int32)
    n = int(new.sum())
    d_held, d_new, d_table, d_ids = dev(held0), dev(new), dev(table), dev(ids)
    head, tail = dev([0], np.int64), dev([cap], np.int64)
    off = torch.empty(R + 1, dtype=torch.int64, device="cuda")
    pos = torch.empty(n, dtype=torch.int32, device="cuda")
    slots = torch.empty(n, dtype=torch.int64, device="cuda")

    def call():
        aibx.kv_tables(d_held, d_new, T, 1000, d_ids, head, tail, d_table, off, d_held, n, pos=pos, slots=slots)

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        call()
    for _ in range(steps):
        graph.replay()
    torch.cuda.synchronize()
    want, ring, h = [table[r] for r in range(R)], Ring(ids, 0, cap), held0.astype(np.int64)
    for _ in range(steps):
        _, kv, wpos, wslots, ring.head, missing, _ = tables(h, new, T, 1000, ring, want)
        h = np.array(kv)
    assert missing == 0 and np.array_equal(d_held.cpu().numpy(), h)
    assert np.array_equal(d_table.cpu().numpy(), table) and int(head) == ring.head
    assert pos.tolist() == wpos and slots.tolist() == wslots
    assert aibx.status_fetch()[0] in (0, aibx.ERR_RANGE)     # (rows may have grown full)


# ------------------------------------------------------------------------------------------
# ancestors


@pytest.mark.parametrize("words,new", [(1, [1]), (1, [0, 26, 64, 1, 0, 33]), (2, [65, 128, 3]), (3, [192, 100, 0, 129]),
                                       (4, [256, 255, 7]), (5, [320]), (6, [384, 1]), (7, [448, 400]), (8, [512, 300, 0, 511, 64, 65])])
@pytest.mark.parametrize("kind", ["random", "chain", "star", "forest"])
def test_masks(words, new, kind):
    rng = np.random.default_rng(words * 100 + len(kind))
    trees = [{"random": random_tree(rng, n), "chain": list(range(-1, n - 1)), "star": [-1] + [0] * (n - 1),
              "forest": [-1] * n}[kind][:n] for n in new]
    off = np.concatenate([[0], np.cumsum(new)]).astype(np.int64)
    n, pad = int(off[-1]), 2
    kv = np.array([x + int(rng.integers(0, 1000)) for x in new], dtype=np.int32)
    parent = dev([p for t in trees for p in t] + [0] * pad, np.int32)
    mask = torch.full((n + pad, words), 7, dtype=torch.int64, device="cuda").view(torch.uint64)
    pos = torch.full((n + pad,), -7, dtype=torch.int32, device="cuda")
    aibx.tree_masks(parent, dev(off), dev(kv), mask, pos=pos)
    sets = [s for t in trees for s in ancestors(t)]
    want = np.concatenate([pack(sets, words), np.full((pad, words), 7, dtype=np.uint64)])
    assert np.array_equal(mask.cpu().numpy(), want)
    depth = [int(kv[r]) - new[r] + len(s) - 1 for r, t in enumerate(trees) for s in ancestors(t)]
    assert pos.tolist() == depth + [-7] * pad
    only = torch.zeros_like(mask.view(torch.int64)).view(torch.uint64)
    aibx.tree_masks(parent, dev(off), None, only)
    assert np.array_equal(only.cpu().numpy()[:n], want[:n])
    assert aibx.status_fetch() == (0, 0)


def test_masks_of_many_requests():
    rng = np.random.default_rng(9)
    new = [int(x) for x in rng.integers(0, 9, 3000)]
    trees = [random_tree(rng, n) for n in new]
    off = np.concatenate([[0], np.cumsum(new)]).astype(np.int64)
    mask = torch.zeros(int(off[-1]), 1, dtype=torch.int64, device="cuda").view(torch.uint64)
    aibx.tree_masks(dev([p for t in trees for p in t], np.int32), dev(off), None, mask)
    assert np.array_equal(mask.cpu().numpy(), pack([s for t in trees for s in ancestors(t)], 1))


def test_masks_refuse_on_the_device():
    """A parent that does not come before its node, and a request with more nodes than bits."""
    new = [5, 70, 4]
    off = np.concatenate([[0], np.cumsum(new)]).astype(np.int64)
    parents = [-1, 0, 2, 9, 1] + [-1] + list(range(69)) + [-5, 0, 1, 3]
    mask = torch.full((79, 1), 7, dtype=torch.int64, device="cuda").view(torch.uint64)
    aibx.tree_masks(dev(parents, np.int32), dev(off), None, mask)
    assert aibx.status_fetch() == (aibx.ERR_RANGE, 4)        # nodes 2 and 3 of the first, 3 of the last; the second request
    got = mask.cpu().numpy()[:, 0].tolist()
    assert got[:5] == [1, 3, 4, 8, 1 | 2 | 16] and got[5:75] == [7] * 70 and got[75:] == [1, 3, 7, 8]


def test_masks_of_fewer_rows_than_nodes():
    """A request that the per-token tensors cut off: positions still count from its first node."""
    off, kv = dev([0, 4, 10], np.int64), dev([50, 90], np.int32)
    mask = torch.zeros(7, 1, dtype=torch.int64, device="cuda").view(torch.uint64)
    pos = torch.zeros(7, dtype=torch.int32, device="cuda")
    aibx.tree_masks(dev([-1, 0, 0, 2, -1, 0, 1], np.int32), off, kv, mask, pos=pos)
    assert mask.cpu().numpy()[:, 0].tolist() == [1, 3, 5, 13, 1, 3, 7]
    assert pos.tolist() == [46, 47, 47, 48, 84, 85, 86]
