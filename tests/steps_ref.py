"""Plain 64-bit references of the calls around a step - block tables, ancestor masks, rotary positions,
attention of drafted trees - and bounds on what their roundings can do."""
import numpy as np

from paged_ref import HALF_STEP, NO_BLOCK, tolerance


def ancestors(parents):
    """Per node of one request the set of nodes that it sees."""
    seen = []
    for i, p in enumerate(parents):
        seen.append({i} | (seen[p] if 0 <= p < i else set()))
    return seen


def pack(sets, words):
    """Sets of whole numbers as rows of 64-bit words."""
    out = np.zeros((len(sets), words), dtype=np.uint64)
    for i, s in enumerate(sets):
        for j in s:
            if j < 64 * words:
                out[i, j // 64] |= np.uint64(1) << np.uint64(j % 64)
    return out


def random_tree(rng, n, roots=1):
    return [-1 if i < roots else int(rng.integers(-1 if rng.random() < 0.1 else 0, i)) for i in range(n)]


def tree_attention(s, b, values, q, scale, sets, window):
    """(out, lse, sum of w |v|, error of a score) in 64 bits, as paged_ref.attention; sets[r][i]: the nodes
    of request r that its node i sees."""
    n, Hq, D = q.shape
    G = Hq // s.H
    out = np.full((b.n_tokens, Hq, D), np.nan)
    lse = np.full((b.n_tokens, Hq), np.nan)
    mag, slack = np.zeros_like(out), np.zeros_like(lse)
    for i, r, _ in b.tokens():
        base = b.length[r] - b.new[r]
        nodes = {j for j in sets[r][i - int(b.tok_off[r])] if j < b.new[r]}
        at = base + max(len(nodes) - 1, 0)
        keys = [j for j in range(base) if window <= 0 or j > at - window]
        keys += sorted(base + j for j in nodes if base + j >= 0)
        keys = [j for j in keys if b.entry(s, r, j) is not None]
        for h in range(Hq):
            if not keys:
                out[i, h], lse[i, h] = 0.0, -np.inf
                continue
            kr = [s.row(b.entry(s, r, j), 0, h // G, j % s.T) for j in keys]
            vr = [s.row(b.entry(s, r, j), 1, h // G, j % s.T) for j in keys]
            z = scale * (values[kr] @ q[i, h])
            m = z.max()
            w = np.exp(z - m)
            t = w.sum()
            lse[i, h] = m + np.log(t)
            out[i, h] = (w / t) @ values[vr]
            mag[i, h] = (w / t) @ np.abs(values[vr])
            slack[i, h] = scale * (D + 4) * 2.0 ** -24 * np.abs(values[kr]).max() * np.abs(q[i, h]).sum() \
                + 4 * 2.0 ** -24 * abs(m)
    return out, lse, mag, slack


def tree_tolerance(s, io, out, mag, slack):
    """paged_ref.tolerance, but over e4m3 the weights of bf16 queries may be bf16: each is off by at most
    half a step of that, relative to itself, so out by at most as much of the sum of w |v|.  (Those of fp16
    queries are the sum of two bf16 numbers, within 2^-16: nearer than the fp16 that is allowed for.)"""
    more = HALF_STEP["bf16"] - HALF_STEP["fp16"] if s.pool == "e4m3" and io == "bf16" else 0.0
    return tolerance(s, io, out, mag, slack) + more * mag


def rotate(x, pos, freq, interleaved, factor):
    """Rows x [n][heads][D] turned, and a bound on what 32-bit arithmetic may be off by, before any
    rounding to the output's type.  Sine and cosine: 2 ulp of theirs, the angle's fraction of a turn rounded
    to 32 bits (2 pi * 0.5 * 2^-24 radians) after two 64-bit roundings of the turns, the factor's product;
    then a product and a sum: all within 8 * 2^-24 of (|x1| + |x2|) * factor."""
    half = len(freq)
    a = pos.astype(np.float64)[:, None] * freq[None]
    c, s = np.cos(a)[:, None] * factor, np.sin(a)[:, None] * factor
    y, err = x.copy(), np.zeros_like(x)
    if interleaved:
        i1, i2 = slice(0, 2 * half, 2), slice(1, 2 * half, 2)
    else:
        i1, i2 = slice(0, half), slice(half, 2 * half)
    x1, x2 = x[..., i1], x[..., i2]
    y[..., i1] = x1 * c - x2 * s
    y[..., i2] = x2 * c + x1 * s
    turns = np.abs(a)[:, None] / (2 * np.pi)
    e = (np.abs(x1) + np.abs(x2)) * factor * (8 * 2.0 ** -24 + 2 * np.pi * turns * 2.0 ** -51)
    err[..., i1] = e
    err[..., i2] = e
    return y, err


# half the step between a type's subnormal numbers
LEAST = {"bf16": 2.0 ** -134, "fp16": 2.0 ** -25, "fp32": 2.0 ** -150}


def within(got, want, err, io):
    """Whether got is want, off by err, rounded once to the type."""
    return (np.abs(got - want) <= err + HALF_STEP[io] * (np.abs(want) + err) + LEAST[io]).all()


class Ring:
    """A free list: ids numbered head .. tail - 1 in a ring."""

    def __init__(self, ids, head, tail):
        self.ids, self.head, self.tail = np.asarray(ids, dtype=np.uint32), head, tail


def tables(held, new, T, num_blocks, ring, rows, match=None, n_tokens=None):
    """rows: list of numpy rows (views of the table), grown in place.  Returns tok_off, kv_len, pos, slots,
    head, blocks that were missing, requests or ids that are wrong."""
    off, kv, pos, slots = [0], [], [], []
    head, missing, wrong = ring.head, 0, 0
    left = min(max(ring.tail - ring.head, 0), len(ring.ids))
    for r, (h, n) in enumerate(zip(held, new)):
        h, n = int(h), int(n)
        if h < 0 or n < 0 or h + n > 2 ** 31 - 1:
            wrong += 1
            h, n = max(h, 0), 0
        row, had, need = rows[r], -(-h // T), -(-(h + n) // T)
        if match is not None:
            for e in range(min(had, len(row))):
                row[e] = match[r][e] if e < len(match[r]) else NO_BLOCK
                wrong += e >= len(match[r])
        if n > 0 and need > len(row):
            wrong += 1
        for e in range(had, min(need, len(row))):
            if left > 0:
                row[e] = ring.ids[head % len(ring.ids)]
                head += 1
                left -= 1
            else:
                row[e] = NO_BLOCK
                missing += 1
        for p in range(h, h + n):
            pos.append(p)
            if match is not None and p // T < had:
                id = match[r][p // T] if p // T < len(match[r]) and p // T < len(row) else NO_BLOCK
            else:
                id = row[p // T] if p // T < len(row) else NO_BLOCK
            slots.append(int(id) * T + p % T if id < num_blocks else -1)
            wrong += id >= num_blocks and id != NO_BLOCK
        kv.append(h + n)
        off.append(off[-1] + n)
    if n_tokens is not None and off[-1] > n_tokens:
        wrong += 1
    return off, kv, pos, slots, head, missing, wrong
