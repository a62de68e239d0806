"""Plain 64-bit reference of the token-wise calls on a paged pool (append, read, attention), in
numpy, position by position, and the inputs their tests share."""
import numpy as np
import torch

NO_BLOCK = 0xFFFFFFFF
DTYPE = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
# largest relative error of one rounding to nearest
HALF_STEP = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11, "fp32": 2.0 ** -24, "e4m3": 2.0 ** -4}


class Shape:
    def __init__(self, H=2, D=64, T=16, layers=2, layer=1, blocks=40, layout=0, inner=0, pool="bf16"):
        self.H, self.D, self.T, self.layers, self.layer = H, D, T, layers, layer
        self.blocks, self.layout, self.inner, self.pool = blocks, layout, inner, pool
        self.elem = 1 if pool == "e4m3" else 2
        self.rows = blocks * layers * 2 * H * T

    def row(self, block, kv, head, slot):
        """Index of a row of D elements (= of its scale byte) in the pool."""
        H, T, L, NB = self.H, self.T, self.layers, self.blocks
        at = slot * H + head if self.inner else head * T + slot
        plane = {0: (block * L + self.layer) * 2 + kv, 1: (self.layer * NB + block) * 2 + kv,
                 2: (self.layer * 2 + kv) * NB + block}[self.layout]
        return plane * H * T + at


class Batch:
    """Requests with `new[r]` tokens out of `length[r]`; tables of `width` entries (blocks at
    random), ragged when `width` is None."""

    def __init__(self, rng, s, new, length, width=None, ragged=False, pad=0, spare=1):
        self.new, self.length = list(new), list(length)
        need = [-(-max(x, 0) // s.T) for x in length]
        ids = rng.permutation(s.blocks)
        assert sum(need) <= s.blocks
        rows, at = [], 0
        for k in need:
            rows.append(list(ids[at:at + k]))
            at += k
        if ragged:
            self.blk_off = np.concatenate([[0], np.cumsum(need)]).astype(np.int64)
            self.table = np.array([b for r in rows for b in r] or [0], dtype=np.uint32)
        else:
            w = width if width is not None else max(need + [0]) + spare
            self.blk_off = None
            self.table = np.full((len(new), w), NO_BLOCK, dtype=np.uint32)
            for r, b in enumerate(rows):
                self.table[r, :len(b)] = b[:w]
        self.tok_off = np.concatenate([[0], np.cumsum(new)]).astype(np.int64)
        self.n_tokens = int(self.tok_off[-1]) + pad
        self.kv_len = np.array(length, dtype=np.int32)

    def entry(self, s, r, pos):
        """Block id of a position, or None where the table has no entry."""
        if pos < 0:
            return None
        k = pos // s.T
        row = self.table[r] if self.blk_off is None else self.table[self.blk_off[r]:self.blk_off[r + 1]]
        if k >= len(row) or row[k] >= s.blocks:
            return None
        return int(row[k])

    def tokens(self):
        for r, n in enumerate(self.new):
            for i in range(n):
                yield int(self.tok_off[r]) + i, r, self.length[r] - n + i


def e4m3_values():
    b = np.arange(256)
    m, e = b & 7, (b >> 3) & 15
    v = np.where(e == 0, m * 2.0 ** -9, (1 + m / 8) * 2.0 ** (e - 7.0))
    v = np.where((b & 127) == 127, np.nan, v)
    return np.where(b >= 128, -v, v)


E4M3 = e4m3_values()


def quantise(x):
    """(e4m3 bytes, scale byte) of a row, by search: the smallest power, the nearest value with
    ties to the even byte."""
    x = np.asarray(x, dtype=np.float64)
    fin = np.abs(x[np.isfinite(x)])
    a = fin.max() if len(fin) else 0.0
    byte = 127
    if a > 0:
        byte = next(b for b in range(1, 255) if a <= 448 * 2.0 ** (b - 127))
    y = x * 2.0 ** (127 - byte)
    mags = E4M3[:127]
    out = np.zeros(len(x), dtype=np.uint8)
    for i, v in enumerate(y):
        if not np.isfinite(v):
            out[i] = 127
            continue
        d = np.abs(mags - abs(v))
        best = np.flatnonzero(d == d.min())
        k = best[0] if len(best) == 1 else [c for c in best if c % 2 == 0][0]
        out[i] = k | (128 if np.signbit(v) else 0)
    return out, byte


def pool_values(s, pool, scales):
    """The pool's rows as 64-bit numbers, [rows][D] (pool: torch tensor on the host)."""
    if s.pool == "e4m3":
        v = E4M3[pool.view(torch.uint8).numpy().reshape(s.rows, s.D)]
        f = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
        return v * f[:, None]
    return pool.double().numpy().reshape(s.rows, s.D)


def attention(s, b, values, q, scale, causal, window):
    """(out, lse, sum of w |v|, error of a score) in 64 bits; rows of tokens no request has stay
    NaN."""
    n, Hq, D = q.shape
    G = Hq // s.H
    out = np.full((b.n_tokens, Hq, D), np.nan)
    lse = np.full((b.n_tokens, Hq), np.nan)
    mag, slack = np.zeros_like(out), np.zeros_like(lse)
    for i, r, p in b.tokens():
        keys = [j for j in range(max(b.length[r], 0)) if (not causal or j <= p) and
                (window <= 0 or j > p - window) and b.entry(s, r, j) is not None]
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
            # fp32 products and sums of D terms; queries over e4m3 are fp16 within 2^-25 of the
            # largest of their row, which is below one fp32 rounding of D terms of that size
            slack[i, h] = scale * (D + 4) * 2.0 ** -24 * np.abs(values[kr]).max() * np.abs(q[i, h]).sum() \
                + 4 * 2.0 ** -24 * abs(m)
    return out, lse, mag, slack


def tolerance(s, io, out, mag, slack):
    """Elementwise bound: the weights rounded to the operand type (half a step), the scores' error
    (twice: in the weight and in the sum), 2^-20 for exponentials and sums, the result rounded
    once."""
    u = HALF_STEP["fp16" if s.pool == "e4m3" else io]
    # fp16 weights below 2^-14 of the largest round on a grid of 2^-25
    grid = 2.0 ** -25 * 512 if (s.pool == "e4m3" or io == "fp16") else 0.0
    return (u + 2 * slack[..., None] + 2.0 ** -20) * mag + HALF_STEP[io] * np.abs(out) + grid * mag.max() + 1e-30
