"""Float64 CPU oracle for the 8-bit block cache.

TEST INFRASTRUCTURE ONLY, like ``kvc_oracle``: the definitions of the C header written out token by
token in NumPy, without the library's blocking or order of evaluation.

* quantise: the scale of a block is the least 2^e, e >= -100, with amax <= top * 2^e (top 448 for
  e4m3, 127 for int8); a code is the format's number nearest to value / scale, halves to even.
* fill, append, evict change a :class:`Cache` in place, exactly as the library must, bit for bit.
* attend: softmax over the tokens that a query sees, in float64.
"""
from __future__ import annotations

import numpy as np

BLOCK = 64
E4M3, INT8 = 0, 1
TOP = {E4M3: 448.0, INT8: 127.0}


def _e4m3_values() -> np.ndarray:
    """The number of each of the 256 codes: sign, 4 exponent bits (bias 7), 3 mantissa bits; no infinities, 0x7f and
    0xff are NaN."""
    v = np.empty(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        x = m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
        v[c] = (-1) ** (c >> 7) * (np.nan if c & 127 == 127 else x)
    return v


VALUES = {E4M3: _e4m3_values(), INT8: np.arange(256, dtype=np.uint8).view(np.int8).astype(np.float64)}


def decode(codes, fmt):
    return VALUES[fmt][codes]


def encode(y, fmt):
    """Codes of numbers already divided by their scale."""
    y = np.asarray(y, dtype=np.float64)
    if fmt == INT8:
        return np.rint(y).astype(np.int8).view(np.uint8)
    grid = VALUES[E4M3][:127]                                  # 0 .. 448, ascending
    a = np.abs(y)
    hi = np.clip(np.searchsorted(grid, a), 0, 126)             # grid[hi] >= a
    lo = np.maximum(hi - 1, 0)
    up, down = grid[hi] - a, a - grid[lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo).astype(np.uint8)
    return code | np.where(np.signbit(y), 128, 0).astype(np.uint8)


def scale_of(amax, fmt):
    e = -100
    while float(amax) > TOP[fmt] * 2.0 ** e:
        e += 1
    return np.float32(2.0 ** e)


class Cache:
    """Pools as the C header lays them out; hb heads to a block."""

    def __init__(self, fmt, blocks, hkv, d, table, layers, unstructured=False, fill=0):
        self.fmt, self.hkv, self.d, self.layers, self.unstructured = fmt, hkv, d, layers, unstructured
        self.hb = 1 if unstructured else hkv
        self.k = np.full((blocks, self.hb, BLOCK, d), fill, np.uint8)
        self.v = np.full((blocks, self.hb, d, BLOCK), fill, np.uint8)
        self.k_scale = np.full((blocks, self.hb), np.nan, np.float32)
        self.v_scale = np.full((blocks, self.hb), np.nan, np.float32)
        self.weight = np.full((blocks, self.hb, BLOCK), np.nan, np.float32)
        self.table = np.asarray(table, np.int32)

    def copy(self):
        c = Cache.__new__(Cache)
        c.__dict__ = {k: v.copy() if isinstance(v, np.ndarray) else v for k, v in self.__dict__.items()}
        return c

    def row(self, b, l, h):
        return ((b * self.layers + l) * self.hkv + h, 0) if self.unstructured else (b * self.layers + l, h)

    def heads(self):
        """(row, place in the block, sequence, layer, head) of every head."""
        for b in range(self.table.shape[0] // (self.layers * (self.hkv if self.unstructured else 1))):
            for l in range(self.layers):
                for h in range(self.hkv):
                    yield self.row(b, l, h) + (b, l, h)

    def length(self, n):
        return int(min(max(n, 0), self.table.shape[1] * BLOCK))

    def block(self, row, j):
        i = int(self.table[row, j])
        return i if 0 <= i < len(self.k) else None

    def put(self, i, hh, k, v, weight):
        """A whole block: rows [n <= 64, d], zeros behind them."""
        pad = ((0, BLOCK - len(k)), (0, 0))
        ks, vs = (scale_of(np.abs(x).max(initial=0.0), self.fmt) for x in (k, v))
        self.k[i, hh] = encode(np.pad(k, pad) / float(ks), self.fmt)
        self.v[i, hh] = encode(np.pad(v, pad) / float(vs), self.fmt).T
        self.k_scale[i, hh], self.v_scale[i, hh] = ks, vs
        if weight is not None:
            self.weight[i, hh] = np.pad(weight, (0, BLOCK - len(k)))

    def tokens(self, row, hh, n):
        """Values of the first n tokens in float64, and which of them are there."""
        k, v, there = np.zeros((n, self.d)), np.zeros((n, self.d)), np.zeros(n, bool)
        w = np.full(n, -np.inf, np.float32)
        for j in range(-(-n // BLOCK)):
            i, s = self.block(row, j), slice(j * BLOCK, min(n, (j + 1) * BLOCK))
            if i is None:
                continue
            m = s.stop - s.start
            k[s] = decode(self.k[i, hh, :m], self.fmt) * float(self.k_scale[i, hh])
            v[s] = decode(self.v[i, hh, :, :m].T, self.fmt) * float(self.v_scale[i, hh])
            w[s], there[s] = self.weight[i, hh, :m], True
        return k, v, w, there


def fill(cache, k, v, idx, lengths, cu, scores=None, weighted=True):
    """k, v: [Lyr, Hkv, T, d] float64; idx: [Lyr, Hkv, T] or None."""
    for row, hh, b, l, h in cache.heads():
        n_b = int(cu[b + 1] - cu[b])
        n = cache.length(min(int(lengths[row]), n_b))
        at = np.arange(n) if idx is None else idx[l, h, cu[b]:cu[b] + n].astype(np.int64)
        at = at + int(cu[b])
        for j in range(-(-n // BLOCK)):
            i, s = cache.block(row, j), at[j * BLOCK:(j + 1) * BLOCK]
            if i is not None:
                w = np.zeros(len(s), np.float32) if scores is None else scores[l, h, s]
                cache.put(i, hh, k[l, h, s], v[l, h, s], w if weighted else None)


def append(cache, layer, k_new, v_new, lengths, weighted=True):
    """k_new, v_new: [Bt, Hkv, M, d] float64."""
    m = k_new.shape[2]
    for row, hh, b, l, h in cache.heads():
        n = int(lengths[row])
        if l != layer or n > cache.table.shape[1] * BLOCK:
            continue
        for j in range(-(-max(n, 0) // BLOCK)):
            slots = [t for t in range(j * BLOCK, min(n, (j + 1) * BLOCK)) if t >= n - m]
            i = cache.block(row, j)
            if not slots or i is None:
                continue
            old = slots[0] - j * BLOCK
            for name, new in (("k", k_new), ("v", v_new)):
                codes = getattr(cache, name)[i, hh]
                codes = codes if name == "k" else codes.T                       # [64, d], a view
                scales = getattr(cache, name + "_scale")
                x = np.stack([new[b, h, t - (n - m)] for t in slots])
                scale = scale_of(np.abs(x).max(initial=0.0), cache.fmt)
                if old:
                    was = scales[i, hh]
                    scale = max(scale, was)
                    if scale > was:
                        codes[:old] = encode(decode(codes[:old], cache.fmt) * (float(was) / float(scale)), cache.fmt)
                scales[i, hh] = scale
                codes[old:old + len(slots)] = encode(x / float(scale), cache.fmt)
            if weighted:
                cache.weight[i, hh, old:old + len(slots)] = 0


def attend(cache, layer, q, lengths, scale, causal=False, max_length=1 << 29):
    """q: [Bt, Hq, M, d] float64.  Returns out, lse, gathered {(row, hh): weight of each token}, and
    per output the two magnitudes that bound the rounding errors: sum p |v| and the largest
    sum |q k| * scale of the row."""
    bt, hq, m, d = q.shape
    group = hq // cache.hkv
    out, lse = np.zeros(q.shape), np.full((bt, hq, m), -np.inf)
    mean_abs, largest = np.zeros(q.shape), np.zeros((bt, hq, m))
    gathered = {}
    for row, hh, b, l, h in cache.heads():
        if l != layer:
            continue
        whole = cache.length(lengths[row])
        n = min(whole, max_length)
        k, v, _, there = cache.tokens(row, hh, n)
        got = np.zeros(n)
        for g in range(h * group, (h + 1) * group):
            for j in range(m):
                seen = there & (np.arange(n) < (whole - m + 1 + j if causal else n))
                if not seen.any():
                    continue
                s = (k[seen] @ q[b, g, j]) * scale
                top = s.max()
                e = np.exp(s - top)
                p = e / e.sum()
                out[b, g, j], mean_abs[b, g, j] = p @ v[seen], p @ np.abs(v[seen])
                lse[b, g, j] = top + np.log(e.sum())
                largest[b, g, j] = (np.abs(k[seen]) @ np.abs(q[b, g, j])).max() * scale
                got[seen] += p
        gathered[row, hh] = got
    return out, lse, gathered, mean_abs, largest


def evict(cache, lengths, keep, table_out, max_keep, keep_first=0, keep_last=0):
    """Returns lengths_out; writes the kept tokens into the blocks of table_out."""
    source, lengths_out = cache.copy(), np.zeros(len(lengths), np.int32)
    target = cache.copy()
    target.table = np.asarray(table_out, np.int32)
    for row, hh, b, l, h in cache.heads():
        n = cache.length(lengths[row])
        kept = max(0, min(int(keep[row]), max_keep, n))
        lengths_out[row] = kept
        k, v, w, _ = source.tokens(row, hh, n)
        rank = w.copy()
        rank[:keep_first] = np.inf
        rank[max(0, n - keep_last):] = np.inf
        order = sorted(range(n), key=lambda t: (-rank[t], t))
        at = np.array(sorted(order[:kept]), dtype=np.int64)
        w = np.where(np.isneginf(w), 0, w).astype(np.float32)                   # absent tokens: zeros
        for j in range(-(-kept // BLOCK)):
            i, s = target.block(row, j), at[j * BLOCK:(j + 1) * BLOCK]
            if i is not None:
                target.put(i, hh, k[s], v[s], w[s])
    for name in ("k", "v", "k_scale", "v_scale", "weight"):
        setattr(cache, name, getattr(target, name))
    return lengths_out
