"""Decoding on packed records, slow and in 64 bits: appending tokens to pages, attention over pages, eviction by accumulated
attention weight.  Written from the record format and the definitions of the operations; shares no code with the library.

A pool is a numpy uint8 array, a page table off [n_seqs][pages] and bits [n_seqs][pages] (0: absent), length [n_seqs]."""
from __future__ import annotations

import numpy as np

from . import record_bytes


def _param_type(shape):
    return np.float16 if shape.fmt == 3 else np.float32


class Slab:
    """Views of one (layer, K|V, kv head) slab of a record of width b at byte `off` of the pool."""

    def __init__(self, shape, pool, off, b, layer, kv, head):
        T, D = shape.T, shape.D
        slabs, i = shape.L * 2 * shape.Hkv, (layer * 2 + kv) * shape.Hkv + head
        off, n = int(off), T * D * int(b) // 8
        self.b = int(b)
        self.codes = pool[off + i * n:off + (i + 1) * n].reshape(T, -1)
        if b != 16:
            t = np.dtype(_param_type(shape))
            m = T * (D // shape.G) * t.itemsize
            at = off + slabs * n
            self.scale = pool[at + i * m:at + (i + 1) * m].view(t).reshape(T, -1)
            at += slabs * m
            self.mn = pool[at + i * m:at + (i + 1) * m].view(t).reshape(T, -1)

    def values(self, shape):
        """float64 [T][D]: what the rows stand for."""
        if self.b == 16:
            return self.codes.view(np.float16).astype(np.float64)
        d = np.arange(shape.D)
        per = 8 // self.b
        code = (self.codes[:, d // per].astype(np.int64) >> (d % per * self.b)) & (2 ** self.b - 1)
        with np.errstate(invalid="ignore"):                      # (rows that no token has may hold anything)
            return code * self.scale.astype(np.float64)[:, d // shape.G] + self.mn.astype(np.float64)[:, d // shape.G]

    def dequantised(self, shape, row):
        """fp16 [D]: the row as a Load gives it (binary32, product and sum rounded separately)."""
        if self.b == 16:
            return self.codes[row].view(np.float16).copy()
        d = np.arange(shape.D)
        per = 8 // self.b
        code = ((self.codes[row, d // per].astype(np.int64) >> (d % per * self.b)) & (2 ** self.b - 1)).astype(np.float32)
        scale, mn = self.scale[row].astype(np.float32)[d // shape.G], self.mn[row].astype(np.float32)[d // shape.G]
        return (code * scale + mn).astype(np.float16)

    def put(self, shape, row, x):
        """Writes fp16 [D] into a row."""
        if self.b == 16:
            self.codes[row] = x.view(np.uint8)
            return
        top = np.float32(2 ** self.b - 1)
        g = x.astype(np.float32).reshape(-1, shape.G)
        mn = g.min(1) + np.float32(0)
        scale = ((g.max(1) + np.float32(0)) - mn) / top
        scale = scale.astype(_param_type(shape)).astype(np.float32)
        code = np.zeros_like(g)
        some = scale != 0
        code[some] = np.clip(np.rint((g[some] - mn[some, None]) / scale[some, None]), 0, top)
        code = code.reshape(-1).astype(np.uint8).reshape(-1, 8 // self.b)
        packed = np.zeros(len(code), dtype=np.uint8)
        for k in range(8 // self.b):
            packed |= code[:, k] << (k * self.b)
        self.codes[row], self.scale[row], self.mn[row] = packed, scale.astype(_param_type(shape)), mn.astype(_param_type(shape))


def present(shape, pool, off, b):
    off, b = int(off), int(b)
    return b in (16, 8, 4, 2) and off >= 0 and off % 16 == 0 and off + record_bytes(shape, b) <= pool.size


def rows_of(row_start, n_seqs, n_rows, s):
    """First row and number of rows of a sequence."""
    if row_start is None:
        return s, 1
    return int(row_start[s]), int(row_start[s + 1]) - int(row_start[s])


def append(shape, pool, off, bits, length, layer, k, v, row_start=None, seen=None, mass=None, pos=None):
    for s in range(len(length)):
        first, c = rows_of(row_start, len(length), len(k), s)
        for j in range(c):
            token = int(length[s]) - c + j
            if token < 0:
                continue
            if mass is not None:
                mass[s, :, token] = 0
            if pos is not None:
                pos[s, :, token] = (int(length[s]) if seen is None else int(seen[s])) - c + j
            page, row = token // shape.T, token % shape.T
            if present(shape, pool, off[s, page], bits[s, page]):
                for h in range(shape.Hkv):
                    Slab(shape, pool, off[s, page], bits[s, page], layer, 0, h).put(shape, row, k[first + j, h])
                    Slab(shape, pool, off[s, page], bits[s, page], layer, 1, h).put(shape, row, v[first + j, h])


def attend(shape, pool, off, bits, length, layer, q, row_start=None, max_rows=16, mass_in=None):
    """-> (out float64 [n_rows][Hq][D], NaN where no row is computed; what a row's logits and values are made of:
    [n_rows][Hq] the sum of |q k| / sqrt(D) at its largest and [n_rows][Hq][D] the sum of weights times |v|; mass float64)."""
    per = shape.Hq // shape.Hkv
    out = np.full(q.shape, np.nan)
    size, spread = np.zeros(q.shape[:2]), np.zeros(q.shape)
    mass = np.zeros((len(length), shape.Hkv, shape.N)) if mass_in is None else mass_in.astype(np.float64)
    for s in range(len(length)):
        n = int(length[s])
        first, c = rows_of(row_start, len(length), len(q), s)
        there = np.zeros(n, dtype=bool)
        for i in range(-(-n // shape.T)):
            there[i * shape.T:(i + 1) * shape.T] = present(shape, pool, off[s, i], bits[s, i])
        for h in range(shape.Hkv):
            kv = np.zeros((2, n, shape.D))
            for i in range(-(-n // shape.T)):
                if there[i * shape.T]:
                    m = min(shape.T, n - i * shape.T)
                    for w in range(2):
                        kv[w, i * shape.T:i * shape.T + m] = Slab(shape, pool, off[s, i], bits[s, i], layer, w, h).values(shape)[:m]
            for j in range(min(c, max_rows)):
                visible = there & (np.arange(n) <= n - c + j)
                for head in range(h * per, (h + 1) * per):
                    x = q[first + j, head].astype(np.float64)
                    if not visible.any():
                        out[first + j, head] = 0
                        continue
                    z = kv[0] @ x / np.sqrt(shape.D)
                    p = np.where(visible, np.exp(z - z[visible].max()), 0)
                    p /= p.sum()
                    out[first + j, head] = p @ kv[1]
                    size[first + j, head] = (np.abs(kv[0]) @ np.abs(x) / np.sqrt(shape.D))[visible].max()
                    spread[first + j, head] = p @ np.abs(kv[1])
                    mass[s, h, :n] += p
    return out, size, spread, mass


def evict(shape, pool, off, bits, length, layers, mass_in, pos_in, keep, sink, recent, seen=None):
    """In place on pool; -> (mass, pos) copies with the kept slots' entries.  layers: (begin, end)."""
    mass, pos = mass_in.copy(), pos_in.copy()
    for li, layer in enumerate(range(*layers)):
        for s in range(len(length)):
            n = int(length[s])
            if n <= keep:
                continue
            for h in range(shape.Hkv):
                m, p = mass_in[li, s, h, :n], pos_in[li, s, h, :n]
                since = (n if seen is None else int(seen[s])) - recent
                rank = sorted(range(n), key=lambda i: (0, 0, i) if p[i] < sink or p[i] >= since else
                              (2, 0, i) if np.isnan(m[i]) else (1, -float(m[i]), i))
                kept = set(rank[:keep])
                holes = [i for i in range(keep) if i not in kept]
                movers = [i for i in range(keep, n) if i in kept]
                for to, at in zip(holes, movers):
                    mass[li, s, h, to], pos[li, s, h, to] = m[at], p[at]
                    a, b = at // shape.T, to // shape.T
                    if not (present(shape, pool, off[s, a], bits[s, a]) and present(shape, pool, off[s, b], bits[s, b])):
                        continue
                    for w in range(2):
                        x = Slab(shape, pool, off[s, a], bits[s, a], layer, w, h)
                        y = Slab(shape, pool, off[s, b], bits[s, b], layer, w, h)
                        if x.b == y.b:
                            y.codes[to % shape.T] = x.codes[at % shape.T]
                            if x.b != 16:
                                y.scale[to % shape.T], y.mn[to % shape.T] = x.scale[at % shape.T], x.mn[at % shape.T]
                        else:
                            y.put(shape, to % shape.T, x.dequantised(shape, at % shape.T))
    return mass, pos
