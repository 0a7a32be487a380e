"""Paged sequences for the tests of decoding: records in a pool in any order with gaps between them, absent pages, rows behind a
sequence's end that hold NaN."""
import numpy as np
import torch

import oracle
import oracle.decode
import paper_2403_11805_amd as kvs
from paper_2403_11805_amd import synth


class Paged:
    """Sequences of `lens` tokens with pages of widths drawn from `widths` (0: absent).  geom: (L, Hkv, Hq, D, N, T, G)."""

    def __init__(self, geom, lens, widths, seed, fmt=0, spare_stride=0, scale=1.0):
        self.rng = np.random.RandomState(seed)
        self.os = oracle.Shape(*geom, fmt)
        self.ks = kvs.Shape(*geom, fmt)
        s, n, pages = self.os, len(lens), self.os.n_chunks
        self.len = np.array(lens, dtype=np.int32)
        self.bits = np.zeros((n, pages + spare_stride), dtype=np.uint8)
        self.off = self.rng.randint(0, 1 << 60, (n, pages + spare_stride)).astype(np.int64)      # absent pages lie anywhere
        self.bits[:, :pages] = self.rng.choice(widths, (n, pages))
        sizes = {w: (oracle.record_bytes(s, w) if w in (16, 8, 4, 2) else 0) for w in set(self.bits.reshape(-1).tolist())}
        order = [(i, j) for i in range(n) for j in range(pages)]
        self.rng.shuffle(order)
        at = 0
        for i, j in order:
            if sizes[self.bits[i, j]]:
                at += 16 * self.rng.randint(0, 4)
                self.off[i, j] = at
                at += sizes[self.bits[i, j]]
        self.pool = np.full(at, 0xff, dtype=np.uint8)                                            # every gap is NaN
        self.kv = []
        for i in range(n):
            kv = (synth.make_kv(synth.Geometry(*geom), seed * 100 + i).float() * scale).half().numpy()
            self.kv.append(kv)
            for j in range(pages):
                w = int(self.bits[i, j])
                if sizes[w]:
                    one = oracle.Shape(s.L, s.Hkv, s.Hq, s.D, s.T, s.T, s.G, fmt)
                    off = np.array([0, sizes[w]], dtype=np.uint64)
                    part = np.ascontiguousarray(kv[:, :, :, j * s.T:(j + 1) * s.T])
                    self.pool[self.off[i, j]:self.off[i, j] + sizes[w]] = \
                        oracle.compress_chunks(one, part, np.array([w], dtype=np.uint8), off)
                    for token in range(max(int(lens[i]), j * s.T), (j + 1) * s.T):
                        self._nothing(i, j, token - j * s.T)

    def _nothing(self, i, j, row):
        for layer in range(self.os.L):
            for w in range(2):
                for h in range(self.os.Hkv):
                    x = oracle.decode.Slab(self.os, self.pool, self.off[i, j], self.bits[i, j], layer, w, h)
                    x.codes[row] = 0xff
                    if x.b != 16:
                        x.scale[row], x.mn[row] = np.nan, np.nan

    def table(self):
        return self.off, self.bits, self.len

    def halves(self, *shape, scale=1.0):
        return (self.rng.standard_normal(shape) * scale).astype(np.float16)

    def book(self, layers=None):
        """mass, pos [layers][n_seqs][Hkv][N]: weights with many ties, positions of tokens that were never moved."""
        shape = (len(self.len), self.os.Hkv, self.os.N)
        shape = shape if layers is None else (layers,) + shape
        mass = (self.rng.randint(0, 12, shape) / 8).astype(np.float32)
        return mass, np.broadcast_to(np.arange(self.os.N, dtype=np.int32), shape).copy()

    def device(self):
        """-> (Pages on the GPU, its pool tensor)."""
        put = lambda a: torch.from_numpy(a.copy()).to("cuda")      # noqa: E731
        pool = put(self.pool)
        return kvs.Pages(self.ks, pool, put(self.off), put(self.bits), put(self.len)), pool


def rows(counts, n_rows=None, lead=0):
    """row_start of these counts, with `lead` rows in front of the first sequence."""
    start = lead + np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    return start.astype(np.int32), int(start[-1]) if n_rows is None else n_rows


def attend_bars(paged, q, out, size, spread):
    """How far out may be from its value in 64 bits, by element.  A logit is a sum of D products in binary32 of q and codes, which reach
    a range of their group, twice the largest |k| = K: with the minima every partial sum is below 6 K sum |q| / sqrt(D), and each of the
    D + 8 roundings is half a step, 2^-24.  Weights change by twice a logit's error
    relatively, and each is rounded to fp16 at worst, as is V (half a step each, 2^-11); then the result is rounded.  exp2 and the sums
    add 2^-20 with room to spare."""
    s = paged.os
    biggest = max(float(np.abs(kv.astype(np.float64)).max()) for kv in paged.kv)
    delta = 2.0 ** -24 * (s.D + 8) * 6 * biggest * np.abs(q.astype(np.float64)).sum(-1) / np.sqrt(s.D)
    delta = delta[..., None] + 2.0 ** -20
    return spread * (2 * delta + 2 * 2.0 ** -11) * 1.01 + np.abs(out) * 2.0 ** -11 + 2.0 ** -24, delta
