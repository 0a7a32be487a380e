"""Latent caches, slow and in 64 bits: appending rows to pages, reading them back, attention.  Written from the record format and the
definitions of the operations; shares no code with the library.

A pool is a numpy uint8 array, a page table off [n_seqs][pages] and bits [n_seqs][pages] (0: absent), length [n_seqs]."""
from __future__ import annotations

from typing import NamedTuple

import numpy as np

from .decode import rows_of


class Shape(NamedTuple):
    L: int
    H: int
    Dc: int
    Dr: int
    Dk: int
    Dv: int
    N: int
    T: int
    G: int
    fmt: int = 0


def _param_type(shape):
    return np.dtype(np.float16 if shape.fmt == 3 else np.float32)


def record_bytes(shape, b):
    b = int(b)
    each = 2 * shape.Dr + (2 * shape.Dc if b == 16 else shape.Dc * b // 8 + 2 * shape.Dc // shape.G * _param_type(shape).itemsize)
    return shape.L * shape.T * each


def present(shape, pool, off, b):
    off, b = int(off), int(b)
    return b in (16, 8, 4, 2) and off >= 0 and off % 16 == 0 and off + record_bytes(shape, b) <= pool.size


class Layer:
    """Views of one layer of a record of width b at byte `off` of the pool."""

    def __init__(self, shape, pool, off, b, layer):
        self.shape, self.b = shape, int(b)
        L, T, at = shape.L, shape.T, int(off)
        t = _param_type(shape)

        def section(row_bytes):
            nonlocal at
            mine = pool[at + layer * T * row_bytes:at + (layer + 1) * T * row_bytes].reshape(T, row_bytes)
            at += L * T * row_bytes
            return mine

        self.codes = section(shape.Dc * self.b // 8)
        if self.b != 16:
            self.scale = section(shape.Dc // shape.G * t.itemsize).view(t)
            self.mn = section(shape.Dc // shape.G * t.itemsize).view(t)
        self.rope = section(shape.Dr * 2).view(np.float16)

    def latents(self):
        """fp16 [T][Dc] as a Load gives them: binary32, product and sum rounded separately."""
        if self.b == 16:
            return self.codes.view(np.float16)
        d, per = np.arange(self.shape.Dc), 8 // self.b
        code = ((self.codes[:, d // per].astype(np.int64) >> (d % per * self.b)) & (2 ** self.b - 1)).astype(np.float32)
        g = d // self.shape.G
        with np.errstate(invalid="ignore", over="ignore"):                # (rows that no token has may hold anything)
            return (code * self.scale.astype(np.float32)[:, g] + self.mn.astype(np.float32)[:, g]).astype(np.float16)

    def put(self, row, c, r):
        self.rope[row] = r
        if self.b == 16:
            self.codes[row] = c.view(np.uint8)
            return
        top, t = np.float32(2 ** self.b - 1), _param_type(self.shape)
        g = c.astype(np.float32).reshape(-1, self.shape.G)
        mn = g.min(1) + np.float32(0)
        scale = ((((g.max(1) + np.float32(0)) - mn) / top).astype(t)).astype(np.float32)
        code = np.zeros_like(g)
        some = scale != 0
        code[some] = np.clip(np.rint((g[some] - mn[some, None]) / scale[some, None]), 0, top)
        code = code.reshape(-1).astype(np.uint8).reshape(-1, 8 // self.b)
        packed = np.zeros(len(code), dtype=np.uint8)
        for k in range(8 // self.b):
            packed |= code[:, k] << (k * self.b)
        self.codes[row], self.scale[row], self.mn[row] = packed, scale.astype(t), mn.astype(t)


def _places(shape, pool, off, bits, length, n_rows, row_start):
    """(row, sequence, token, layer-independent page or None) of every row that has a token."""
    for s in range(len(length)):
        first, c = rows_of(row_start, len(length), n_rows, s)
        for j in range(c):
            token = int(length[s]) - c + j
            if token >= 0:
                page = token // shape.T
                yield first + j, s, token, page if present(shape, pool, off[s, page], bits[s, page]) else None


def append(shape, pool, off, bits, length, layer, c, r, row_start=None):
    for row, s, token, page in _places(shape, pool, off, bits, length, len(c), row_start):
        if page is not None:
            Layer(shape, pool, off[s, page], bits[s, page], layer).put(token % shape.T, c[row], r[row])


def read(shape, pool, off, bits, length, layer, c, r, row_start=None):
    """In place on c and r."""
    for row, s, token, page in _places(shape, pool, off, bits, length, len(c), row_start):
        if page is not None:
            at = Layer(shape, pool, off[s, page], bits[s, page], layer)
            c[row], r[row] = at.latents()[token % shape.T], at.rope[token % shape.T]


class Rows(NamedTuple):
    """One layer of a sequence: float64 latents [n][Dc] and position parts [n][Dr], and which tokens' pages are there."""
    c: np.ndarray
    r: np.ndarray
    there: np.ndarray


def sequence(shape, pool, off, bits, n, layer):
    c, r, there = np.zeros((n, shape.Dc)), np.zeros((n, shape.Dr)), np.zeros(n, dtype=bool)
    for i in range(-(-n // shape.T)):
        a, b = i * shape.T, min(n, (i + 1) * shape.T)
        if present(shape, pool, off[i], bits[i]):
            at = Layer(shape, pool, off[i], bits[i], layer)
            c[a:b], r[a:b], there[a:b] = at.latents()[:b - a], at.rope[:b - a], True
    return Rows(c, r, there)


def attend(shape, pool, off, bits, length, layer, q, w, row_start=None, max_rows=None):
    """-> (out float64 [n_rows][H][Dv], NaN where no row is computed; what its error is made of, by element of out:
    logits [n_rows][H], the largest sums of |products| of a row's logits in the two forms, absorbed and expanded;
    spread, the weighted |values|; spread_c, the weighted |latents| times |w|)."""
    H, Dk, Dr = shape.H, shape.Dk, shape.Dr
    out = np.full((len(q), H, shape.Dv), np.nan)
    sizes = {k: np.zeros((len(q), H)) for k in ("absorbed", "absorbed_all", "expanded", "expanded_all")}
    spread, spread_c = np.zeros_like(out), np.zeros_like(out)
    w = w.astype(np.float64)
    for s in range(len(length)):
        n = int(length[s])
        first, c = rows_of(row_start, len(length), len(q), s)
        if c == 0:
            continue
        x = sequence(shape, pool, off[s], bits[s], n, layer)
        for h in range(H):
            wk, wv = w[:, h, :Dk], w[:, h, Dk:]
            k, v = x.c @ wk, x.c @ wv
            for j in range(c if max_rows is None else min(c, max_rows)):
                a = q[first + j, h].astype(np.float64)
                seen = x.there & (np.arange(n) <= n - c + j)
                if not seen.any():
                    out[first + j, h] = 0
                    continue
                z = (k @ a[:Dk] + x.r @ a[Dk:]) / np.sqrt(Dk + Dr)
                p = np.where(seen, np.exp(z - z[seen].max()), 0)
                p /= p.sum()
                out[first + j, h] = p @ v
                rope = np.abs(x.r) @ np.abs(a[Dk:])
                wide = np.abs(x.c) @ (np.abs(wk) @ np.abs(a[:Dk]))
                for name, size in (("absorbed", np.abs(x.c) @ np.abs(wk @ a[:Dk])), ("absorbed_all", wide + rope),
                                   ("expanded", np.abs(k) @ np.abs(a[:Dk])), ("expanded_all", wide + rope)):
                    sizes[name][first + j, h] = size[seen].max() / np.sqrt(Dk + Dr)
                spread[first + j, h] = p @ np.abs(v)
                spread_c[first + j, h] = (p @ np.abs(x.c)) @ np.abs(wv)
    return out, sizes, spread, spread_c
