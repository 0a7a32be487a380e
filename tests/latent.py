"""Paged latent caches for the tests: records in a pool in any order with gaps between them, absent pages, rows behind a sequence's end
that hold NaN."""
import numpy as np
import torch

import oracle.latent as ol
import paper_2403_11805_amd as kvs

from paged import rows  # noqa: F401


def put(a):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).to("cuda")


class Latent:
    """Sequences of `lens` tokens with pages of widths drawn from `widths` (0: absent).  geom: (L, H, Dc, Dr, Dk, Dv, N, T, G)."""

    def __init__(self, geom, lens, widths, seed, fmt=0, spare_stride=0):
        self.rng = np.random.RandomState(seed)
        self.os, self.ks = ol.Shape(*geom, fmt), kvs.LatentShape(*geom, fmt)
        s, n, pages = self.os, len(lens), geom[6] // geom[7]
        self.len = np.array(lens, dtype=np.int32)
        self.bits = np.zeros((n, pages + spare_stride), dtype=np.uint8)
        self.off = self.rng.randint(0, 1 << 60, (n, pages + spare_stride)).astype(np.int64)      # absent pages lie anywhere
        self.bits[:, :pages] = self.rng.choice(widths, (n, pages))
        order = [(i, j) for i in range(n) for j in range(pages) if self.bits[i, j] in (16, 8, 4, 2)]
        self.rng.shuffle(order)
        at = 0
        for i, j in order:
            at += 16 * self.rng.randint(0, 4)
            self.off[i, j] = at
            at += ol.record_bytes(s, self.bits[i, j])
        self.pool = np.full(max(at, 16), 0xff, dtype=np.uint8)                                   # every gap is NaN
        mult = np.where(self.rng.rand(s.Dc) < 0.02, 4.0, 1.0)
        for i, j in order:
            for layer in range(s.L):
                x = ol.Layer(s, self.pool, self.off[i, j], self.bits[i, j], layer)
                for row in range(max(0, min(s.T, int(lens[i]) - j * s.T))):
                    x.put(row, (self.rng.standard_normal(s.Dc) * mult).astype(np.float16), self.halves(s.Dr))

    def table(self):
        return self.off, self.bits, self.len

    def halves(self, *shape, scale=1.0):
        return (self.rng.standard_normal(shape) * scale).astype(np.float16)

    def weights(self):
        s = self.os
        return self.halves(s.Dc, s.H, s.Dk + s.Dv, scale=s.Dc ** -0.5)

    def queries(self, n, scale=2.0):
        return self.halves(n, self.os.H, self.os.Dk + self.os.Dr, scale=scale)

    def at(self, s, token, layer):
        """The layer's view of the page that holds a token, and its row there."""
        i = token // self.os.T
        return ol.Layer(self.os, self.pool, self.off[s, i], self.bits[s, i], layer), token % self.os.T

    def device(self):
        """-> (LatentPages on the GPU, its pool tensor)."""
        pool = put(self.pool)
        return kvs.LatentPages(self.ks, pool, put(self.off), put(self.bits), put(self.len)), pool


def attend(p, layer, q, w, row_start=None, max_rows=1, expanded=False, n_tokens=None):
    """The library's output as numpy; what it does not write is 7."""
    pages, pool = p.device()
    if expanded:
        n_tokens = max(1, int(p.len.sum())) if n_tokens is None else n_tokens
        need = kvs.kv_latent_prompts_workspace_bytes(p.ks, len(p.len), n_tokens)
    else:
        need = kvs.kv_latent_attend_workspace_bytes(p.ks, len(p.len), max_rows)
    ws = torch.full((need,), 0xff, dtype=torch.uint8, device="cuda")
    out = torch.full((len(q), p.os.H, p.os.Dv), 7.0, dtype=torch.float16, device="cuda")
    if expanded:
        kvs.kv_latent_attend_prompts(pages, layer, put(q), put(w), ws, out, n_tokens, row_start=put(row_start))
    else:
        kvs.kv_latent_attend_tokens(pages, layer, put(q), put(w), ws, out, row_start=put(row_start), max_rows=max_rows)
    torch.cuda.synchronize()
    assert np.array_equal(pool.cpu().numpy(), p.pool), "attention wrote to the pool"
    return out.cpu().numpy()


def bars(p, out, sizes, spread, spread_c, expanded):
    """How far an output may be from its value in 64 bits, by element.  What is rounded to fp16 on the way is off by half a step, 2^-11:
      the logits' left factor - absorbed, a query in the latents' space, expanded, a key - so that a logit is off by 2^-11 of the sum of its
        |products| (`sizes`), and by 2^-24 of the sum of all |products| behind it for each of the Dc + Dk + Dr additions, and 16 more;
      the probabilities, and (expanded) the values; the result.
    Weights change by twice a logit's error relatively.  Probabilities that are subnormal halves are off by 2^-25 where the largest is at
    least 2^7: n 2^-32 of the largest value.  Sums over tokens and over latents are of binary32: 2^-24 for each addition, of the sum of the
    |terms|; the joined latents keep 22 bits; exp2 and the joining add 2^-20 with room to spare."""
    s, form = p.os, "expanded" if expanded else "absorbed"
    n = int(p.len.max())
    logit = 2.0 ** -11 * sizes[form] + 2.0 ** -24 * (s.Dc + s.Dk + s.Dr + 16) * sizes[form + "_all"] + 2.0 ** -20
    weights = 2 * logit[..., None] + 2.0 ** -11 * (2 if expanded else 1) + n * 2.0 ** -32
    return 1.02 * (spread * weights + spread_c * (2.0 ** -24 * (n + s.Dc + 64) + 2.0 ** -21)) + np.abs(out) * 2.0 ** -11 + 2.0 ** -24


def check_attend(p, layer, q, w, row_start=None, max_rows=1, expanded=False):
    got = attend(p, layer, q, w, row_start, max_rows, expanded)
    want, *made = ol.attend(p.os, p.pool, *p.table(), layer, q, w, row_start, None if expanded else max_rows)
    computed = ~np.isnan(want)
    assert np.all(got[~computed] == 7), "a row that belongs to no sequence was written"
    bar = bars(p, want, *made, expanded)
    off = np.abs(got.astype(np.float64) - want)
    assert np.all(np.isfinite(got)) and np.all(off[computed] <= bar[computed]), float(np.nanmax(off / bar))
    return got
