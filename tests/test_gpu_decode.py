"""GPU parity of decoding on packed records (append, attention over pages, eviction) against the oracle in 64 bits.

Bars: appended and evicted bytes are equal; attention is within the roundings that tests/paged.py counts."""
import numpy as np
import pytest
import torch

import oracle.decode as od
import paper_2403_11805_amd as kvs

from paged import Paged, attend_bars, rows

pytestmark = pytest.mark.gpu

MIXED = (16, 8, 4, 2)


def put(a):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).to("cuda")


def attend(p, layer, q, row_start=None, max_rows=1, mass_in=None, with_mass=False):
    """-> (out, mass) of the library as numpy; whatever it does not write is 7."""
    pages, pool = p.device()
    ws = torch.full((kvs.kv_attend_workspace_bytes(p.ks, len(p.len), max_rows, with_mass),), 0xff, dtype=torch.uint8, device="cuda")
    out = torch.full(q.shape, 7.0, dtype=torch.float16, device="cuda")
    mass = torch.full((len(p.len), p.ks.n_kv_heads, p.ks.n_tokens), 7.0, device="cuda") if with_mass else None
    kvs.kv_attend_tokens(pages, layer, put(q), ws, out, row_start=put(row_start), max_rows=max_rows, mass_in=put(mass_in), mass=mass)
    torch.cuda.synchronize()
    assert np.array_equal(pool.cpu().numpy(), p.pool), "attention wrote to the pool"
    return out.cpu().numpy(), None if mass is None else mass.cpu().numpy()


def check_attend(p, layer, q, row_start=None, max_rows=1, mass_in=None, with_mass=False):
    got, mass = attend(p, layer, q, row_start, max_rows, mass_in, with_mass)
    want, size, spread, want_mass = od.attend(p.os, p.pool, *p.table(), layer, q, row_start, max_rows, mass_in)
    bar, delta = attend_bars(p, q, want, size, spread)
    computed = ~np.isnan(want)
    assert np.all(got[~computed] == 7), "a row that belongs to no sequence was written"
    off = np.abs(got.astype(np.float64) - want)
    assert np.all(np.isfinite(got)) and np.all(off[computed] <= bar[computed]), float(np.nanmax(off / bar))
    if with_mass:
        base = 0 if mass_in is None else mass_in
        for s, n in enumerate(p.len):
            _, c = od.rows_of(row_start, len(p.len), len(q), s)
            untouched = mass[s, :, n:] if c else mass[s]
            assert np.all(untouched == 7)
            if c:
                w = want_mass[s, :, :n]
                np.testing.assert_allclose(mass[s, :, :n], w, rtol=0, atol=0 if n == 0 else float(
                    (2 * delta.max() + 2.0 ** -20) * (w - (0 if mass_in is None else base[s, :, :n])).max() + 2.0 ** -23 * np.abs(w).max()))


@pytest.mark.parametrize("D,G", [(64, 64), (128, 64), (128, 128), (256, 64), (256, 128), (256, 256)])
@pytest.mark.parametrize("widths", [(16,), (8,), (4,), (2,)])
@pytest.mark.parametrize("fmt", [0, 3])
def test_attend_one_width(D, G, widths, fmt):
    p = Paged((2, 2, 6, D, 96, 32, G), [96, 1, 33, 95], widths, 3, fmt)
    check_attend(p, 1, p.halves(4, 6, D, scale=2.0), with_mass=True)


@pytest.mark.parametrize("geom,lens,counts,widths", [
    ((1, 1, 1, 64, 16, 16, 64), [1], [1], (16,)),                                    # one token, one head
    ((2, 3, 3, 128, 160, 16, 64), [160, 17, 16, 15, 0], [1, 1, 1, 1, 1], MIXED),     # pages of one tile: widths change inside a unit
    ((1, 2, 8, 128, 192, 48, 128), [192, 47, 49, 100], [3, 0, 4, 1], MIXED),         # pages of three tiles
    ((1, 1, 7, 256, 128, 64, 128), [128, 2, 77], [5, 2, 4], MIXED + (0,)),           # 35 query rows, absent pages
    ((3, 2, 4, 64, 1024, 16, 64), [1024, 999, 3], [2, 1, 3], MIXED + (0, 0)),        # long: divided in shares
    ((1, 1, 32, 64, 128, 16, 64), [128, 100], [16, 7], MIXED),                       # 512 query rows
    ((1, 2, 4, 64, 64, 16, 64), [2, 5], [3, 8], (8, 16)),                            # more new rows than tokens
    ((1, 1, 64, 64, 96, 16, 64), [90], [16], MIXED),                                 # 1024 query rows, the most
])
@pytest.mark.parametrize("with_mass", [False, True])
def test_attend_rows_and_pages(geom, lens, counts, widths, with_mass):
    p = Paged(geom, lens, widths, 5, spare_stride=1)
    start, n_rows = rows(counts, lead=2)
    q = p.halves(n_rows + 3, geom[2], geom[3], scale=1.5)
    mass_in = p.book()[0] if with_mass else None
    check_attend(p, geom[0] - 1, q, start, max(counts + [1]), mass_in, with_mass)


def test_attend_without_any_page():
    p = Paged((1, 2, 4, 64, 64, 16, 64), [64, 30], (0,), 1)
    p.pool = np.zeros(4096, dtype=np.uint8)
    got, mass = attend(p, 0, p.halves(2, 4, 64), with_mass=True)
    assert not got.any() and not mass[0].any() and not mass[1, :, :30].any()


BAD = ((8, 16), (-16, 16), (1 << 62, 4), (0, 3), (0, 255), (0, 1), (0, 18))


def spoil(p, s=0):
    """The first pages of a sequence get offsets that are odd, reach past the pool or lie far away, and widths of no format."""
    for j, (off, b) in enumerate(BAD + ((p.pool.size - 16, 16), (p.pool.size, 2), (p.pool.size + 16, 2))):
        p.off[s, j], p.bits[s, j] = off, b


def test_attend_bad_pages_are_absent():
    p = Paged((1, 1, 2, 128, 192, 16, 64), [192], (16,), 9)
    spoil(p)
    check_attend(p, 0, p.halves(1, 2, 128), with_mass=True)


def test_append_to_bad_pages_writes_nothing():
    p = Paged((1, 1, 2, 128, 192, 16, 64), [192], (16,), 9)
    spoil(p)
    k, v = p.halves(192, 1, 128), p.halves(192, 1, 128)
    start, _ = rows([192])
    pages, pool = p.device()
    kvs.kv_append_tokens(pages, 0, put(k), put(v), row_start=put(start))
    want = p.pool.copy()
    od.append(p.os, want, *p.table(), 0, k, v, start)
    assert np.array_equal(pool.cpu().numpy(), want) and not np.array_equal(want, p.pool)


def test_evict_does_not_move_rows_of_bad_pages():
    p = Paged((1, 1, 2, 128, 384, 16, 64), [384, 380], (16,), 9)
    spoil(p)
    mass, pos = p.book(1)
    for keep in (100, 200):
        pool, m, q = run_evict(p, (0, 1), mass, pos, keep, 0, 40)
        want = p.pool.copy()
        wm, wp = od.evict(p.os, want, *p.table(), (0, 1), mass, pos, keep, 0, 40)
        assert np.array_equal(pool, want) and np.array_equal(m[..., :keep], wm[..., :keep]) and np.array_equal(q[..., :keep], wp[..., :keep])


@pytest.mark.parametrize("hot", [0, 17, 300, 511])
@pytest.mark.parametrize("D", [64, 256])
def test_attend_one_key_far_above_the_others(hot, D):
    """Every logit before it lies further below than fp16 reaches; those behind it must not be lost where they tie."""
    p = Paged((1, 1, 2, D, 512, 16, 64), [512], (16,), 2, scale=0.05)
    od.Slab(p.os, p.pool, p.off[0, hot // 16], 16, 0, 0, 0).put(p.os, hot % 16, np.full(D, 20, dtype=np.float16))
    p.kv[0][0, 0, 0, hot] = 20
    check_attend(p, 0, np.full((1, 2, D), 3.0, dtype=np.float16), with_mass=True)


@pytest.mark.parametrize("fmt", [0, 3])
@pytest.mark.parametrize("width,apart", [(8, 5), (4, 8), (2, 10)])
def test_attend_logits_keep_the_bits_of_small_products(width, apart, fmt):
    """q is 0 but for two dimensions that are summed by different matrix instructions and lie 2^apart apart, so that every sum of q * code
    fits 24 bits and is exact in binary32: 1025 * (2^apart + 1) * (2^width - 1) < 2^24.  What is left to round: scale and minimum (2, of
    at most K sum |q|), the factor to base 2 (2), the logit it gives (1), its difference to the reference (2, twice the size): 8 halves of
    a step, 2^-24, counted as 12.  At width 8 the sum takes all 24 bits below a range (twice K), where each of the two instructions may
    chop twice at 2^-23 of it: 16 more.  A weight is off by that in its own logit and in the sum's, 2 ln 2 times it
    relatively; exp2, the sums over 64 tokens and the division add less than 2^-20."""
    p = Paged((1, 2, 6, 64, 64, 16, 64), [64, 50], (width,), 12, fmt)
    biggest = max(float(np.abs(kv.astype(np.float64)).max()) for kv in p.kv)
    top = 2.0 ** np.floor(np.log2(16 * 8 / (1.45 * biggest)))                # logits to base 2 up to 16
    q = np.zeros((2, 6, 64), dtype=np.float16)
    q[..., 8] = top * 1025 / 1024
    q[..., 0] = q[..., 8].astype(np.float64) * 2.0 ** -apart
    q[1::2] *= -1
    _, mass = attend(p, 0, q, with_mass=True)
    want = od.attend(p.os, p.pool, *p.table(), 0, q, None, 1, None)[3]
    delta = (12 + (16 if width == 8 else 0)) * 2.0 ** -24 * biggest * np.abs(q.astype(np.float64)).sum(-1).max() / 8 * np.log2(np.e)
    for s, n in enumerate(p.len):
        np.testing.assert_allclose(mass[s, :, :n], want[s, :, :n], rtol=2 * np.log(2) * delta + 2.0 ** -20, atol=0)


def many(D, n_seqs, N, seed, lens=None):
    rng = np.random.RandomState(seed)
    p = Paged((1, 2, 4, D, N, 16, 64), rng.randint(0, N + 1, n_seqs) if lens is None else lens, (16, 16, 16, 8, 0), seed)
    return p, rows(rng.randint(0, 3, n_seqs))


@pytest.mark.parametrize("D,n_seqs,N", [(64, 65, 64), (128, 130, 48), (64, 200, 1024), (256, 70, 512)])
def test_attend_many_sequences(D, n_seqs, N):
    """More sequences than a wavefront has lanes, many of them empty or without rows; the last ones of each list get the longest work
    in front of them.  200 sequences of up to 32 units are more than the workgroups take in whole steps, the others less."""
    p, (start, n_rows) = many(D, n_seqs, N, 31)
    check_attend(p, 0, p.halves(n_rows + 1, 4, D), start, 2, None, True)


def test_attend_one_long_sequence_among_many_short_ones():
    p, (start, n_rows) = many(64, 100, 2048, 32, [1] * 99 + [2048])
    check_attend(p, 0, p.halves(n_rows, 4, 64), start, 2, None, True)


def test_attend_rows_above_max_rows_are_left():
    p = Paged((1, 2, 8, 64, 64, 16, 64), [60, 20], (16,), 33)
    start, n_rows = rows([5, 1])
    q = p.halves(n_rows, 8, 64)
    check_attend(p, 0, q, start, 3, None, True)
    got, _ = attend(p, 0, q, start, 3)
    assert np.all(got[3:5] == 7) and not np.any(got[[0, 1, 2, 5]] == 7)


@pytest.mark.parametrize("what", [np.nan, np.inf, -np.inf])
def test_keys_of_later_tokens_do_not_matter(what):
    """A row's logits behind its own token are left out whatever they are."""
    p = Paged((1, 1, 2, 128, 64, 16, 128), [40], (16,), 34)
    start, n_rows = rows([4])
    q = p.halves(n_rows, 2, 128)
    want, _ = attend(p, 0, q, start, 4)
    od.Slab(p.os, p.pool, p.off[0, 2], 16, 0, 0, 0).put(p.os, 39 - 32, np.full(128, what, dtype=np.float16))
    got, _ = attend(p, 0, q, start, 4)
    assert np.array_equal(got[:3], want[:3])


@pytest.mark.parametrize("D,G", [(64, 64), (128, 64), (128, 128), (256, 64), (256, 256)])
@pytest.mark.parametrize("width", MIXED)
@pytest.mark.parametrize("fmt", [0, 3])
@pytest.mark.parametrize("n,what", [(40, np.nan), (48, np.inf), (33, -np.inf)])
def test_values_of_later_tokens_do_not_matter(D, G, width, fmt, n, what):
    """V of the two newest tokens is not finite in a few dimensions: the rows in front of them and all weights stay as they were, the others are NaN."""
    p = Paged((1, 2, 4, D, 64, 16, G), [n, 20], (width,), 36, fmt)
    start, n_rows = rows([4, 1])
    q = p.halves(n_rows, 4, D)
    want, weights = attend(p, 0, q, start, 4, None, True)
    for token in (n - 2, n - 1):
        x = od.Slab(p.os, p.pool, p.off[0, token // 16], width, 0, 1, 1)
        if width == 16:
            x.codes[token % 16].view(np.float16)[[3, D - 1]] = what
        else:
            x.scale[token % 16, 0] = what
    got, mass = attend(p, 0, q, start, 4, None, True)
    assert np.array_equal(got[[0, 1, 4]], want[[0, 1, 4]]) and np.array_equal(mass, weights)
    assert np.array_equal(got[2:4, :2], want[2:4, :2]) and np.isnan(got[2:4, 2:]).all()


def test_pages_past_four_gib():
    """The same sequences in a pool whose records lie behind byte 2^32: every call does the same there."""
    at = (1 << 32) + 4096
    p = Paged((2, 2, 4, 128, 96, 16, 64), [96, 50], MIXED, 35)
    pages, near = p.device()
    pool = torch.zeros(at + p.pool.size, dtype=torch.uint8, device="cuda")
    pool[at:] = near
    far = kvs.Pages(p.ks, pool, pages.off + at, pages.bits, pages.length)
    k, v, q = (put(p.halves(2, h, 128)) for h in (2, 2, 4))
    mass, pos = (put(a) for a in p.book(1))
    results = []
    for pg in (pages, far):
        ws = torch.zeros(kvs.kv_attend_workspace_bytes(p.ks, 2, 1, True), dtype=torch.uint8, device="cuda")
        ws2 = torch.zeros(kvs.kv_evict_workspace_bytes(p.ks, 2, 1, 40), dtype=torch.uint8, device="cuda")
        m, o = mass.clone(), pos.clone()
        out = torch.zeros((2, 4, 128), dtype=torch.float16, device="cuda")
        kvs.kv_append_tokens(pg, 1, k, v, mass=m[0], pos=o[0])
        kvs.kv_attend_tokens(pg, 1, q, ws, out, mass_in=m[0], mass=m[0])
        kvs.kv_evict_tokens(pg, 1, 2, m, o, 40, 2, 8, ws2, m, o)
        results.append((out, m, o))
    for a, b in zip(*results):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    assert bool(results[0][0].any()) and torch.equal(pool[at:], near) and not bool(pool[:at].any())


def test_attend_reads_rows_with_a_stride():
    p = Paged((2, 2, 4, 128, 64, 16, 128), [64, 20], MIXED, 6)
    qkv = torch.from_numpy(p.halves(2, 4 + 2 * 2, 128)).cuda()
    pages, _ = p.device()
    ws = torch.empty(kvs.kv_attend_workspace_bytes(p.ks, 2), dtype=torch.uint8, device="cuda")
    out, same = torch.empty((2, 4, 128), dtype=torch.float16, device="cuda"), torch.empty((2, 4, 128), dtype=torch.float16, device="cuda")
    kvs.kv_attend_tokens(pages, 1, qkv[:, :4], ws, out)
    kvs.kv_attend_tokens(pages, 1, qkv[:, :4].contiguous(), ws, same)
    assert torch.equal(out, same)


def test_attend_mass_accumulates_in_place():
    p = Paged((1, 2, 4, 64, 256, 16, 64), [256, 77], MIXED, 8)
    pages, _ = p.device()
    q = put(p.halves(2, 4, 64, scale=2.0))
    ws = torch.empty(kvs.kv_attend_workspace_bytes(p.ks, 2, 1, True), dtype=torch.uint8, device="cuda")
    out = torch.empty((2, 4, 64), dtype=torch.float16, device="cuda")
    once, twice = torch.zeros((2, 2, 256), device="cuda"), torch.zeros((2, 2, 256), device="cuda")
    kvs.kv_attend_tokens(pages, 0, q, ws, out, mass=once)
    for _ in range(2):
        kvs.kv_attend_tokens(pages, 0, q, ws, out, mass_in=twice, mass=twice)
    assert torch.equal(once + once, twice)
    total = once.sum(-1).cpu().numpy()                     # two query heads a kv head, each with weights that add up to one
    np.testing.assert_allclose(total, 2.0, rtol=256 * 2.0 ** -23)


@pytest.mark.parametrize("geom,fmt", [((2, 3, 3, 64, 64, 16, 64), 0), ((1, 1, 1, 64, 48, 16, 64), 3), ((2, 2, 4, 128, 96, 32, 64), 3),
                                      ((1, 2, 2, 128, 96, 48, 128), 0), ((1, 1, 8, 256, 64, 16, 64), 0), ((2, 1, 1, 256, 64, 16, 256), 3)])
@pytest.mark.parametrize("counts", [None, [4, 0, 31, 1], [2, 40, 0, 0]])
def test_append(geom, fmt, counts):
    lens = [geom[4], 5, 33, 17]
    p = Paged(geom, lens, MIXED + (0,), 4, fmt)
    start, n_rows = (None, 4) if counts is None else rows(counts, lead=1)
    k, v = p.halves(n_rows + (0 if counts is None else 2), geom[1], geom[3]), None
    v = p.halves(*k.shape)
    k[0, 0] = 1.0                                          # a group without range
    v[-1, -1, :64] = -0.0
    mass, pos = p.book()
    seen = np.array([100, 5, 1000, 17], dtype=np.int32)
    pages, pool = p.device()
    dm, dp = put(mass), put(pos)
    kvs.kv_append_tokens(pages, geom[0] - 1, put(k), put(v), row_start=put(start), seen=put(seen), mass=dm, pos=dp)
    want = p.pool.copy()
    od.append(p.os, want, *p.table(), geom[0] - 1, k, v, start, seen, mass, pos)
    assert np.array_equal(pool.cpu().numpy(), want)
    assert np.array_equal(dm.cpu().numpy(), mass) and np.array_equal(dp.cpu().numpy(), pos)


def test_append_of_many_sequences_and_rows():
    """More than 64 and more than 4096 sequences (the row's sequence takes two and three steps to find), and a prompt of many rows."""
    for n in (65, 4100):
        p = Paged((1, 1, 1, 64, 16, 16, 64), [3] * n, (16,), 11)
        counts = [(i * 5) % 3 for i in range(n)]
        start, n_rows = rows(counts)
        k, v = p.halves(n_rows, 1, 64), p.halves(n_rows, 1, 64)
        pages, pool = p.device()
        kvs.kv_append_tokens(pages, 0, put(k), put(v), row_start=put(start))
        want = p.pool.copy()
        od.append(p.os, want, *p.table(), 0, k, v, start)
        assert np.array_equal(pool.cpu().numpy(), want)
    p = Paged((1, 4, 4, 128, 1024, 16, 64), [1000, 1024], MIXED, 12)
    start, n_rows = rows([900, 1024])
    k, v = p.halves(n_rows, 4, 128), p.halves(n_rows, 4, 128)
    pages, pool = p.device()
    kvs.kv_append_tokens(pages, 0, put(k), put(v), row_start=put(start))
    want = p.pool.copy()
    od.append(p.os, want, *p.table(), 0, k, v, start)
    assert np.array_equal(pool.cpu().numpy(), want)


def run_evict(p, layers, mass, pos, keep, sink, recent, seen=None, in_place=False):
    pages, pool = p.device()
    need = kvs.kv_evict_workspace_bytes(p.ks, len(p.len), layers[1] - layers[0], keep)
    ws = torch.full((need,), 0xff, dtype=torch.uint8, device="cuda")
    mi, pi = put(mass), put(pos)
    mo, po = (mi, pi) if in_place else (torch.full_like(mi, 7.0), torch.full_like(pi, 7))
    kvs.kv_evict_tokens(pages, *layers, mi, pi, keep, sink, recent, ws, mo, po, seen=put(seen))
    torch.cuda.synchronize()
    return pool.cpu().numpy(), mo.cpu().numpy(), po.cpu().numpy()


@pytest.mark.parametrize("geom,lens,widths,keep,sink,recent", [
    ((1, 1, 1, 64, 32, 16, 64), [2], (16,), 1, 0, 0),
    ((2, 2, 2, 64, 64, 16, 64), [64, 10, 33, 0], (16,), 20, 2, 5),
    ((2, 2, 4, 128, 96, 32, 64), [96, 50], (16,), 49, 0, 49),
    ((1, 3, 3, 128, 96, 48, 128), [96, 90, 1], (8,), 31, 4, 8),
    ((2, 1, 8, 256, 128, 16, 64), [128, 127], MIXED, 60, 4, 10),           # rows change their width
    ((1, 2, 2, 64, 1088, 16, 64), [1088, 1025], MIXED + (0,), 300, 4, 64),  # more slots than threads, absent pages
    ((1, 1, 1, 64, 64, 16, 64), [64, 64], (4,), 64, 10, 54),               # nothing to do
    ((1, 1, 1, 64, 64, 16, 64), [64], (2,), 1000, 0, 0),                   # a budget beyond the capacity
])
@pytest.mark.parametrize("fmt", [0, 3])
@pytest.mark.parametrize("in_place", [False, True])
def test_evict(geom, lens, widths, keep, sink, recent, fmt, in_place):
    p = Paged(geom, lens, widths, 14, fmt)
    layers = (geom[0] - 1, geom[0])
    mass, pos = p.book(1)
    mass[..., ::7] = 0.0
    mass[..., 1::7] = -0.0
    if geom[4] > 50:
        mass[0, 0, 0, 5], mass[0, 0, 0, 6], mass[0, 0, 0, 40] = np.nan, np.inf, -np.inf
    pool, m, q = run_evict(p, layers, mass, pos, keep, sink, recent, in_place=in_place)
    want = p.pool.copy()
    wm, wp = od.evict(p.os, want, *p.table(), layers, mass, pos, keep, sink, recent)
    assert np.array_equal(pool, want)
    for s, n in enumerate(lens):
        c = min(n, keep)
        assert np.array_equal(m[0, s, :, :c], wm[0, s, :, :c], equal_nan=True) and np.array_equal(q[0, s, :, :c], wp[0, s, :, :c])
        if not in_place:
            assert np.all(m[0, s, :, c:] == 7) and np.all(q[0, s, :, c:] == 7)
        else:
            assert np.array_equal(m[0, s, :, c:], mass[0, s, :, c:], equal_nan=True)


@pytest.mark.parametrize("N,lens,keep,sink,recent", [(4112, [4112, 4100], 1500, 4, 200), (8192, [8192, 70], 8000, 0, 0),
                                                     (12304, [12304, 8200], 5000, 0, 100), (32784, [32784, 32769], 9000, 16, 1000)])
@pytest.mark.parametrize("kind", ["ties", "all equal", "distinct"])
def test_evict_of_long_sequences(N, lens, keep, sink, recent, kind):
    """Ranges of slots that take a lane more than 4, 8 and 32 keys."""
    p = Paged((1, 1, 1, 64, N, 16, 64), lens, (16,), 17)
    mass, pos = p.book(1)
    if kind == "all equal":
        mass[:] = 0.25
    elif kind == "distinct":
        mass = p.rng.permutation(mass.size).reshape(mass.shape).astype(np.float32) - 1000
    pool, m, q = run_evict(p, (0, 1), mass, pos, keep, sink, recent)
    want = p.pool.copy()
    wm, wp = od.evict(p.os, want, *p.table(), (0, 1), mass, pos, keep, sink, recent)
    assert np.array_equal(pool, want)
    for s, n in enumerate(lens):
        c = min(n, keep)
        assert np.array_equal(m[0, s, :, :c], wm[0, s, :, :c]) and np.array_equal(q[0, s, :, :c], wp[0, s, :, :c])


def test_evict_again_and_again():
    """Two evictions in a row with other weights, positions carried along, all layers: the newest tokens stay by position although
    they lie anywhere."""
    p = Paged((2, 2, 2, 64, 128, 16, 64), [128, 100], (16,), 15)
    mass, pos = p.book(2)
    seen = np.array([500, 100], dtype=np.int32)
    pos = pos + (seen - p.len)[None, :, None, None].astype(np.int32)
    pool1, m1, p1 = run_evict(p, (0, 2), mass, pos, 70, 4, 20, seen, True)
    w = p.pool.copy()
    wm, wp = od.evict(p.os, w, *p.table(), (0, 2), mass, pos, 70, 4, 20, seen)
    assert np.array_equal(pool1, w) and np.array_equal(p1[..., :70], wp[..., :70])
    p.pool, p.len = pool1, np.array([70, 70], dtype=np.int32)
    m2 = (m1 + p.book(2)[0]).astype(np.float32)
    pool2, m3, p3 = run_evict(p, (0, 2), m2, p1, 31, 0, 20, seen, True)
    wm, wp = od.evict(p.os, w, *p.table(), (0, 2), m2, p1, 31, 0, 20, seen)
    assert np.array_equal(pool2, w) and np.array_equal(p3[..., :31], wp[..., :31]) and np.array_equal(m3[..., :31], wm[..., :31])
    assert all(set(range(480, 500)) <= set(p3[layer, 0, h, :31].tolist()) for layer in range(2) for h in range(2))


def test_decode_steps_captured_and_replayed():
    """Append, attention with weights and eviction as one graph on a stream of its own, replayed with other lengths, rows and
    weights: every replay equals the same calls made eagerly."""
    p = Paged((2, 2, 4, 128, 160, 32, 64), [100, 41, 160], MIXED, 21)
    pages, pool = p.device()
    k, v, q = (put(p.halves(3, h, 128)) for h in (2, 2, 4))
    book = (2, 3, 2, 160)
    mass, pos = torch.rand(book, device="cuda"), torch.arange(160, dtype=torch.int32, device="cuda").expand(book).contiguous()
    seen = put(p.len)
    out = torch.zeros((2, 3, 4, 128), dtype=torch.float16, device="cuda")
    ws = torch.empty(kvs.kv_attend_workspace_bytes(p.ks, 3, 1, True), dtype=torch.uint8, device="cuda")
    ws2 = torch.empty(kvs.kv_evict_workspace_bytes(p.ks, 3, 2, 90), dtype=torch.uint8, device="cuda")

    def step():
        for layer in range(2):
            kvs.kv_append_tokens(pages, layer, k, v, seen=seen, mass=mass[layer], pos=pos[layer])
            kvs.kv_attend_tokens(pages, layer, q, ws, out[layer], mass_in=mass[layer], mass=mass[layer])
        kvs.kv_evict_tokens(pages, 0, 2, mass, pos, 90, 4, 16, ws2, mass, pos, seen=seen)

    state = [pool, mass, pos, out]
    before = [t.clone() for t in state]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for lens in ([100, 41, 160], [101, 1, 33], [128, 0, 159]):
        pages.length.copy_(torch.tensor(lens, dtype=torch.int32))
        seen.copy_(torch.tensor([n + 7 for n in lens], dtype=torch.int32))
        for t in (k, v, q):
            t.normal_()
        for t, b in zip(state, before):
            t.copy_(b)
        step()
        torch.cuda.synchronize()
        eager = [t.clone() for t in state]
        for t, b in zip(state, before):
            t.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        for t, e in zip(state, eager):
            assert torch.equal(t.view(torch.uint8), e.view(torch.uint8))


def test_two_graphs_share_a_workspace():
    """Two captured calls over other layers with one workspace, replayed in turn, with other work on the same memory between them."""
    p = Paged((2, 2, 8, 128, 512, 16, 64), [512, 300], MIXED, 23)
    pages, _ = p.device()
    q = put(p.halves(2, 8, 128))
    ws = torch.empty(kvs.kv_attend_workspace_bytes(p.ks, 2, 1, True), dtype=torch.uint8, device="cuda")
    out, mass = torch.zeros((2, 2, 8, 128), dtype=torch.float16, device="cuda"), torch.zeros((2, 2, 2, 512), device="cuda")

    def call(layer):
        kvs.kv_attend_tokens(pages, layer, q, ws, out[layer], mass=mass[layer])

    want = []
    for layer in range(2):
        call(layer)
        want.append((out[layer].clone(), mass[layer].clone()))
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for layer, graph in enumerate(graphs):
        with torch.cuda.graph(graph):
            call(layer)
    for turn in range(4):
        for layer, graph in enumerate(graphs):
            ws.fill_(0xff if turn % 2 else 0x3c)
            out.zero_()
            mass.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out[layer], want[layer][0]) and torch.equal(mass[layer], want[layer][1])


def test_the_tensors_of_pages_are_fixed():
    p = Paged((1, 1, 1, 64, 16, 16, 64), [4], (16,), 24)
    pages, _ = p.device()
    for name in ("pool", "off", "bits", "length", "shape", "n_seqs"):
        with pytest.raises(AttributeError):
            setattr(pages, name, getattr(pages, name))
    pages.length.fill_(3)


def test_two_streams_at_once():
    """The same sequences attended from two streams with workspaces of their own."""
    p = Paged((1, 4, 8, 128, 2048, 16, 64), [2048, 1999], MIXED, 22)
    pages, _ = p.device()
    q = [put(p.halves(2, 8, 128)) for _ in range(2)]
    need = kvs.kv_attend_workspace_bytes(p.ks, 2, 1, True)
    alone, got = [], []
    for i in range(2):
        ws, out = torch.empty(need, dtype=torch.uint8, device="cuda"), torch.empty((2, 8, 128), dtype=torch.float16, device="cuda")
        mass = torch.zeros((2, 4, 2048), device="cuda")
        kvs.kv_attend_tokens(pages, 0, q[i], ws, out, mass=mass)
        alone.append((out, mass))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    spaces = [(torch.empty(need, dtype=torch.uint8, device="cuda"), torch.empty((2, 8, 128), dtype=torch.float16, device="cuda"),
               torch.zeros((2, 4, 2048), device="cuda")) for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        for i, st in enumerate(streams):
            ws, out, mass = spaces[i]
            kvs.kv_attend_tokens(pages, 0, q[i], ws, out, mass=mass, stream=st)
    torch.cuda.synchronize()
    for (ws, out, mass), (o, m) in zip(spaces, alone):
        assert torch.equal(out, o) and torch.equal(mass, m)


def test_a_packed_context_continues_without_a_load():
    """The path as a program has it: a cache is scored, planned and compressed on the device, then decoding goes on over the plan's own
    offsets and widths; the attention equals that over the cache the Load gives back."""
    from paper_2403_11805_amd import synth
    geom = (2, 2, 4, 128, 256, 16, 64)
    ks = kvs.Shape(*geom)
    kv = synth.make_kv(synth.Geometry(*geom), 5, "cpu", 1, 4.0).cuda()
    n = ks.n_chunks
    density = torch.rand(n, device="cuda")
    bits, off = torch.empty(n, dtype=torch.uint8, device="cuda"), torch.empty(n + 1, dtype=torch.int64, device="cuda")
    dst = torch.empty(n, dtype=torch.int32, device="cuda")
    kvs.kv_plan_chunks_dev(ks, density, 1, 1, 3, bits, off, dst)
    pool = torch.empty(n * kvs.kv_record_bytes(ks, 8), dtype=torch.uint8, device="cuda")
    kvs.kv_compress_chunks(ks, kv, bits, off, pool)
    loaded = torch.empty_like(kv)
    kvs.kv_swapin_chunks(ks, pool, off[:n], dst, bits, loaded)
    pages = kvs.Pages(ks, pool, off[None, :n].contiguous(), bits[None], torch.tensor([250], dtype=torch.int32, device="cuda"))
    q = torch.randn((1, 4, 128), device="cuda").half()
    ws = torch.empty(kvs.kv_attend_workspace_bytes(ks, 1), dtype=torch.uint8, device="cuda")
    out = torch.empty_like(q)
    for layer in range(2):
        kvs.kv_attend_tokens(pages, layer, q, ws, out)
        k, v = loaded[layer].double()[:, :, :250].repeat_interleave(2, 1)
        a = torch.softmax((k * q[0].double()[:, None]).sum(-1) / 128 ** 0.5, -1)
        want = (a[..., None] * v).sum(1)
        # both sides' K differ by an fp16 rounding (2^-11 of each element, which moves a logit by at most that of sum |q k|)
        move = (k.abs() * q[0].double()[:, None].abs()).sum(-1).max(-1).values / 128 ** 0.5 * 2.0 ** -11
        spread = (a[..., None] * v.abs()).sum(1)
        bar = spread * (2 * move[:, None] + 4 * 2.0 ** -11)
        assert bool(((out[0].double() - want).abs() <= bar).all())
