"""GPU parity of latent caches (append, read, attention in both forms) against the oracle in 64 bits.

Bars: appended and read bytes are equal; attention is within the roundings that tests/latent.py counts."""
import numpy as np
import pytest
import torch

import oracle.latent as ol
import paper_2403_11805_amd as kvs

from latent import Latent, attend, check_attend, put, rows

pytestmark = pytest.mark.gpu

MIXED = (16, 8, 4, 2)


def append(p, layer, c, r, row_start=None):
    pages, pool = p.device()
    kvs.kv_latent_append_tokens(pages, layer, put(c), put(r), row_start=put(row_start))
    torch.cuda.synchronize()
    return pool.cpu().numpy()


def read(p, layer, n_rows, row_start=None):
    pages, pool = p.device()
    c = torch.full((n_rows, p.os.Dc), 7.0, dtype=torch.float16, device="cuda")
    r = torch.full((n_rows, p.os.Dr), 7.0, dtype=torch.float16, device="cuda")
    kvs.kv_latent_read_tokens(pages, layer, c, r, row_start=put(row_start))
    torch.cuda.synchronize()
    assert np.array_equal(pool.cpu().numpy(), p.pool)
    return c.cpu().numpy(), r.cpu().numpy()


MOVED = [
    ((1, 1, 256, 32, 64, 64, 16, 16, 64), [1], [1]),
    ((2, 3, 512, 64, 128, 128, 160, 32, 128), [160, 33, 32, 31, 0], [1, 1, 1, 1, 1]),
    ((3, 1, 256, 64, 64, 128, 192, 48, 256), [192, 47, 49, 100], [192, 0, 49, 7]),
    ((2, 2, 512, 32, 128, 64, 128, 64, 512), [128, 2, 77], [40, 5, 77]),           # more new rows than tokens
    ((1, 2, 512, 64, 64, 64, 9008, 16, 64), [9000, 300], [8700, 300]),               # several rows a wavefront
    ((1, 1, 256, 32, 64, 64, 9008, 16, 64), [9008, 1, 3], [9007, 1, 2]),
]


@pytest.mark.parametrize("geom,lens,counts", MOVED)
@pytest.mark.parametrize("fmt", [0, 3])
def test_append_and_read(geom, lens, counts, fmt):
    p = Latent(geom, lens, MIXED + (0,), 3, fmt, spare_stride=1)
    start, n_rows = rows(counts, lead=2)
    c, r = p.halves(n_rows + 3, geom[2]), p.halves(n_rows + 3, geom[3])
    c[::5] = np.round(c[::5])                                   # codes that lie between two
    c[1::7] = 0.25                                              # groups without a range
    layer = geom[0] - 1
    got, want = append(p, layer, c, r, start), p.pool.copy()
    ol.append(p.os, want, *p.table(), layer, c, r, start)
    assert np.array_equal(got, want)
    p.pool = want
    c_got, r_got = read(p, layer, n_rows + 3, start)
    c_want, r_want = np.full_like(c, 7.0), np.full_like(r, 7.0)
    ol.read(p.os, p.pool, *p.table(), layer, c_want, r_want, start)
    assert np.array_equal(c_got.view(np.uint16), c_want.view(np.uint16)) and np.array_equal(r_got.view(np.uint16), r_want.view(np.uint16))


@pytest.mark.parametrize("dims", [(256, 32, 64, 64), (256, 64, 128, 64), (512, 32, 64, 128), (512, 64, 128, 128)])
@pytest.mark.parametrize("width", [16, 8, 4, 2])
@pytest.mark.parametrize("fmt", [0, 3])
@pytest.mark.parametrize("expanded", [False, True])
def test_attend_one_width(dims, width, fmt, expanded):
    p = Latent((2, 5, *dims, 96, 32, 64), [96, 1, 33, 95], (width,), 3, fmt)
    check_attend(p, 1, p.queries(4), p.weights(), expanded=expanded)


@pytest.mark.parametrize("geom,lens,counts,widths", [
    ((1, 1, 256, 32, 64, 64, 16, 16, 64), [1], [1], (16,)),                                    # one token, one head
    ((2, 3, 512, 64, 128, 64, 160, 16, 64), [160, 17, 16, 15, 0], [1, 1, 1, 1, 1], MIXED),     # pages end inside a tile
    ((1, 8, 256, 64, 64, 128, 192, 48, 128), [192, 47, 49, 100], [3, 0, 4, 1], MIXED),         # pages of three half tiles
    ((1, 7, 512, 32, 64, 64, 128, 64, 512), [128, 2, 77], [5, 2, 4], MIXED + (0,)),            # 35 query rows, absent pages
    ((2, 4, 512, 64, 128, 128, 1024, 16, 128), [1024, 999, 3], [2, 1, 3], MIXED + (0, 0)),     # long: divided in shares
    ((1, 20, 256, 32, 64, 64, 128, 16, 256), [128, 100], [16, 7], MIXED),                      # 320 query rows
    ((1, 4, 512, 64, 64, 64, 64, 16, 64), [2, 5], [3, 8], (8, 16)),                            # more new rows than tokens
    ((1, 130, 512, 64, 128, 128, 96, 16, 64), [90, 41], [2, 1], MIXED),                        # more heads than a tile has rows
])
@pytest.mark.parametrize("expanded", [False, True])
def test_attend_rows_and_pages(geom, lens, counts, widths, expanded):
    p = Latent(geom, lens, widths, 5, spare_stride=1)
    start, n_rows = rows(counts, lead=2)
    check_attend(p, geom[0] - 1, p.queries(n_rows + 3), p.weights(), start, max(counts + [1]), expanded)


@pytest.mark.parametrize("geom,lens,counts", [
    ((1, 2, 256, 32, 64, 64, 512, 16, 64), [500, 301], [500, 300]),                 # several row tiles, several heads
    ((1, 8, 512, 64, 128, 128, 320, 32, 128), [320, 129, 128, 1], [130, 129, 127, 1]),
    ((1, 1, 512, 64, 128, 64, 1024, 64, 512), [1024], [257]),
])
def test_prompts(geom, lens, counts):
    p = Latent(geom, lens, MIXED, 7)
    start, n_rows = rows(counts)
    check_attend(p, 0, p.queries(n_rows), p.weights(), start, expanded=True)


def test_prompts_that_do_not_fit_are_left_out():
    p = Latent((1, 2, 256, 32, 64, 64, 128, 16, 64), [100, 128, 20], MIXED, 7)
    start, n_rows = rows([5, 6, 7])
    q, w = p.queries(n_rows), p.weights()
    whole = attend(p, 0, q, w, start, expanded=True)
    got = attend(p, 0, q, w, start, expanded=True, n_tokens=110)         # room for 110 / 32 + 3 tiles: the first sequence's four
    assert np.array_equal(got[:5], whole[:5]) and np.all(got[5:] == 7)


@pytest.mark.parametrize("expanded", [False, True])
def test_attend_without_any_page(expanded):
    p = Latent((1, 4, 256, 32, 64, 64, 64, 16, 64), [64, 30], (0,), 1)
    assert not attend(p, 0, p.queries(2), p.weights(), expanded=expanded).any()


BAD = ((8, 16), (-16, 16), (1 << 62, 4), (0, 3), (0, 255), (0, 1), (0, 18))


def spoil(p, s=0):
    """The first pages of a sequence get offsets that are odd, reach past the pool or lie far away, and widths of no format."""
    for j, (off, b) in enumerate(BAD + ((p.pool.size - 16, 16), (p.pool.size, 2), (p.pool.size + 16, 2))):
        p.off[s, j], p.bits[s, j] = off, b


@pytest.mark.parametrize("expanded", [False, True])
def test_bad_pages_are_absent(expanded):
    p = Latent((1, 2, 256, 32, 64, 64, 192, 16, 64), [192], (16,), 9)
    spoil(p)
    check_attend(p, 0, p.queries(1), p.weights(), expanded=expanded)


def test_append_and_read_leave_bad_pages():
    p = Latent((1, 2, 512, 64, 64, 64, 192, 16, 64), [192], (16,), 9)
    spoil(p)
    start, _ = rows([192])
    c, r = p.halves(192, 512), p.halves(192, 64)
    want = p.pool.copy()
    ol.append(p.os, want, *p.table(), 0, c, r, start)
    assert np.array_equal(append(p, 0, c, r, start), want) and not np.array_equal(want, p.pool)
    c_want, r_want = np.full_like(c, 7.0), np.full_like(r, 7.0)
    ol.read(p.os, p.pool, *p.table(), 0, c_want, r_want, start)
    c_got, r_got = read(p, 0, 192, start)
    assert np.array_equal(c_got, c_want) and np.array_equal(r_got, r_want) and np.any(c_got == 7.0)


@pytest.mark.parametrize("expanded", [False, True])
@pytest.mark.parametrize("value", [np.inf, -np.inf, np.nan])
def test_latents_that_are_not_finite_reach_only_rows_that_see_them(expanded, value):
    p = Latent((1, 5, 512, 64, 128, 128, 96, 16, 64), [90, 64, 33], (16,), 2)
    counts = [4, 4, 4]
    start, n_rows = rows(counts)
    q, w = p.queries(n_rows), p.weights()
    clean = attend(p, 0, q, w, start, 4, expanded)
    for s, token in ((0, 88), (1, 61), (2, 32)):                 # seen by the sequence's last 2, 2 and 1 rows
        x, row = p.at(s, token, 0)
        x.codes[row].view(np.float16)[[3, 500]] = value
    got = attend(p, 0, q, w, start, 4, expanded)
    blind = np.array([1, 1, 0, 0, 1, 0, 0, 0, 1, 1, 1, 0], dtype=bool)
    blind[4:8] = [True, False, False, False]
    assert np.array_equal(got[blind], clean[blind])
    assert not np.isfinite(got[~blind]).all(-1).any(), "a row that sees them is finite"


@pytest.mark.parametrize("expanded", [False, True])
def test_queries_that_are_not_finite_stay_in_their_row(expanded):
    p = Latent((1, 5, 256, 64, 64, 128, 96, 16, 64), [90, 64], MIXED, 2)
    start, n_rows = rows([3, 2])
    q, w = p.queries(n_rows), p.weights()
    clean = attend(p, 0, q, w, start, 3, expanded)
    q[1, 2, 5], q[3, 4, 70] = np.nan, np.inf
    got = attend(p, 0, q, w, start, 3, expanded)
    hit = np.zeros((5, 5), dtype=bool)
    hit[1, 2] = hit[3, 4] = True
    assert np.array_equal(got[~hit], clean[~hit]) and np.isnan(got[hit]).all()


@pytest.mark.parametrize("expanded", [False, True])
def test_masks_of_minus_infinity_in_the_position_parts(expanded):
    """A position part may rule a token out for every query: of logits that are all -inf a row is zeros."""
    p = Latent((1, 3, 256, 32, 64, 64, 64, 16, 64), [50, 40], (16,), 4)
    q, w = np.abs(p.queries(2)), p.weights()
    for token in range(50):
        x, row = p.at(0, token, 0)
        x.rope[row][:] = -np.inf
    for token in range(0, 40, 3):
        x, row = p.at(1, token, 0)
        x.rope[row][:] = -np.inf
    got = attend(p, 0, q, w, expanded=expanded)
    assert not got[0].any()
    x = ol.sequence(p.os, p.pool, p.off[1], p.bits[1], 40, 0)
    keep = np.arange(40) % 3 != 0
    for h in range(3):
        z = (x.c[keep] @ w[:, h, :64].astype(float) @ q[1, h, :64].astype(float) + x.r[keep] @ q[1, h, 64:].astype(float)) / np.sqrt(96)
        a = np.exp(z - z.max())
        np.testing.assert_allclose(got[1, h], (a / a.sum()) @ x.c[keep] @ w[:, h, 64:].astype(float), atol=0.03)


@pytest.mark.parametrize("expanded", [False, True])
def test_logits_far_apart(expanded):
    """Large logits of either sign, in ascending and descending order along a sequence: the references move, and far ones vanish."""
    p = Latent((1, 2, 256, 32, 64, 64, 256, 16, 64), [256, 250], (16,), 4)
    q, w = p.queries(2, scale=0.25), p.weights()
    q[:, :, 64:] = 1.0
    for s, sign in ((0, 1), (1, -1)):
        for token in range(p.len[s]):
            x, row = p.at(s, token, 0)
            x.rope[row][:] = sign * (token - 128) * 0.5
    check_attend(p, 0, q, w, expanded=expanded)
