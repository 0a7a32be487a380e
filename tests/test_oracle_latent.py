"""The oracle of latent caches, pinned by what can be worked out otherwise: sizes, closed forms, a softmax written out, the codec of the
per-head caches."""
import numpy as np
import pytest

import oracle
import oracle.decode as od
import oracle.latent as ol

GEOM = (2, 3, 256, 32, 64, 64, 64, 16, 64)


def pages(shape, widths):
    """One sequence of a page per width, back to back."""
    sizes = [ol.record_bytes(shape, w) for w in widths]
    off = np.concatenate([[0], np.cumsum(sizes)])
    return np.zeros(off[-1], dtype=np.uint8), off[None, :-1].astype(np.int64), np.array([widths], dtype=np.uint8)


def test_record_bytes_by_hand():
    s = ol.Shape(*GEOM)
    assert ol.record_bytes(s, 16) == 2 * 16 * (512 + 64)
    assert ol.record_bytes(s, 4) == 2 * 16 * (128 + 64 + 2 * 4 * 4)
    assert ol.record_bytes(s._replace(fmt=3), 2) == 2 * 16 * (64 + 64 + 2 * 4 * 2)


@pytest.mark.parametrize("fmt", [0, 3])
@pytest.mark.parametrize("b", [8, 4, 2])
def test_codes_are_those_of_a_head_cache(fmt, b):
    """A latent row packs like a K row of one kv head with the same group."""
    rng = np.random.RandomState(1)
    s = ol.Shape(*GEOM, fmt)
    head = oracle.Shape(2, 1, 1, 256, 16, 16, 64, fmt)
    pool, off, bits = pages(s, [b])
    other = np.zeros(oracle.record_bytes(head, b), dtype=np.uint8)
    x = rng.standard_normal((16, 256)).astype(np.float16)
    for row in range(16):
        ol.Layer(s, pool, 0, b, 1).put(row, x[row], np.zeros(32, dtype=np.float16))
        od.Slab(head, other, 0, b, 1, 0, 0).put(head, row, x[row])
    a, c = ol.Layer(s, pool, 0, b, 1), od.Slab(head, other, 0, b, 1, 0, 0)
    assert np.array_equal(a.codes, c.codes) and np.array_equal(a.scale, c.scale) and np.array_equal(a.mn, c.mn)
    for row in range(16):
        assert np.array_equal(a.latents()[row], c.dequantised(head, row))


def test_append_then_read_gives_the_rows_within_half_a_step():
    rng = np.random.RandomState(2)
    s = ol.Shape(*GEOM)
    pool, off, bits = pages(s, [16, 8, 4, 2])
    c, r = rng.standard_normal((64, 256)).astype(np.float16), rng.standard_normal((64, 32)).astype(np.float16)
    start = np.array([0, 64])
    ol.append(s, pool, off, bits, [64], 1, c, r, start)
    got, r_got = np.zeros_like(c), np.zeros_like(r)
    ol.read(s, pool, off, bits, [64], 1, got, r_got, start)
    assert np.array_equal(r, r_got) and np.array_equal(c[:16], got[:16])
    for page, b in enumerate((16, 8, 4, 2)):
        g = c[16 * page:16 * page + 16].astype(np.float64).reshape(16, 4, 64)
        step = np.ptp(g, axis=-1, keepdims=True) / (2 ** b - 1)
        off_by = np.abs(got[16 * page:16 * page + 16].reshape(16, 4, 64) - g)
        assert np.all(off_by <= step / 2 + 2.0 ** -11 * np.abs(g).max() + 1e-6)
    other = np.zeros_like(c)
    ol.read(s, pool, off, bits, [64], 0, other, r_got, start)
    assert not other.any(), "another layer was written"


def test_attention_is_a_softmax_over_keys_and_values_of_every_head():
    rng = np.random.RandomState(3)
    s = ol.Shape(*GEOM)
    pool, off, bits = pages(s, [16, 0, 16, 16])
    bits[0, 1] = 0
    off[0, 2:] = [ol.record_bytes(s, 16), 2 * ol.record_bytes(s, 16)]
    c, r = rng.standard_normal((61, 256)).astype(np.float16), rng.standard_normal((61, 32)).astype(np.float16)
    ol.append(s, pool, off, bits, [61], 0, c, r, np.array([0, 61]))
    q, w = rng.standard_normal((3, 3, 96)).astype(np.float16), (rng.standard_normal((256, 3, 128)) / 16).astype(np.float16)
    got, sizes, spread, spread_c = ol.attend(s, pool, off, bits, [61], 0, q, w, np.array([0, 3]), 2)
    assert np.isnan(got[2]).all()
    for j in range(2):
        tokens = [t for t in range(58 + j + 1) if t // 16 != 1]
        for h in range(3):
            logits = []
            for t in tokens:
                k = np.concatenate([c[t].astype(float) @ w[:, h, :64].astype(float), r[t].astype(float)])
                logits.append(float(k @ q[j, h].astype(float)) / 96 ** 0.5)
            a = np.exp(np.array(logits) - max(logits))
            want = sum(x * (c[t].astype(float) @ w[:, h, 64:].astype(float)) for x, t in zip(a / a.sum(), tokens))
            np.testing.assert_allclose(got[j, h], want, rtol=1e-10, atol=1e-12)
            assert np.all(np.abs(want) <= spread[j, h] + 1e-12) and np.all(spread[j, h] <= spread_c[j, h] + 1e-12)
            assert max(np.abs(logits)) <= sizes["absorbed_all"][j, h] and max(np.abs(logits)) <= sizes["expanded_all"][j, h]


def test_equal_keys_average_the_values():
    s = ol.Shape(1, 1, 256, 32, 64, 64, 16, 16, 64)
    pool, off, bits = pages(s, [16])
    c = np.tile(np.arange(16, dtype=np.float16)[:, None], (1, 256))
    ol.append(s, pool, off, bits, [16], 0, c, np.zeros((16, 32), dtype=np.float16), np.array([0, 16]))
    w = np.zeros((256, 1, 128), dtype=np.float16)
    w[0, 0, 64:] = 1                                                # values are the latents' first number, keys are zero
    out = ol.attend(s, pool, off, bits, [16], 0, np.ones((4, 1, 96), dtype=np.float16), w, np.array([0, 4]))[0]
    np.testing.assert_allclose(out[:, 0, 0], [6.0, 6.5, 7.0, 7.5])
