"""The bar of test_probabilities_keep_22_bits tells probabilities of 22 bits from such of 11."""
import numpy as np
import pytest

from halves import cancelling, exact_values, halves_bar, kept_to_bits


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("n", [20, 37, 64])
def test_bar_tells_22_bits_from_11(D, n):
    _, _, v, weights = cancelling(D, n, 41)
    want, bar = exact_values(weights, v), halves_bar(weights, v)
    assert np.all(np.abs(exact_values(kept_to_bits(weights, 22), v) - want) <= bar)
    off = np.abs(exact_values(kept_to_bits(weights, 11), v) - want) / bar
    assert off.max() > 2 and (off > 1).mean() > 0.1, (off.max(), (off > 1).mean())
