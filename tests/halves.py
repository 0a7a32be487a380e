"""A call of attention whose result is almost nothing but the rounding of its probabilities.

q picks one dimension of K, so that logits are one number of K over sqrt(head_dim) each.  V is large and, weighed, adds up to
almost nothing: the last token's row is what takes away the sum of the others', as near as a half can say it.  So the last
rounding of a result is small, V and the products with it are exact, and the error left is that of the weights, and of sums in binary32.

Bounds, relative to sum p |v| with n tokens:
  exponents   log2(e) / sqrt(D) in binary32 (2^-25 of at most 2) and the difference to the reference (at most 16 + 2, half a step 2^-20), times ln 2:  0.75 * 2^-20
  exp2        one step of binary32                                                                                                                    2^-23
  p           as the sum of two halves of 11 bits                                                                                                     2^-22
  sums        one step, 2^-23, for each of the 2 n products, and 24 for the states' and shares' common references                                      (2 n + 24) 2^-23
and half a step of the result itself, 2^-11.  The weights' sum is off by no more than that, but of a result that is almost nothing."""
import numpy as np


def cancelling(D, n, seed):
    """-> q [D], k [n][D], v [n][D] as halves, weights [n] in 64 bits."""
    rng = np.random.RandomState(seed)
    q, k = np.zeros(D, dtype=np.float16), np.zeros((n, D), dtype=np.float16)
    q[0] = 1
    k[:, 0] = rng.uniform(-1, 1, n) * np.sqrt(D)
    k[-1, 0] = np.sqrt(D) * 2                                   # the one that cancels weighs most
    z = k[:, 0].astype(np.float64) / np.sqrt(D)
    weights = np.exp(z - z.max())
    weights /= weights.sum()
    v = rng.uniform(-2000, 2000, (n, D)).astype(np.float16)
    v[-1] = -(weights[:-1] @ v[:-1].astype(np.float64)) / weights[-1]
    return q, k, v, weights


def exact_values(weights, v):
    return weights @ v.astype(np.float64)


def halves_bar(weights, v):
    n, spread = len(weights), weights @ np.abs(v.astype(np.float64))
    return spread * (0.75 * 2.0 ** -20 + 2.0 ** -23 + 2.0 ** -22 + (2 * n + 24) * 2.0 ** -23) + np.abs(exact_values(weights, v)) * 2.0 ** -11 + 2.0 ** -24


def kept_to_bits(weights, bits):
    """The probabilities as attention has them, 2^7 for the largest, with so many leading bits, the others cut off; as weights."""
    p = weights / weights.max() * 128
    step = 2.0 ** (np.floor(np.log2(p)) - (bits - 1))
    return np.floor(p / step) * step / 128 * weights.max()
