"""Softmax weights as sums of two 8-bit terms: what the rounding does to sums over many keys, on the CPU (no GPU needed)."""
import numpy as np
import pytest

from tests import paged8_weights as W


@pytest.mark.parametrize("kind", ["single", "pair"])
def test_offsets_of_the_weights_are_spread_evenly(kind):
    """A weight below the last step is rounded up for that share of the offsets; equal keys are then off by the offsets' deviation
    from an even spread, under every column of values.  Computed for every threshold at once: sorted by offset, the running sum
    of the values minus its share of the whole."""
    for n in (64, 1000, 2176, 5056, 20000, 131072):
        rows = np.arange(n)
        order = np.argsort(W.offset(kind, rows), kind="stable")
        off = W.offset(kind, rows)[order]
        for period, v in W.waves(rows):
            c = np.concatenate([[0.0], np.cumsum(v[order])])
            want = c[-1] * (off + 0.5)                                        # below a threshold at this offset
            miss = max(np.abs(c[:-1] - want).max(), np.abs(c[1:] - want).max())
            assert miss <= (W.MISS if n <= 20000 else 4 * W.MISS), (n, period, miss)


@pytest.mark.parametrize("kind", ["single", "pair"])
def test_rounded_weights(kind):
    """One weight: relative 2^-9 (pairs 2^-8) where the second term is a normal number, else a step; zero stays zero."""
    r = np.random.RandomState(0)
    rows = r.randint(0, 1 << 20, 200000)
    t = 2.0 ** r.uniform(-30, 8.7 if kind == "single" else 11, rows.size)
    err = np.abs(W.rounded(kind, t, rows) - t)
    # half a place of the second term, at most 2^-9 (2^-8) of the weight, and the offset, at most half a step; below a place of
    # the first term the whole step
    assert np.all(err <= t * (2.0 ** -9 if kind == "single" else 2.0 ** -8) + W.STEP[kind])
    assert np.all(W.rounded(kind, np.zeros(rows.size), rows) == 0)


@pytest.mark.parametrize("kind", ["single", "pair"])
@pytest.mark.parametrize("n", [2176, 5056, 20000])
def test_a_flat_tail_keeps_its_weight_whatever_its_values(kind, n):
    rows = np.arange(n)
    for ratio in 2.0 ** -np.arange(8, 22, 0.37):
        t = np.full(n, W.LARGEST[kind] * ratio)
        t[5] = W.LARGEST[kind]
        diff = W.rounded(kind, t, rows) - t
        diff[5] = 0
        for period, v in W.waves(rows):
            limit = (2.0 ** -9 if kind == "single" else 2.0 ** -8) * abs((t * v).sum() - t[5] * v[5]) + W.MISS * W.STEP[kind]
            # where a place of the second term is wider than the offsets, keys differ by that place, 2^-8 (2^-7) of a weight
            limit += W.MISS * 2.0 ** (-8 if kind == "single" else -7) * W.LARGEST[kind] * ratio
            assert abs((diff * v).sum()) <= limit, (ratio, period, (diff * v).sum(), limit)
