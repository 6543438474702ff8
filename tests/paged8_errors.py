"""Bounds on the error of whole rows of decode attention over the paged 8-bit cache, for inputs without extremes: logits of a
few units over dozens of keys or more, so that no key carries the row alone."""
import numpy as np

#: |out - want| / |out| of a row.  bf16 rounds a value by 2^-8 of itself at most, evenly spread: 2^-8 / sqrt(3) of the norm at the
#: worst place of a binade.  The two terms of a weight are off by at most 2^-8 of it (2^-9 on single CTAs), evenly spread and
#: independent from key to key: 2^-8 / sqrt(3) of the norm again, as the values are independent too.  Together 0.82 * 2^-8; the
#: rest is room for what a few dozen values deviate from their mean square.
NORM = 2.0 ** -8
#: |lse - want|.  Logits are sums of up to 1152 products of 8-bit numbers, exact in fp32 and added in fp32: 1152 * 2^-24 of
#: scale * sum |q k| in any order, which is below 14 for the inputs here
LSE = 2.0 ** -10


def row_errors(out, lse, want, want_lse):
    """Asserts the bounds for every row (query, head); rows without a key are exact."""
    empty = ~np.isfinite(want_lse)
    assert np.array_equal(np.isneginf(lse), empty) and np.all(out[empty] == 0)
    norm = np.linalg.norm(want[~empty], axis=-1)
    err = np.linalg.norm(out[~empty] - want[~empty], axis=-1)
    dl = np.abs(lse[~empty] - want_lse[~empty])
    assert np.all(err <= NORM * norm), "row error %.2e" % (err / norm).max()
    assert np.all(dl <= LSE), "lse error %.2e" % dl.max()
    return (err / norm).max(initial=0), dl.max(initial=0)
