"""Sequences whose attention shows every one of their tiles of 128 rows: what a tile adds cannot be taken for rounding.

Every tile has a column of the values to itself, or shares it with a few others, and is 2 or 3 there and 0 elsewhere.  All rows of a tile have the same
logit, 0 to 2 times a factor of the query head's (0, 1, -1, 1/2), rising along the sequence, so that its pieces have different maxima.  All
terms are positive, so that errors do not add up beyond the largest relative one of a term.

How far outputs may be off, relative to their value: a weight's two terms by `weight`; no weight is below e^-2 of the largest, far above the
floor.  A column adds at most 5 tiles in fp32, 640 terms, 2^-23 each if the products' sums are cut off: 2^-13.6; a row sum adds
rows / 128 terms a thread (at most 313, 2^-24 each) and a few dozen more, 2^-15.5; logits up to 16 in units of log2 and the exponential 2^-19.  2^-12 holds them
all.  Then one rounding to bf16, 2^-8.  The logarithm of a row sum is off by the error of the sum, 2^-15 with what the logits add, and by roundings of
2^-24 of itself and of its parts, up to 16 each: 2^-14 in all."""
import numpy as np

HEAD_FACTORS = (0.0, 1.0, -1.0, 0.5)
AMPLITUDES = (2.0, 3.0)
LSE = 2.0 ** -14


class Tiles:
    """Sequence `b`, KV head `j` with n_tok tokens and n_rep representatives of groups of g: rows that are present and what they hold."""

    def __init__(self, n_rep, n_tok, g, ds, b=0, j=0):
        self.rows = np.array(list(range(n_rep)) + list(range(n_rep * g, n_tok)), dtype=np.int64)
        tile = self.rows // 128
        self.ids, self.of = np.unique(tile, return_inverse=True)
        n = len(self.ids)
        self.count = np.bincount(self.of, minlength=n).astype(np.float64)
        at = np.arange(n)
        self.ds = ds
        self.column = (at * 5 + 13 * b + 7 * j) % ds
        self.amplitude = np.array([AMPLITUDES[(i // ds + i) % 2] for i in range(n)])
        self.level = np.rint(4.0 * at / max(n - 1, 1)) / 2

    def attend(self, factor, share=None):
        """(out [ds], lse) for a query head of this factor; share: how much of each tile takes part."""
        w = np.exp(factor * self.level) * self.count * (1.0 if share is None else share)
        return np.bincount(self.column, w * self.amplitude, self.ds) / w.sum(), np.log(w.sum())


def tolerance(weight):
    return (1 + 2.0 ** -8) * (1 + weight + 2.0 ** -12) - 1


def differs(out, lse, want, want_lse, weight):
    """Whether a query's outputs are further from `want` than rounding explains."""
    return bool(np.any(np.abs(out - want) > tolerance(weight) * want) or abs(lse - want_lse) > LSE)


# shape, heads, kv, page, [(n_rep, n_tok)], group; weight: what a weight's two terms are off by
SINGLE, PAIR = 2.0 ** -9, 2.0 ** -8
CASES = [
    ("mla512", 16, 1, 64, [(0, 9000)], 64, SINGLE), ("mla512", 33, 1, 64, [(0, 21000)], 64, SINGLE), ("mla512", 64, 1, 16, [(0, 2600), (0, 1900)], 64, SINGLE),
    ("mla512", 9, 1, 32, [(200, 200 * 64 + 3000), (0, 700)], 64, SINGLE), ("mla512", 70, 1, 64, [(0, 30001), (0, 29224)], 64, PAIR),
    ("mla512", 128, 1, 128, [(0, 9000)], 128, PAIR), ("mla512", 128, 1, 64, [(0, 6000)] + [(0, 300 + 37 * i) for i in range(30)], 64, PAIR),
    ("mla512", 100, 1, 16, [(300, 300 * 16 + 2500)], 16, PAIR), ("mla128", 8, 1, 64, [(0, 20001)], 64, SINGLE), ("mla128", 64, 1, 32, [(0, 5000), (0, 3333)], 64, SINGLE),
    ("gqa64", 4, 1, 64, [(0, 40001)], 64, SINGLE), ("gqa64", 40, 2, 16, [(0, 5003), (0, 4303), (0, 77)], 64, SINGLE), ("gqa128", 8, 2, 64, [(0, 5003), (0, 4303), (0, 3603)], 64, SINGLE),
    ("gqa128", 40, 2, 128, [(0, 7000), (0, 6300)], 128, SINGLE), ("gqa128", 32, 8, 64, [(0, 9001)] + [(0, 200 + 61 * i) for i in range(25)], 64, SINGLE),
]
