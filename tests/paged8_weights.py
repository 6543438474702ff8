"""The rounding of softmax weights in decode attention over the paged 8-bit cache, restated on the CPU in float64 (one weight at
a time, from the formats' definitions), and the bound on what it does to a sum over many keys of equal weight."""
import numpy as np

#: weights are scaled so that the largest of a row is at least this when its maximum is set
LARGEST = {"single": 2.0 ** 5, "pair": 2.0 ** 8}
#: step of the second term below the normal range of e4m3 (2^-9, the single-CTA kernel multiplies the term by 2^4 before)
STEP = {"single": 2.0 ** -13, "pair": 2.0 ** -9}
#: steps by which the rounded weights of equal keys under +1 / -1 values of period 2 .. 32 miss their sum, at most
#: (test_offsets_of_the_weights_are_spread_evenly computes it from the offsets)
MISS = 64


def to_format(x, mantissa, e_min, top):
    """Nearest value (ties to even) with `mantissa` fraction bits, smallest normal 2^e_min, saturating at top."""
    x = np.clip(np.asarray(x, dtype=np.float64), -top, top)
    e = np.maximum(np.frexp(np.abs(x))[1] - 1, e_min)
    step = np.ldexp(1.0, e - mantissa)
    return np.rint(x / step) * step


def e4m3(x):
    return to_format(x, 3, -6, 448.0)


def e5m2(x):
    return to_format(x, 2, -14, 57344.0)


def offset(kind, row):
    """Offset of the key in this row, in steps, from [-1/2, 1/2]: the row times the golden ratio, modulo 1.  The pair kernel
    reads it from a table of which every tile of 128 rows takes another one of 1024 windows, four places apart."""
    row = np.asarray(row, dtype=np.int64)
    if kind == "pair":
        row = row % 128 + 4 * (613 * (row // 128) % 1024)
    u = (row * 0x9E3779B9) % 2 ** 32
    return np.where(u >= 2 ** 31, u - 2.0 ** 32, u) * 2.0 ** -32


def rounded(kind, t, row, terms=2):
    """What the products see of weight t of the key in this row."""
    t = np.asarray(t, dtype=np.float64)
    hi = e4m3(t) if kind == "single" else e5m2(t)
    if terms == 1:
        return hi
    gain = 2.0 ** -9 / STEP[kind]
    return hi + e4m3((t - hi) * gain + offset(kind, row) * 2.0 ** -9) / gain


def waves(rows):
    """Columns of values with a period: [(period, +1 / -1 in halves of it)], and all ones."""
    return [(p, np.where(rows % p < p / 2, 1.0, -1.0)) for p in (2, 3, 4, 5, 7, 8, 12, 16, 24, 31, 32)] + [(1, np.ones(len(rows)))]
