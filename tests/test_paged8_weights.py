"""Softmax weights as sums of two 8-bit terms: what the rounding does to sums over many keys, on the CPU (no GPU needed)."""
import numpy as np
import pytest
import torch

from tests import paged8_reference as R
from tests import paged8_weights as W
from tests.paged8_errors import row_errors


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


@pytest.mark.parametrize("kind", ["single", "pair"])
@pytest.mark.parametrize("q_terms,w_terms", [(2, 2), (1, 2), (2, 1)])
def test_row_errors_tell_one_term_from_two(kind, q_terms, w_terms):
    """The bounds of tests/paged8_errors.py hold for the arithmetic as it is meant and for nothing less."""
    r = np.random.RandomState(2)
    heads, page, n, d_sem, d_pos = 8, 64, 1500, 512, 64
    n_pages = -(-n // page)
    sem, pos = (R.encode(np.clip(r.randn(n_pages, 1, page, d) * 60, -448, 448)) for d in (d_sem, d_pos))
    scale = (2.0 ** r.randint(-7, -4, (n_pages, 1))).astype(np.float32)
    q_sem, q_pos = (torch.from_numpy(0.4 * r.randn(1, 1, heads, d)).bfloat16().double().numpy() for d in (d_sem, d_pos))
    table = np.arange(n_pages, dtype=np.int32)[None]
    sm = 1.0 / np.sqrt(192.0)
    want, want_lse, _, _ = R.attend(q_sem, q_pos, sem, pos, scale, None, table, [0], [n], page, page, sm)
    rows = np.arange(n)
    s = scale[rows // page, 0].astype(np.float64)
    v, k = (R.decode(torch.from_numpy(c)).reshape(n_pages * page, -1)[:n] for c in (sem, pos))
    q = np.concatenate([q_sem[0, 0], q_pos[0, 0]], -1)
    f = 2.0 ** (7 - np.floor(np.log2(np.abs(q).max(-1, keepdims=True))))       # the largest element into [128, 256)
    hi = W.e4m3(q * f)
    q8 = (hi + (W.e4m3(q * f - hi) if q_terms == 2 else 0.0)) / f
    y = sm * s * (q8 @ np.concatenate([v, k], -1).T)                           # [heads, n]
    top = (y + np.log(s)).max(-1, keepdims=True)
    t = W.rounded(kind, W.LARGEST[kind] * np.exp(y + np.log(s) - top), np.broadcast_to(rows, y.shape), w_terms)
    total = (W.LARGEST[kind] * np.exp(y - top)).sum(-1, keepdims=True)
    out = torch.from_numpy((t @ v) / total).bfloat16().double().numpy()[None, None]
    lse = (np.log(total / W.LARGEST[kind]) + top)[None, None, :, 0]
    if (q_terms, w_terms) == (2, 2):
        row_errors(out, lse, want, want_lse)
    else:
        with pytest.raises(AssertionError):
            row_errors(out, lse, want, want_lse)
