"""What tests/paged4_tiles.py states, on the CPU: no tile can be lost, doubled or weighted wrongly without being seen."""
import numpy as np
import pytest

from tests import paged4_tiles as T

DS = {"mla512": 512, "mla128": 128, "gqa128": 128, "gqa64": 64}


@pytest.mark.parametrize("case", T.CASES, ids=lambda c: f"{c[0]}-{c[1]}-{c[4][0][1]}")
def test_every_tile_shows(case):
    shape, heads, kv, page, states, g, weight = case
    factors = sorted({T.HEAD_FACTORS[h % 4] for h in range(heads // kv)})
    for b, (r, n) in enumerate(states):
        t = T.Tiles(r, n, g, DS[shape], b)
        assert len(t.rows) <= 40064 and np.bincount(t.column).max() <= 5         # what the bound counts
        want = {f: t.attend(f) for f in factors}
        for f in factors:
            assert not T.differs(want[f][0] * (1 + 2.0 ** -8 + weight / 2), want[f][1] + 1e-5, *want[f], weight)
        pieces = [(i, i + 1) for i in range(len(t.ids))] + [(i, min(i + 5, len(t.ids))) for i in range(0, len(t.ids), 5)]
        for lo, hi in pieces:
            for times in (0.0, 0.5, 2.0):
                if hi - lo == len(t.ids):
                    continue
                share = np.ones(len(t.ids))
                share[lo:hi] = times
                assert any(T.differs(*t.attend(f, share), *want[f], weight) for f in factors), (b, lo, hi, times)
