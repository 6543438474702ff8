"""Long sequences over the paged 4-bit cache, cut into pieces and merged: every tile shows in the outputs (tests/paged4_tiles.py)."""
import numpy as np
import pytest
import torch

from tests import paged4_tiles as T
from tests.test_paged4_gpu import DEV, SHAPES, B, i32, no_timeout  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("case", T.CASES, ids=lambda c: f"{c[0]}-{c[1]}-{c[4][0][1]}")
def test_every_tile_is_there_once(B, case):
    shape, heads, kv, page, states, g, weight = case
    variant, ds, dp = SHAPES[shape]
    nb, rep = len(states), heads // kv
    p = B.make_params(variant, nb, 1, heads, kv, ds, dp, g, 0, 1.0)
    tiles = [[T.Tiles(r, n, g, ds, b, j) for j in range(kv)] for b, (r, n) in enumerate(states)]
    width = max(-(-n // page) for _, n in states)
    used = np.zeros((nb, width), dtype=bool)
    for b in range(nb):
        used[b, tiles[b][0].rows // page] = True
    table = np.full((nb, width), -1, dtype=np.int32)
    table[used] = np.random.RandomState(1).permutation(int(used.sum()) + 3)[:int(used.sum())]
    cache = B.new_paged4_cache(p, int(used.sum()) + 3, page, width, DEV)
    cache.tensors[6].copy_(torch.from_numpy(table))
    for b in range(nb):
        rows = tiles[b][0].rows
        slots = torch.from_numpy(table[b, rows // page].astype(np.int64) * page + rows % page).int().to(DEV)
        sem, pos = torch.zeros((len(rows), kv, ds), device=DEV), torch.zeros((len(rows), kv, dp), device=DEV)
        for j, t in enumerate(tiles[b]):
            of = torch.from_numpy(t.of).to(DEV)
            sem[torch.arange(len(rows), device=DEV), j, torch.from_numpy(t.column).to(DEV)[of]] = torch.from_numpy(t.amplitude).float().to(DEV)[of]
            pos[:, j, 0] = torch.from_numpy(t.level).float().to(DEV)[of]
        B.paged4_write(p, cache, sem.bfloat16(), pos.bfloat16(), slots)
    q_pos = torch.zeros((nb, 1, heads, dp), dtype=torch.bfloat16, device=DEV)
    for h in range(heads):
        q_pos[:, 0, h, 0] = T.HEAD_FACTORS[h % rep % 4]
    q_sem = torch.zeros((nb, 1, heads, ds), dtype=torch.bfloat16, device=DEV) if variant == "mla" else None
    out, lse = B.decode_attention_paged4(p, cache, q_sem, q_pos, i32([r for r, _ in states]), i32([n for _, n in states]), want_lse=True)
    out, lse = out[:, 0].double().cpu().numpy(), lse[:, 0].double().cpu().numpy()
    for b in range(nb):
        for j in range(kv):
            want = {f: tiles[b][j].attend(f) for f in T.HEAD_FACTORS}
            for h in range(rep):
                w, wl = want[T.HEAD_FACTORS[h % 4]]
                o, l = out[b, j * rep + h], lse[b, j * rep + h]
                assert not T.differs(o, l, w, wl, weight), (b, j, h, float((np.abs(o - w) / np.maximum(w, 1e-30)).max()), l - wl)
