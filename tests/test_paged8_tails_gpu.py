"""Decode attention over the paged 8-bit cache on the GPU: long flat tails of a softmax."""
import math

import numpy as np
import pytest
import torch

from tests import paged8_weights as W

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
SHAPES = {"mla512": ("mla", 512, 64), "mla128": ("mla", 128, 64), "gqa128": ("gqa", 128, 128), "gqa64": ("gqa", 64, 64)}


@pytest.fixture(scope="module")
def B():
    from paper_2604_12452_b200 import build
    build.build()
    from paper_2604_12452_b200 import binding
    return binding


@pytest.fixture(autouse=True)
def no_timeout(B):
    yield
    assert B.lca_last_device_status() == 0


@pytest.mark.parametrize("n", [2176, 5056, 20000])
@pytest.mark.parametrize("shape,heads,kind,nb", [("gqa64", 16, "single", 296), ("gqa128", 16, "single", 296), ("gqa128", 32, "single", 296), ("gqa128", 64, "single", 148),
                                                 ("mla128", 16, "single", 296), ("mla512", 16, "single", 148), ("mla512", 32, "single", 148),
                                                 ("mla512", 128, "pair", 74)])
def test_a_flat_tail_keeps_its_weight_whatever_its_values(B, shape, heads, kind, nb, n):
    """One key far above all others, which have the logit 0, and values with a period: a weight at the end of what its 8-bit terms
    hold is rounded up for some keys and down for others, and no period of the values may find out which.  Every sequence (all on
    the same pages) has a CTA of its own, so that none of its tiles gets a maximum of its own.  Column c of the values is +1 / -1
    with a period (2 to 32, or all ones), head h sees the tail at 2^-8 ... 2^-21 of the peak."""
    variant, d_sem, d_pos = SHAPES[shape]
    page = 128
    n_pages = -(-n // page)
    p = B.make_params(variant, nb, 1, heads, 1, d_sem, d_pos, page, 0, 1.0)
    cache = B.new_paged8_cache(p, n_pages, page, n_pages, DEV)
    sem, pos, ss, sp, table = cache.tensors
    table.copy_(torch.arange(n_pages, dtype=torch.int32, device=DEV).expand(nb, -1))
    waves = W.waves(np.arange(n_pages * page))
    cols = np.stack([waves[c % len(waves)][1] for c in range(d_sem)], 1)
    codes = np.where(cols > 0, 0x38, 0xb8).astype(np.uint8)                    # +-1
    codes[5] = 0                                                               # the peak's values are 0
    sem.copy_(torch.from_numpy(codes.reshape(n_pages, 1, page, d_sem)))
    pos[0, 0, 5] = 0x38                                                        # its key is (1, ..., 1), all others are 0
    tops = math.log(2) * np.linspace(8.0, 21.0, heads)
    q_pos = torch.from_numpy(np.broadcast_to(tops[:, None] / d_pos, (nb, 1, heads, d_pos)).copy()).bfloat16().to(DEV)
    q_sem = torch.zeros((nb, 1, heads, d_sem), dtype=torch.bfloat16, device=DEV) if variant == "mla" else None
    out, lse = B.decode_attention_paged8(p, cache, q_sem, q_pos, None, torch.full((nb,), n, dtype=torch.int32, device=DEV), want_lse=True)
    assert torch.equal(out, out[:1].expand_as(out)) and torch.equal(lse, lse[:1].expand_as(lse))
    peak = np.exp(q_pos[0, 0].double().sum(-1).cpu().numpy())                   # [heads], relative to a tail weight of 1
    total = peak + n - 1
    tail = np.where(np.arange(n)[:, None] == 5, 0.0, cols[:n]).sum(0)           # [d_sem]
    want = tail[None] / total[:, None]
    # a weight's two terms: 2^-9 (pairs 2^-8) of it, in common; bf16: 2^-8; the logit of the peak, up to 15, through fp32 sums
    # and exp2: 2^-13; what the offsets leave: MISS steps, in units of the largest weight, or of a place of the second term,
    # 2^-8 (2^-7) of a weight
    places = W.STEP[kind] / W.LARGEST[kind] * peak + 2.0 ** (-8 if kind == "single" else -7)
    tol = np.abs(want) * (2.0 ** -8 + 2.0 ** (-9 if kind == "single" else -8) + 2.0 ** -13) + (W.MISS * places / total)[:, None]
    err = np.abs(out[0, 0].double().cpu().numpy() - want)
    worst = np.unravel_index(np.argmax(err / tol), err.shape)
    print("%s %d heads, %d rows: largest error %.1e, %.2f of the tolerance" % (shape, heads, n, err.max(), (err / tol).max()))
    assert np.all(err <= tol), (worst, waves[worst[1] % len(waves)][0], float(err[worst]), float(want[worst]), float(tol[worst]))
    assert np.all(np.abs(lse[0, 0].double().cpu().numpy() - np.log(total)) <= 2.0 ** -11)
