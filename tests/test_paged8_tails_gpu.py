"""Decode attention over the paged 8-bit cache on the GPU: long flat tails of a softmax, and the error of whole rows."""
import math

import numpy as np
import pytest
import torch

from tests import paged8_reference as R
from tests import paged8_weights as W
from tests.paged8_errors import row_errors

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


CASES = [("mla512", 16, 1, 64, [(0, 9000)], 1), ("mla512", 128, 1, 64, [(0, 3000), (0, 1700), (20, 20 * 64 + 900)], 1),
         ("mla512", 40, 1, 32, [(3, 3 * 64 + 70), (17, 17 * 64 + 333)], 2), ("mla512", 32, 1, 16, [(0, 1000), (0, 1)], 1),
         ("mla512", 80, 1, 32, [(3, 3 * 64 + 70), (17, 17 * 64 + 333)], 1), ("mla512", 24, 1, 64, [(0, 700), (9, 9 * 64 + 64)], 3),
         ("mla128", 32, 1, 64, [(0, 777), (5, 5 * 64 + 1)], 1), ("gqa128", 32, 8, 64, [(70, 70 * 64 + 500), (0, 2000)], 1),
         ("gqa128", 8, 2, 16, [(0, 5003), (0, 130)], 4), ("gqa128", 70, 1, 64, [(0, 900)], 1), ("gqa64", 24, 2, 128, [(0, 12001), (0, 50)], 1)]


@pytest.mark.parametrize("impl", [0, 1])
@pytest.mark.parametrize("shape,heads,kv,page,states,q_len", CASES)
def test_error_of_whole_rows(B, shape, heads, kv, page, states, q_len, impl):
    """Ordinary inputs: the norm of a row's error against the norm of the row (tests/paged8_errors.py), and the lse."""
    variant, d_sem, d_pos = SHAPES[shape]
    g = 64 if page <= 64 else 128
    r = np.random.RandomState(heads + page)
    width = max(-(-t // page) for _, t in states)
    n_pages = sum(-(-t // page) for _, t in states) + 1
    ids = r.permutation(n_pages)
    table = np.full((len(states), width), -1, dtype=np.int32)
    at = 0
    for b, (n, t) in enumerate(states):
        for e in range(-(-t // page)):
            if any(R.present(n, t, g, x) for x in range(e * page, (e + 1) * page)):
                table[b, e] = ids[at]
                at += 1
    code = lambda d: R.encode(np.clip(r.randn(n_pages, kv, page, d) * 60, -448, 448))  # noqa: E731
    scale = lambda: (2.0 ** r.randint(-7, -4, (n_pages, kv))).astype(np.float32)       # noqa: E731
    pool = [code(d_sem), code(d_pos), scale(), scale() if variant == "gqa" else None]
    q_pos = torch.from_numpy(0.4 * r.randn(len(states), q_len, heads, d_pos)).bfloat16()
    q_sem = torch.from_numpy(0.4 * r.randn(len(states), q_len, heads, d_sem)).bfloat16() if variant == "mla" else None
    sm = 1.0 / math.sqrt(192.0 if variant == "mla" else d_pos)
    p = B.make_params(variant, len(states), 1, heads, kv, d_sem, d_pos, g, 0, sm)
    dev = [None if x is None else torch.from_numpy(x).to(DEV) for x in pool]
    cache = B.paged8_cache(*dev, torch.from_numpy(table).to(DEV))
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)             # noqa: E731
    old = B.lca_set_attention_impl(impl)
    try:
        out, lse = B.decode_attention_paged8(p, cache, None if q_sem is None else q_sem.to(DEV), q_pos.to(DEV), i32([s[0] for s in states]),
                                             i32([s[1] for s in states]), want_lse=True)
        torch.cuda.synchronize()
    finally:
        B.lca_set_attention_impl(old)
    want, want_lse, _, _ = R.attend(None if q_sem is None else q_sem.double().numpy(), q_pos.double().numpy(), *pool, table,
                                    [s[0] for s in states], [s[1] for s in states], g, page, sm)
    print("row error %.2e, lse error %.2e" % row_errors(out.double().cpu().numpy(), lse.double().cpu().numpy(), want, want_lse))
