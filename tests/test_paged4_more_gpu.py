"""Paged 4-bit cache: NaN among drafted tokens, and row copies of more rows than the launch has warps for."""
import numpy as np
import pytest
import torch

from tests import paged4_reference as R
from tests.test_paged4_gpu import DEV, SHAPES, B, build, i32, no_timeout, to_gpu  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("impl", [0, 1])
@pytest.mark.parametrize("shape,heads,kv", [("mla512", 16, 1), ("mla512", 6, 1), ("mla512", 40, 1), ("mla128", 8, 1), ("gqa128", 8, 2), ("gqa64", 4, 2)])
def test_nan_in_a_drafts_row_with_several_queries(B, shape, heads, kv, impl):
    # the row of the second of four tokens: the first query does not see it.  Sequences with the row in the middle of a tile, as a tile's first, and alone there
    variant, ds, dp = SHAPES[shape]
    q_len, states = 4, [(0, 70), (0, 131), (0, 260), (0, 130)]
    pool, table = build(shape, kv, 16, states, 64, 3)
    g = torch.Generator().manual_seed(1)
    q_pos = torch.randn((4, q_len, heads, dp), generator=g).bfloat16().to(DEV)
    q_sem = torch.randn((4, q_len, heads, ds), generator=g).bfloat16().to(DEV) if variant == "mla" else None
    p = B.make_params(variant, 4, 1, heads, kv, ds, dp, 64, 0, 0.1)
    n_tok = i32([n for _, n in states])

    def run():
        cache, _ = to_gpu(B, pool, table)
        old = B.lca_set_attention_impl(impl)
        try:
            out, lse = B.decode_attention_paged4(p, cache, q_sem, q_pos, None, n_tok, want_lse=True)
            torch.cuda.synchronize()
        finally:
            B.lca_set_attention_impl(old)
        return out, lse
    clean = run()
    assert torch.isfinite(clean[0]).all() and torch.isfinite(clean[1]).all()
    rep, hk = heads // kv, kv - 1
    of_head = torch.arange(heads, device=DEV) // rep == hk
    for part in ("sem", "pos"):
        shifts = pool.shift_sem if part == "sem" else pool.shift_pos
        for b in (0, 1, 3):                                                    # (sequence 2 stays as it is)
            x = states[b][1] - q_len + 1
            at = table[b, x // 16], hk, x % 16, 0
            saved = shifts[at]
            shifts[at] |= 0xf0                                                 # columns 32 .. 63
            out, lse = run()
            shifts[at] = saved
            logits = variant == "mla" or part == "pos"
            for i in range(q_len):
                bad, bad_lse = torch.isnan(out[b, i]), torch.isnan(lse[b, i])
                if i >= 1:                                                     # sees the row
                    cols = torch.ones(ds, dtype=torch.bool, device=DEV)
                    if not logits:
                        cols[:32], cols[64:] = False, False
                    assert torch.equal(bad, of_head[:, None] & cols) and torch.equal(bad_lse, of_head & logits)
                else:
                    # its logits are its own: lse as before, but for the order in which maxima are raised (rows share that decision)
                    assert float((lse[b, i] - clean[1][b, i]).abs().max()) < 1e-4
                    if variant == "gqa" and part == "pos":                     # a weight of zero times finite values
                        assert float((out[b, i].float() - clean[0][b, i].float()).norm() / clean[0][b, i].float().norm()) < 2.0 ** -8
                assert torch.equal(out[b, i, ~of_head], clean[0][b, i, ~of_head]) and torch.equal(lse[b, i, ~of_head], clean[1][b, i, ~of_head])
            others = [s for s in range(4) if s != b]
            assert torch.equal(out[others], clean[0][others]) and torch.equal(lse[others], clean[1][others])


# a launch has 75776 warps: groups of four MLA rows, eight KV heads of a row, or eight vectors of other numbers of KV heads
@pytest.mark.parametrize("shape,kv,n", [("mla512", 1, 4 * 75776 + 4 * 9000 + 3), ("mla128", 1, 4 * 75776 + 2), ("gqa64", 8, 75776 + 1203), ("gqa64", 3, 8 * 75776 // 3 + 5001),
                                        ("gqa128", 1, 8 * 75776 + 13), ("gqa64", 24, 75776 + 77)])
def test_more_rows_than_warps(B, shape, kv, n):
    # in one call and in parts that no warp comes round a second time for (the other tests compare those with the reference)
    variant, ds, dp = SHAPES[shape]
    p = B.make_params(variant, 1, 1, kv, kv, ds, dp, 64, 0, 1.0)
    page, part = 64, 20000
    n_pages = -(-n // page) + 5
    g = torch.Generator(device=DEV).manual_seed(1)
    slots = torch.randperm(n_pages * page, generator=g, device=DEV)[:n].int()
    slots[torch.randint(0, n, (n // 50,), generator=g, device=DEV)] = -1
    slots[n - 1] = n_pages * page
    sem, pos = (torch.randn((n, kv, d), generator=g, device=DEV, dtype=torch.bfloat16) * torch.randint(1, 50, (n, kv, 1), generator=g, device=DEV).bfloat16() for d in (ds, dp))
    whole, parts = (B.new_paged4_cache(p, n_pages, page, 1, DEV) for _ in range(2))
    B.paged4_write(p, whole, sem, pos, slots)
    for i in range(0, n, part):
        B.paged4_write(p, parts, sem[i:i + part], pos[i:i + part], slots[i:i + part])
    for a, b in zip(whole.tensors, parts.tensors):
        assert a is None or torch.equal(a, b)
    assert int(whole.tensors[4].ne(0).sum()) == kv * int(((slots >= 0) & (slots < n_pages * page)).sum())      # (no row has an exponent byte of 0)
    a = [torch.full_like(x, 7.0) for x in (sem, pos)]
    B.paged4_read(p, whole, slots, *a)
    for i in range(0, n, part):
        b = [torch.full_like(x[i:i + part], 7.0) for x in (sem, pos)]
        B.paged4_read(p, whole, slots[i:i + part], *b)
        assert torch.equal(a[0][i:i + part], b[0]) and torch.equal(a[1][i:i + part], b[1])
