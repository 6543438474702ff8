"""Paged 8-bit cache, host side: invalid calls are refused before anything is launched, workspace sizes, and the 64-bit
reference against itself (no GPU needed)."""
import numpy as np
import pytest
import torch

from tests import paged8_reference as R


@pytest.fixture(scope="module")
def B():
    from paper_2604_12452_b200 import build
    build.build()
    from paper_2604_12452_b200 import binding
    return binding


def cache(B, **kw):
    c = B.LcaPaged8(16, 16, 16, None, 16, 8, 16, 4)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


@pytest.fixture()
def p(B):
    return B.make_params("mla", 2, 1, 16, 1, 512, 64, 64, 64, 0.07)


def test_page_update_refusals(B, p):
    before = B.lca_launch_count()
    call = lambda c=None, n_rep=16, n_tok=16, hr=16, ht=16, fr=16, nf=16, sm=16, n=8, per=0, off=16, st=16, q=None: B.lca_page_update(  # noqa: E731
        q or p, c or cache(B), n_rep, n_tok, hr, ht, fr, nf, sm, n, per, off, st)
    for k in ("n_tok", "ht", "fr", "nf", "st"):
        assert call(**{k: None}) == -1, k
    assert call(n_rep=None) == -1 and call(hr=None) == -1                     # both or neither
    assert call(sm=None) == -1 and call(n=-1) == -1 and call(per=-1) == -1
    assert call(off=None) == -1                                               # packed slots need the offsets
    assert call(per=3) == -1                                                  # 8 != batch * 3
    assert call(c=cache(B, block_table=None)) == -1 and call(c=cache(B, table_width=0)) == -1 and call(c=cache(B, n_pages=0)) == -1
    assert call(c=cache(B, page_size=48)) == -2 and call(c=cache(B, page_size=0)) == -2
    assert call(c=cache(B, n_pages=1 << 28)) == -1                            # 2^28 * 16 rows
    assert call(c=cache(B, table_width=1 << 28)) == -1
    assert call(c=cache(B, page_size=128)) == -1                              # groups of 64 in pages of 128
    bad = B.make_params("mla", 0, 1, 16, 1, 512, 64, 64, 64, 0.07)
    assert call(q=bad) == -1
    assert B.lca_launch_count() == before


def test_write_refusals(B, p):
    before = B.lca_launch_count()
    call = lambda c=None, sem=16, pos=16, slots=16, n=8, q=None: B.lca_paged8_write(q or p, c or cache(B), sem, pos, slots, n)  # noqa: E731
    assert call(sem=None) == -1 and call(pos=None) == -1 and call(slots=None) == -1 and call(n=-1) == -1 and call(n=1 << 31) == -1
    assert call(n=0) == 0                                                     # nothing to write
    assert call(sem=24) == -3 and call(pos=24) == -3 and call(c=cache(B, pages_sem=24)) == -3
    assert call(c=cache(B, pages_pos=None)) == -1 and call(c=cache(B, scale_sem=None)) == -1
    assert call(c=cache(B, scale_pos=16)) == -1                               # MLA: one scale
    gqa = B.make_params("gqa", 2, 1, 16, 2, 128, 128, 64, 64, 0.07)
    assert call(q=gqa) == -1                                                  # GQA: two
    assert call(q=B.make_params("mla", 2, 1, 16, 1, 256, 64, 64, 64, 0.07)) == -2
    assert B.lca_launch_count() == before


def test_attention_and_update_refusals(B, p):
    before = B.lca_launch_count()
    big = 1 << 40
    call = lambda c=None, qs=16, qp=16, n=1, nr=16, nt=16, out=16, ws=16, wsb=big, q=None: B.lca_decode_attention_paged8(  # noqa: E731
        q or p, c or cache(B), qs, qp, n, nr, nt, out, None, ws, wsb)
    assert call(qs=None) == -1 and call(qp=None) == -1 and call(nt=None) == -1 and call(out=None) == -1 and call(n=0) == -1
    assert call(ws=None) == -1 and call(ws=24) == -1 and call(wsb=64) == -4
    assert call(qs=24) == -3 and call(qp=24) == -3 and call(out=24) == -3
    assert call(c=cache(B, page_size=128)) == -1                              # with representatives: group % page
    assert call(c=cache(B, block_table=None)) == -1 and call(c=cache(B, page_size=8)) == -2
    assert call(n=1 << 30) == -1                                              # 2^35 query rows
    need = B.lca_paged8_workspace_bytes(p, cache(B), 1)
    assert need > 0 and call(wsb=need - 1) == -4
    assert B.lca_paged8_workspace_bytes(p, cache(B), 0) == 0 and B.lca_paged8_workspace_bytes(p, cache(B, page_size=5), 1) == 0
    up = lambda c=None, tail=16, qbar=None, nr=16, nt=16, new=32, sem=16, pos=16, an=16, ws=16, wsb=big, stride=64, q=None: B.lca_decode_update_paged8(  # noqa: E731
        q or p, c or cache(B), tail, tail, stride, qbar, nr, nt, new, sem, pos, an, ws, wsb)
    assert up(nr=None) == -1 and up(nt=None) == -1 and up(new=None) == -1 and up(new=16) == -1      # n_rep_new is another array
    assert up(sem=None) == -1 and up(pos=None) == -1 and up(an=None) == -1 and up(tail=None) == -1
    assert up(stride=63) == -1 and up(ws=None) == -1 and up(wsb=8) == -4 and up(sem=24) == -3 and up(tail=24) == -3
    wide = B.make_params("mla", 2, 1, 16, 1, 512, 64, 512, 64, 0.07)
    assert up(q=wide, stride=512) == -2                                       # 512 rows of 576 bytes exceed shared memory
    assert B.lca_launch_count() == before


def test_descriptor_checks_element_sizes(B):
    t = torch.zeros((4, 1, 16, 512), dtype=torch.uint8)
    s = torch.ones((4, 1))
    with pytest.raises(ValueError):
        B.paged8_cache(t.float(), t[..., :64].contiguous(), s, None, torch.zeros((2, 3), dtype=torch.int32))
    with pytest.raises(ValueError):
        B.paged8_cache(t, t[..., :64].contiguous(), s, None, torch.zeros((2, 3), dtype=torch.int64))
    with pytest.raises(ValueError):
        B.paged8_cache(t, t[..., :64], s, None, torch.zeros((2, 3), dtype=torch.int32))               # not contiguous
    c = B.paged8_cache(t, t[..., :64].contiguous(), s, None, torch.zeros((2, 3), dtype=torch.int32))
    assert (c.n_pages, c.page_size, c.table_width) == (4, 16, 3)


def test_reference_codes_are_the_format():
    codes = torch.arange(256, dtype=torch.uint8)
    mine, theirs = R.decode(codes), codes.view(R.FP8).double().numpy()
    assert np.array_equal(np.isnan(mine), np.isnan(theirs)) and np.array_equal(mine[~np.isnan(mine)], theirs[~np.isnan(theirs)])
    x = np.concatenate([np.random.RandomState(0).randn(4000) * 100, np.linspace(-0.1, 0.1, 999), [448, 449, 464, 1e9, -1e9]])
    want = torch.from_numpy(x).clamp(-448, 448).to(R.FP8).view(torch.uint8).numpy()
    # torch converts by way of float32: no difference unless a value lies within 2^-24 of a boundary
    assert np.array_equal(R.encode(x), want)
    assert R.block_scale([0.0, np.nan, np.inf]) == 2.0 ** -100 and R.block_scale([448.0]) == 1.0 and R.block_scale([449.0]) == 2.0


def test_limits_of_tables_and_of_the_launch(B):
    big = B.make_params("mla", 1 << 20, 1, 16, 1, 512, 64, 64, 64, 0.07)
    before = B.lca_launch_count()
    wide = cache(B, table_width=1 << 11)                                      # 2^20 sequences x 2^11 entries
    assert B.lca_page_update(big, wide, 16, 16, 16, 16, 16, 16, None, 0, 0, None, 16) == -1
    assert B.lca_decode_attention_paged8(big, wide, 16, 16, 1, 16, 16, 16, None, 16, 1 << 40) == -1
    assert B.lca_decode_update_paged8(big, wide, None, None, 64, 16, 16, 16, 32, 16, 16, 16, 16, 1 << 40) == -1
    heads = B.make_params("gqa", 1, 1, 1 << 16, 1 << 16, 64, 64, 64, 64, 0.07)
    assert B.lca_paged8_write(heads, cache(B, n_pages=1 << 15, scale_pos=16), 16, 16, 16, 8) == -1       # 2^31 blocks
    assert B.lca_launch_count() == before


def test_helpers_refuse_tensors_that_are_not_on_the_current_device(B, p):
    c = B.new_paged8_cache(p, 8, 16, 4, "cpu")
    i = torch.zeros(64, dtype=torch.int32)
    before = B.lca_launch_count()
    with pytest.raises(ValueError):
        B.page_update(p, c, i, i, i, i, i, i, i, i, i)
    with pytest.raises(ValueError):
        B.paged8_write(p, c, torch.zeros((4, 1, 512), dtype=torch.bfloat16), torch.zeros((4, 1, 64), dtype=torch.bfloat16), i[:4])
    with pytest.raises(ValueError):
        B.decode_attention_paged8(p, c, torch.zeros((2, 1, 16, 512)).bfloat16(), torch.zeros((2, 1, 16, 64)).bfloat16(), i, i)
    with pytest.raises(ValueError):
        B.decode_update_paged8(p, c, None, None, i, i, qbar=torch.zeros((2, 1, 576)))
    assert B.lca_launch_count() == before


def test_descriptor_refuses_pools_that_do_not_fit_together(B):
    t, s = torch.zeros((4, 2, 16, 128), dtype=torch.uint8), torch.ones((4, 2))
    table = torch.zeros((2, 3), dtype=torch.int32)
    B.paged8_cache(t, t, s, s, table)
    for bad in ((t, t[:3], s, s, table), (t, t, s[:3], s, table), (t, t, s, torch.ones((4, 1)), table), (t, t, s, s, table[0]),
                (t, t, s.int(), s, table), (t, t, s, s, table.float()), (None, t, s, s, table)):
        with pytest.raises(ValueError):
            B.paged8_cache(*bad)
