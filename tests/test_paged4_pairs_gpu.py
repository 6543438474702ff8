"""Decode attention over the paged 4-bit cache for the MLA shape with more than 64 query rows (CTA pairs, blocks of 128 rows)."""
import math

import numpy as np
import pytest
import torch

from tests.test_paged4_gpu import DEV, B, build, check_attend, i32, no_timeout, to_gpu  # noqa: F401

pytestmark = pytest.mark.gpu

# A weight's terms are e5m2 and e4m3 here: in [1, 2) the first one is off by at most 2^-3, the second one by half a step of what that
# leaves, 2^-8 in all.  The floor is half a step of 2^-9 where the largest weight is at least 2^8 (2^-18 of it), held to one step,
# 2^-17, for every 64 rows.
PAIR = dict(weight=2.0 ** -8, floor=2.0 ** -17)


@pytest.mark.parametrize("heads,q_len", [(65, 1), (66, 1), (100, 1), (127, 1), (128, 1), (129, 1), (13, 5), (40, 7), (128, 2), (1, 65), (3, 90)])
def test_rows_of_every_number(B, heads, q_len):
    states = [(0, 1), (2, 2 * 64 + 140), (0, 0), (1, 64 + q_len), (0, 129), (7, 7 * 64), (0, 640)]
    check_attend(B, "mla512", heads, 1, 32, states, 64, q_len, seed=heads + q_len, bias=0.6, **PAIR)


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("n", [1, 15, 16, 63, 64, 65, 127, 128, 129, 191, 255, 257, 513])
def test_lengths_around_tiles_and_halves_of_them(B, page, n):
    check_attend(B, "mla512", 72, 1, page, [(0, n), (0, n + 1)], 128, 1, seed=n, reps=False, **PAIR)


def test_representatives_tokens_and_what_lies_between(B):
    # the representatives' last tile, absent rows, the tokens' first tile; pages present in part
    for g, states in ((16, [(9, 9 * 16 + 1), (130, 130 * 16 + 70), (33, 33 * 16)]), (128, [(1, 128), (127, 127 * 128 + 3), (129, 129 * 128 + 500)])):
        check_attend(B, "mla512", 80, 1, 16, states, g, 2, seed=g, bias=-1.1, **PAIR)


def test_more_sequences_than_pairs(B):
    rng = np.random.RandomState(0)
    check_attend(B, "mla512", 96, 1, 16, [(0, int(n)) for n in rng.randint(0, 300, 300)], 64, 1, seed=2, **PAIR)


@pytest.mark.parametrize("rows", [9000, 30001])
def test_long_sequences_are_cut_and_merged(B, rows):
    check_attend(B, "mla512", 70, 1, 64, [(0, rows), (0, rows - 777)], 64, 1, seed=rows, reps=False, **PAIR)


@pytest.mark.parametrize("heads", [70, 128])
def test_growing_maximum(B, heads):
    def rise(pool, table):                                                     # logits of tens, rising along the sequence
        for e in range(table.shape[1]):
            pool.exp_sem[table[0, e]] = 119 + e // 3
    check_attend(B, "mla512", heads, 1, 64, [(0, 64 * 30)], 64, 1, seed=9, edit=rise, q_gain=0.05, **PAIR)
    check_attend(B, "mla512", heads, 1, 64, [(0, 64 * 30 + 5)], 64, 1, seed=9, q_gain=4.0, **PAIR)


def test_exponents_and_shifts_of_every_size(B):
    def small(pool, table):
        r = np.random.RandomState(7)
        pool.exp_sem[...] = r.choice([33, 60, 120, 127, 5], pool.exp_sem.shape)
        pool.shift_sem[...] = r.randint(0, 15, pool.shift_sem.shape) | (r.randint(0, 15, pool.shift_sem.shape) << 4)
        pool.shift_pos[...] = r.randint(0, 15, pool.shift_pos.shape) | (r.randint(0, 15, pool.shift_pos.shape) << 4)
    check_attend(B, "mla512", 90, 1, 16, [(0, 16 * 23 + 3), (0, 16 * 9)], 64, 1, seed=11, edit=small, **PAIR)


def test_entries_that_are_no_pages(B):
    def edit(pool, table):
        table[0, 1], table[0, 3], table[1, 0], table[1, 2] = -1, 1 << 30, 2 ** 31 - 1, -(2 ** 31)
    check_attend(B, "mla512", 128, 1, 32, [(0, 200), (0, 81), (0, 32)], 64, 2, seed=4, edit=edit, **PAIR)

    def none(pool, table):
        table[:] = -5
    check_attend(B, "mla512", 128, 1, 32, [(0, 200), (0, 81)], 64, 1, seed=4, edit=none, **PAIR)


def test_nan_and_infinity_stay_where_they_belong(B):
    heads, states = 128, [(0, 50), (0, 260), (0, 140), (0, 40)]
    pool, table = build("mla512", 1, 64, states, 64, 3)
    pool.shift_sem[table[1, 2], 0, 3, 2] |= 0xf0                               # one block of a latent: key and value
    q = [torch.randn((4, 1, heads, d), generator=torch.Generator().manual_seed(1)).bfloat16() for d in (512, 64)]
    q[0][3, 0, 5, 11], q[1][3, 0, heads - 1, 0] = float("inf"), float("nan")   # a row of either CTA
    p = B.make_params("mla", 4, 1, heads, 1, 512, 64, 64, 0, 0.07)
    cache, _ = to_gpu(B, pool, table)
    out, lse = B.decode_attention_paged4(p, cache, q[0].to(DEV), q[1].to(DEV), None, i32([s[1] for s in states]), want_lse=True)
    want = torch.zeros((4, heads), dtype=torch.bool)
    want[1] = True
    want[3, 5], want[3, heads - 1] = True, True
    assert torch.equal(torch.isnan(out[:, 0]).all(-1).cpu(), want) and torch.equal(torch.isnan(out[:, 0]).any(-1).cpu(), want)
    assert torch.equal(torch.isnan(lse[:, 0]).cpu(), want)


def test_flat_tail_behind_one_large_logit(B):
    # the tail's values are 1, the peak's 0; keys differ in the rope part alone
    page, n, heads = 128, 60000, 128
    p = B.make_params("mla", 1, 1, heads, 1, 512, 64, 64, 0, 1.0)
    n_pages = -(-n // page)
    cache = B.new_paged4_cache(p, n_pages, page, n_pages, DEV)
    sem, pos = torch.ones((n, 1, 512), dtype=torch.bfloat16, device=DEV), torch.zeros((n, 1, 64), dtype=torch.bfloat16, device=DEV)
    sem[5] = 0
    pos[5] = 1
    B.paged4_write(p, cache, sem, pos, torch.arange(n, dtype=torch.int32, device=DEV))
    cache.tensors[6].copy_(torch.arange(n_pages, dtype=torch.int32, device=DEV)[None])
    q_sem, q_pos = torch.zeros((1, 1, heads, 512), dtype=torch.bfloat16, device=DEV), torch.zeros((1, 1, heads, 64), dtype=torch.bfloat16, device=DEV)
    tops = [4.0, 9.0, 11.0, 12.0]
    for h in range(heads):
        q_pos[0, 0, h] = tops[h % 4] / 64
    out, lse = B.decode_attention_paged4(p, cache, q_sem, q_pos, None, i32([n]), want_lse=True)
    for h in (0, 1, 2, 3, 61, 66, 127):
        t = float(q_pos[0, 0, h].double().sum())
        l = math.exp(t) + n - 1
        share = (n - 1) / l
        assert float((out[0, 0, h].double() - share).abs().max()) <= (2.0 ** -8 + 2.0 ** -8) * share + 64 * 2.0 ** -17 * math.exp(t) / l
        assert abs(float(lse[0, 0, h]) - math.log(l)) < 1e-4


def test_rows_behind_the_batch_and_the_workspace_stay_as_they_are(B):
    states = [(0, 50), (0, 0), (0, 3333)]
    pool, table = build("mla512", 1, 16, states, 64, 3)
    p = B.make_params("mla", 3, 1, 100, 1, 512, 64, 64, 0, 0.1)
    cache, _ = to_gpu(B, pool, table)
    q = [torch.randn((3, 2, 100, d), device=DEV).bfloat16() for d in (512, 64)]
    for shift in (0, 8):                                                       # outputs on 32 bytes, and on 16 only
        flat = torch.full((4 * 2 * 100 * 512 + 8,), 7.0, dtype=torch.bfloat16, device=DEV)
        out, lse = flat[shift:shift + 4 * 2 * 100 * 512].view(4, 2, 100, 512), torch.full((4, 2, 100), 7.0, device=DEV)
        ws = torch.full((B.lca_paged4_workspace_bytes(p, cache, 2) + 64,), 0xff, dtype=torch.uint8, device=DEV)      # NaN everywhere
        n = ws.numel() - 64
        assert B.lca_decode_attention_paged4(p, cache, *q, 2, None, i32([s[1] for s in states]), out, lse, ws, n) == 0
        torch.cuda.synchronize()
        assert torch.all(out[3:] == 7) and torch.all(lse[3:] == 7) and torch.all(ws[n:] == 0xff)
        assert torch.isfinite(out).all() and torch.all(out[1] == 0)
        if shift:
            assert torch.equal(out[:3], first)
        first = out[:3].clone()


def test_the_same_bits_every_time_on_any_stream_and_in_a_graph(B):
    # signals cross from one CTA to the other: a missing one would show as a difference
    states = [(3, 3 * 64 + 900), (0, 2700), (2, 2 * 64 + 90), (0, 1)] * 20
    pool, table = build("mla512", 1, 64, states, 64, 8)
    p = B.make_params("mla", len(states), 1, 128, 1, 512, 64, 64, 0, 0.07)
    cache, _ = to_gpu(B, pool, table)
    g = torch.Generator().manual_seed(1)
    q = [torch.randn((len(states), 1, 128, d), generator=g).bfloat16().to(DEV) for d in (512, 64)]
    n_rep, n_tok = i32([s[0] for s in states]), i32([s[1] for s in states])
    first, _ = B.decode_attention_paged4(p, cache, *q, n_rep, n_tok)
    side, ws = torch.cuda.Stream(), B.workspace_paged4(p, cache, 1, DEV)
    ws2 = torch.empty_like(ws)
    a, b = torch.empty_like(first), torch.empty_like(first)
    torch.cuda.synchronize()
    for _ in range(30):                                                        # two at once, a workspace each
        B.decode_attention_paged4(p, cache, *q, n_rep, n_tok, out=a, ws=ws)
        B.decode_attention_paged4(p, cache, *q, n_rep, n_tok, out=b, ws=ws2, stream=side)
        torch.cuda.synchronize()
        assert torch.equal(a, first) and torch.equal(b, first)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.decode_attention_paged4(p, cache, *q, n_rep, n_tok, out=a, ws=ws)
    a.zero_()
    for _ in range(5):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(a, first)
    n_tok.sub_(1).clamp_(min=0)                                                # the graph reads what is there when it is replayed
    graph.replay()
    want, _ = B.decode_attention_paged4(p, cache, *q, n_rep, n_tok)
    torch.cuda.synchronize()
    assert torch.equal(a, want) and not torch.equal(a, first)
