"""Paged 8-bit cache on the GPU: the variants that only large calls take, calls from two threads, tensors of other shapes."""
import threading

import numpy as np
import pytest
import torch

from tests import paged8_reference as R
from tests.test_paged8_gpu import DEV, SHAPES, B, Tables, check_attend, check_write, compare, decode_case, i32, no_timeout, pool, to_gpu  # noqa: F401

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------------------- page update
@pytest.mark.parametrize("tokens", [[16 * 1000] * 3, [16 * 8] * 700, [16 * 2000 - 3], [16 * 2100], [1] * 40 + [16 * 900, 0, 16 * 1500 + 1],
                                    [16 * 9, 16 * 8, 5], [16 * 30] * 90 + [3] * 600,
                                    [1] * 300 + [16 * 700] + [20] * 100, [5] * 600 + [16 * 400 - 1, 0, 16 * 300]])
def test_page_update_of_many_entries(B, tokens):
    """Prompts, their condensation and their end: thousands of entries taken and given back, by few sequences and by many, one of
    them far longer than the others; with slots (the whole cluster) and without."""
    page = g = 16
    nb, width = len(tokens), -(-max(tokens) // page) + 1
    T = Tables(B, nb, width, sum(-(-t // page) for t in tokens) + nb + 5, page, g, seed=nb)
    full = [(0, t) for t in tokens]
    assert T.update(full, sum(tokens) + 9) == 0                                # everything taken, packed slots
    assert T.update([(0, 0)] * nb, 0, slots=False) == 0                        # everything given back
    assert int(T.n_free) == T.free.numel()
    assert T.update(full, 0, slots=False) == 0                                 # taken without slots
    half = [(t // g // 2, t) for t in tokens]
    assert T.update(half, sum(tokens)) == 0                                    # half of it condensed: given back and taken in one call
    assert T.update([(r, max(t - 40, r * g)) for r, t in half], 0, slots=False) == 0
    assert T.update(half, 40 * nb, per_seq=40) == 0                            # slots in places of their own
    assert T.update([(0, 0)] * nb, 3) == 0
    assert int(T.n_free) == T.free.numel()


def test_page_update_of_one_long_sequence_takes_no_longer_than_of_a_longer_one(B):
    """What one sequence takes and gives back is shared by a warp, whatever the number of entries of the whole call."""
    page, times = 16, []
    for pages in (2000, 2100):
        p = B.make_params("mla", 1, 1, 16, 1, 512, 64, page, 0, 1.0)
        table = torch.full((1, pages), -1, dtype=torch.int32, device=DEV)
        cache = B.paged8_cache(None, None, None, None, table, page_size=page, n_pages=pages)
        free, n_free, held, status = torch.arange(pages, dtype=torch.int32, device=DEV), i32([pages]), i32([0]), i32([-1])
        state = [i32([0]), i32([pages * page])]
        ev = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
        best = 1e9
        for _ in range(5):
            torch.cuda.synchronize()
            ev[0].record()
            for _ in range(10):
                for to in state[::-1]:
                    B.page_update(p, cache, None, to, None, held, free, n_free, None, None, status)
            ev[1].record()
            torch.cuda.synchronize()
            best = min(best, ev[0].elapsed_time(ev[1]) / 20)
        assert int(status) == 0 and int(n_free) == pages
        times.append(best * 1e3)
    print("2000 pages %.1f us, 2100 pages %.1f us" % tuple(times))
    assert times[0] <= 2 * times[1], times


@pytest.mark.parametrize("shift", [1, 2, 3])
def test_page_update_slot_maps_at_any_address(B, shift):
    tokens = [3000, 0, 17, 5001, 999, 1]
    page, width = 32, 160
    n = sum(tokens) + 7
    p = B.make_params("mla", len(tokens), 1, 16, 1, 512, 64, 64, 0, 1.0)
    perm = np.random.RandomState(shift).permutation(400)
    table = torch.full((len(tokens), width), -1, dtype=torch.int32, device=DEV)
    cache = B.paged8_cache(None, None, None, None, table, page_size=page, n_pages=400)
    whole = torch.full((n + 8,), -7, dtype=torch.int32, device=DEV)
    slots, status = whole[shift:shift + n], i32([-1])
    assert slots.data_ptr() % 16 != 0
    B.page_update(p, cache, None, i32(tokens), None, i32([0] * len(tokens)), i32(perm), i32([400]), slots, torch.empty(len(tokens) + 1, dtype=torch.int32, device=DEV),
                  status)
    ref = R.Pages(np.full((len(tokens), width), -1), perm, 400, page, 64, 400)
    want, _ = ref.update([(0, t) for t in tokens])
    flat = [s for w in want for s in w]
    assert int(status) == 0 and whole.cpu().tolist() == [-7] * shift + flat + [-1] * (n - len(flat)) + [-7] * (8 - shift)


# ------------------------------------------------------------------------------------------------------------- write
@pytest.mark.parametrize("shape,kv,page,n_rows", [("mla512", 1, 16, 20000), ("mla512", 1, 64, 80000), ("mla128", 1, 32, 40000),
                                                  ("gqa128", 8, 16, 10000), ("gqa128", 4, 32, 9000), ("gqa64", 8, 64, 30000), ("gqa64", 2, 128, 30000)])
def test_write_of_whole_prompts(B, shape, kv, page, n_rows):
    """So many rows that a CTA (a warp) looks for the runs of several rows: whole pages, runs that start inside one, padding."""
    variant, _, d_sem, d_pos = SHAPES[shape]
    r = np.random.RandomState(page + kv)
    slots, used = [], 0
    pages = iter(r.permutation(2 * n_rows // page + 64))
    while len(slots) < n_rows:
        kind = r.randint(0, 12)
        n, first = (page, 0) if kind < 8 else (r.randint(1, page + 1), 0) if kind < 10 else (0, 0)
        if kind == 10:
            first = r.randint(1, page)
            n = r.randint(1, page - first + 1)
        pg = int(next(pages))
        slots += [pg * page + first + k for k in range(n)] if kind < 11 else [-1] * r.randint(1, 40)
        used = max(used, pg + 1)
    slots = slots[:n_rows]
    gain = np.exp(2.0 * r.randn(n_rows, 1, 1)).astype(np.float32)
    sem, pos = (torch.from_numpy(r.standard_normal((n_rows, kv, d)).astype(np.float32) * gain).bfloat16() for d in (d_sem, d_pos))
    q = np.random.RandomState(3)
    code = lambda d: q.randint(0, 127, (used, kv, page, d), dtype=np.uint8)    # noqa: E731
    scale = lambda: (2.0 ** q.randint(-8, -4, (used, kv))).astype(np.float32)  # noqa: E731
    check_write(B, shape, kv, page, slots, sem, pos, (code(d_sem), code(d_pos), scale(), scale() if variant == "gqa" else None), used)


@pytest.mark.parametrize("shape,kv", [("mla512", 1), ("gqa128", 2)])
def test_write_after_a_rollback(B, shape, kv):
    """Draft rows, one of them large, are written, taken back, and others appended in their place: the scale covers every row
    written since the page was opened, and the rows before the drafts stay as they were rounded with it."""
    variant, _, d_sem, d_pos = SHAPES[shape]
    page, g = 16, 16
    p = B.make_params(variant, 1, 1, kv, kv, d_sem, d_pos, g, 0, 1.0)
    cache = B.new_paged8_cache(p, 4, page, 3, DEV)
    free, n_free, held, status = i32([2, 0, 3, 1]), i32([4]), i32([0]), i32([-1])
    gen = torch.Generator().manual_seed(3)
    ref, tok = [x.cpu().numpy().copy() if x is not None else None for x in cache.tensors[:4]], 0
    for to, gain in ((7, 1.0), (12, 40.0), (7, None), (9, 0.3), (20, 5.0), (16, None), (18, 0.1)):      # the last pair: at a page's place 0
        slots = torch.empty(max(to - tok, 1), dtype=torch.int32, device=DEV)
        B.page_update(p, cache, None, i32([to]), None, held, free, n_free, slots, i32([0, 0]), status)
        assert int(status) == 0
        if gain is not None:
            rows = [(torch.randn((to - tok, kv, d), generator=gen) * gain).bfloat16() for d in (d_sem, d_pos)]
            B.paged8_write(p, cache, rows[0].to(DEV), rows[1].to(DEV), slots)
            ref = list(R.write(*ref, rows[0].double().numpy(), rows[1].double().numpy(), slots.cpu().tolist(), page))
        tok = to
    for got, want in zip(cache.tensors[:4], ref):
        if want is not None:
            got = got.cpu().numpy()
            if want.dtype == np.uint8:
                got, want = np.where(got == 128, 0, got), np.where(want == 128, 0, want)
            assert np.array_equal(got, want)


# ------------------------------------------------------------------------------------------------------------ attend
@pytest.mark.parametrize("shape,heads,kv,nb", [("gqa64", 4, 2, 700), ("gqa128", 2, 1, 300), ("mla512", 2, 1, 600), ("mla512", 34, 1, 300), ("mla512", 66, 1, 300), ("mla128", 20, 1, 400),
                                               ("gqa64", 33, 1, 257)])
def test_attend_more_sequences_than_threads(B, shape, heads, kv, nb):
    r = np.random.RandomState(nb)
    states = [(0, int(n)) for n in r.randint(0, 40, nb)]
    for b in r.randint(0, nb, 12):
        states[b] = (0, int(r.randint(200, 900)))
    states[-1], states[0] = (2, 2 * 64 + 77), (0, 0)
    check_attend(B, shape, heads, kv, 16, states, 64, 1, seed=nb, bias=0.3)


# --------------------------------------------------------------------------------------------------------- refusals
def test_helpers_refuse_queries_of_other_strides(B):
    """More positions than the call reads would put every sequence but the first at the wrong place."""
    p, cache, q_sem, q_pos, n_rep, n_tok, qbar = decode_case(B, 16, 4)
    p.n_summary_q = 10
    tail = [torch.randn((3, 64, 16, d), device=DEV).bfloat16() for d in (512, 64)]
    two = [torch.cat([x, x], 1) for x in (q_sem, q_pos)]
    wide = torch.cat([q_pos, q_pos], 2)
    before = B.lca_launch_count()
    calls = [lambda: B.decode_update_paged8(p, cache, *tail, n_rep, n_tok),
             lambda: B.decode_update_paged8(p, cache, tail[0][:, :10].contiguous(), tail[1], n_rep, n_tok),
             lambda: B.decode_attention_paged8(p, cache, two[0], q_pos, n_rep, n_tok),
             lambda: B.decode_attention_paged8(p, cache, q_sem, wide, n_rep, n_tok),
             lambda: B.decode_attention_paged8(p, cache, q_sem, two[1], n_rep, n_tok)]
    for k, call in enumerate(calls):
        with pytest.raises(ValueError):
            call()
            pytest.fail("call %d was not refused" % k)
    assert B.lca_launch_count() == before
    # what fits is taken: the exact tensors, and more sequences than the call has
    a = B.decode_update_paged8(p, cache, *[x[:, :10].contiguous() for x in tail], n_rep, n_tok)
    b = B.decode_update_paged8(p, cache, *[torch.cat([x[:, :10], x[:1, :10]]) for x in tail], n_rep, n_tok)
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    assert torch.equal(B.decode_attention_paged8(p, cache, q_sem, q_pos, n_rep, n_tok)[0],
                       B.decode_attention_paged8(p, cache, torch.cat([q_sem, q_sem]), torch.cat([q_pos, q_pos]), n_rep, n_tok)[0])


def test_updates_of_two_group_sizes_from_two_threads(B):
    """The same kernel with two amounts of shared memory above 48 KB, called from two threads at once."""
    errors = []

    def worker(g):
        try:
            states = [(0, 2 * g)]
            pool_ = pool("mla512", 2 * g // 16, 16, 5, 1)
            cache, keep = to_gpu(B, pool_, torch.arange(2 * g // 16, dtype=torch.int32, device=DEV)[None].contiguous())
            p = B.make_params("mla", 1, 1, 16, 1, 512, 64, g, 16, 0.08)
            qbar = torch.randn((1, 1, 576), generator=torch.Generator().manual_seed(1)).to(DEV)
            n_rep, n_tok = i32([states[0][0]]), i32([states[0][1]])
            first = B.decode_update_paged8(p, cache, None, None, n_rep, n_tok, qbar=qbar)
            outs = dict(n_rep_new=first[0].clone(), rep_sem=first[1].clone(), rep_pos=first[2].clone(), anchor=first[3].clone(),
                        ws=B.workspace(p, B.LCA_WS_UPDATE, DEV))
            barrier.wait()
            for _ in range(4000):
                B.decode_update_paged8(p, cache, None, None, n_rep, n_tok, qbar=qbar, **outs)
        except Exception as e:                                                 # noqa: BLE001
            errors.append((g, e))

    barrier = threading.Barrier(4, timeout=60)
    threads = [threading.Thread(target=worker, args=(g,)) for g in (96, 368, 112, 352)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not errors, errors


@pytest.mark.parametrize("shape,kv,g", [("mla512", 1, 368), ("mla128", 1, 1056), ("gqa128", 2, 800), ("gqa64", 1, 1504)])
def test_update_of_the_largest_groups(B, shape, kv, g):
    """The largest group that shared memory holds, and the next one, which is refused."""
    variant, _, d_sem, d_pos = SHAPES[shape]
    page, n_pages = 16, g // 16 + 3
    pool_ = pool(shape, n_pages, page, 7, kv)
    table = np.random.RandomState(g).permutation(n_pages)[None, :g // 16 + 1].astype(np.int32)
    cache, _ = to_gpu(B, pool_, torch.from_numpy(table).to(DEV))
    dk = d_pos + (d_sem if variant == "mla" else 0)
    qbar = torch.randn((1, kv, dk), generator=torch.Generator().manual_seed(4)) * 0.2
    p = B.make_params(variant, 1, 1, kv, kv, d_sem, d_pos, g, 3, 0.08)
    new, sem, pos, anchor = B.decode_update_paged8(p, cache, None, None, i32([0]), i32([g + 3]), qbar=qbar.to(DEV))
    _, want_sem, want_pos, want_anchor = R.update(*pool_, table, [0], [g + 3], qbar.numpy(), g, 3, page, 0.08)
    assert new.tolist() == [1] and anchor.cpu().tolist() == want_anchor.tolist()
    vmax = np.abs(R.decode(torch.from_numpy(pool_[0]))).max() * pool_[2].max()
    for h in range(kv):                                                        # as in test_update_against_the_definition
        err = np.abs(sem[0, h].double().cpu().numpy() - want_sem[0, h])
        assert np.all(err <= 2.0 ** -8 * np.abs(want_sem[0, h]) + (g + 8) * 2.0 ** -23 * vmax)
        assert np.array_equal(pos[0, h].double().cpu().numpy(), want_pos[0, h])
    p.group_size = g + 16
    with pytest.raises(B.LcaError):
        B.decode_update_paged8(p, cache, None, None, i32([0]), i32([g + 3]), qbar=qbar.to(DEV))


# --------------------------------------------------------------------------------------------------- the run of calls
@pytest.mark.parametrize("variant,kv", [("mla", 1), ("gqa", 2)])
def test_the_loop_with_the_last_queries(B, variant, kv):
    """Prompts, then a decode loop in which the summary query is the mean of the last g queries: tables, slots, representatives,
    anchors and attention against the 64-bit statements, the group that is condensed chosen by queries of the loop itself."""
    g, w, page, heads, scale, lens = 16, 32, 16, 4 * kv, 0.06, [70, 33, 200]
    d_sem, d_pos = (512, 64) if variant == "mla" else (128, 128)
    nb, mla = len(lens), variant == "mla"
    gen = torch.Generator().manual_seed(17)
    rnd = lambda *s: torch.randn(s, generator=gen).bfloat16().to(DEV)          # noqa: E731
    p = B.make_params(variant, nb, max(lens), heads, kv, d_sem, d_pos, g, w, scale)
    T = sum(lens)
    q_sem, q_pos = (rnd(T, heads, d_sem) if mla else None), rnd(T, heads, d_pos)
    cond = B.condense_varlen(p, lens, q_sem, q_pos, rnd(T, kv, d_sem), rnd(T, kv, d_pos))
    ends = np.cumsum(lens)
    last = lambda q: torch.stack([q[e - g:e] for e in ends])                   # noqa: E731
    tail = [last(q_sem) if mla else None, last(q_pos)]
    m = [int(b - a) for a, b in zip(cond["group_offsets"], cond["group_offsets"][1:])]
    n_pages, width = 48, 32
    cache = B.new_paged8_cache(p, n_pages, page, width, DEV)
    sem_p, pos_p, ss, sp, table = cache.tensors
    free, n_free, held_rep, held_tok, status = i32(list(range(n_pages))), i32([n_pages]), i32([0] * nb), i32([0] * nb), i32([5])
    n_rep, n_tok = i32(m), i32(lens)
    slots, offsets = torch.empty(cond["cache_row_offsets"][-1], dtype=torch.int32, device=DEV), torch.empty(nb + 1, dtype=torch.int32, device=DEV)
    slot = torch.empty(nb, dtype=torch.int32, device=DEV)
    pages = R.Pages(table.cpu().numpy(), range(n_pages), n_pages, page, g, n_pages)

    def move(out, **kw):
        B.page_update(p, cache, n_rep, n_tok, held_rep, held_tok, free, n_free, out, offsets, status, **kw)
        want, st = pages.update(list(zip(n_rep.tolist(), n_tok.tolist())))
        flat = [s for x in want for s in (x + [-1] * (1 - len(x)) if kw else x)]
        assert int(status) == st == 0 and out.tolist() == flat and table.tolist() == pages.table

    move(slots)
    B.paged8_write(p, cache, cond["cache_sem"], cond["cache_pos"], slots)
    anchors = set()
    for step in range(50):
        n_tok += 1
        move(slot, rows_per_seq=1)
        B.paged8_write(p, cache, rnd(nb, kv, d_sem), rnd(nb, kv, d_pos), slot)
        qs, qp = (rnd(nb, 1, heads, d_sem) if mla else None), rnd(nb, 1, heads, d_pos)
        out, lse = B.decode_attention_paged8(p, cache, qs, qp, n_rep, n_tok, want_lse=True)
        pools = [None if x is None else x.cpu().numpy() for x in (sem_p, pos_p, ss, sp)]
        if step % 8 == 0:
            want = R.attend(None if qs is None else qs.double().cpu().numpy(), qp.double().cpu().numpy(), *pools, table.cpu().numpy(),
                            n_rep.tolist(), n_tok.tolist(), g, page, scale)
            compare(out, lse, *want, n=260, top=1.0)
        for t, q in zip(tail, (qs, qp)):
            if t is not None:
                t[:, step % g] = q[:, 0]
        new, rsem, rpos, anchor = B.decode_update_paged8(p, cache, *tail, n_rep, n_tok)
        mean = [t.double().view(nb, g, kv, heads // kv, -1).mean((1, 3)) for t in tail if t is not None]
        ref = R.update(*pools, table.cpu().numpy(), n_rep.tolist(), n_tok.tolist(), torch.cat(mean, -1).cpu().numpy(), g, w, page, scale)
        assert new.tolist() == ref[0].tolist() and anchor.tolist() == ref[3].tolist()
        for (b, h), row in ref[1].items():                                     # g + 8 roundings of 2^-24 each way, one to bf16
            assert np.all(np.abs(rsem[b, h].double().cpu().numpy() - row) <= 2.0 ** -8 * np.abs(row) + (g + 8) * 2.0 ** -23 * 8)
            assert np.array_equal(rpos[b, h].double().cpu().numpy(), ref[2][b, h])
            anchors.add(int(anchor[b, h]))
        n_rep.copy_(new)
        move(slot, rows_per_seq=1)
        B.paged8_write(p, cache, rsem, rpos, slot)
    assert len(anchors) > 3                                                    # the queries of the loop decide
