"""Paged 4-bit cache on the GPU against 64-bit statements of the same calls (tests/paged4_reference.py)."""
import math

import numpy as np
import pytest
import torch

from tests import paged4_reference as R
from tests import paged8_reference as R8

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


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def new_pool(shape, n_pages, page, seed, kv):
    variant, d_sem, d_pos = SHAPES[shape]
    return R.Pool(n_pages, kv, page, d_sem, d_pos, variant == "mla", seed)


def to_gpu(B, pool, table=None):
    t = [None if x is None else torch.from_numpy(np.ascontiguousarray(x)).to(DEV) for x in pool.arrays()]
    return B.paged4_cache(*t, None if table is None else torch.from_numpy(table).to(DEV)), t


# -------------------------------------------------------------------------------------------------- write, read back
def check_write(B, shape, kv, page, slots, rows_sem, rows_pos, pool):
    variant, d_sem, d_pos = SHAPES[shape]
    p = B.make_params(variant, 1, 1, kv, kv, d_sem, d_pos, 64, 0, 1.0)
    cache, t = to_gpu(B, pool)
    B.paged4_write(p, cache, rows_sem.to(DEV), rows_pos.to(DEV), i32(slots))
    pool.write(rows_sem.double().numpy(), rows_pos.double().numpy(), slots)
    torch.cuda.synchronize()
    got = [None if x is None else x.cpu().numpy() for x in t]
    for name, g, w in zip(("pages_sem", "pages_pos", "shift_sem", "shift_pos", "exp_sem", "exp_pos"), got, pool.arrays()):
        if w is None:
            continue
        if name.startswith("pages"):                       # NaN blocks hold any codes, both zeros are the same value
            g, w = R.unpack(g), R.unpack(w)
            g, w = np.where(g == 8, 0, g), np.where(w == 8, 0, w)
            s = R.unpack_shifts(pool.shift_sem if name == "pages_sem" else pool.shift_pos).repeat(32, -1)
            g, w = np.where(s == 15, 0, g), np.where(s == 15, 0, w)
        assert np.array_equal(g, w), (name, int((g != w).sum()), np.argwhere(g != w)[:3])
    # read back, in another order and with slots that are none
    want = {"sem": pool.sem(), "pos": pool.pos()}
    ask = [s for s in reversed(slots)] + [slots[0], -1, pool.pages_sem.shape[0] * page, 3]
    sem, pos = (torch.full((len(ask), kv, d), 7.0, dtype=torch.bfloat16, device=DEV) for d in (d_sem, d_pos))
    B.paged4_read(p, cache, i32(ask), sem, pos)
    for x, w in ((sem, want["sem"]), (pos, want["pos"])):
        x = x.double().cpu().numpy()
        w = torch.from_numpy(w).float().bfloat16().double().numpy()            # 2^128: infinity
        for i, s in enumerate(ask):
            ref = w[s // page, :, s % page] if 0 <= s < w.shape[0] * page else np.full(x[i].shape, 7.0)
            assert np.array_equal(x[i], ref, equal_nan=True), (i, s)


@pytest.mark.parametrize("shape,kv", [("mla512", 1), ("mla128", 1), ("gqa128", 3), ("gqa64", 2), ("gqa64", 1), ("gqa128", 8), ("gqa128", 16), ("gqa64", 8),
                                      ("gqa64", 9), ("gqa128", 5)])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_write_and_read_rows_in_any_order(B, shape, kv, page):
    variant, d_sem, d_pos = SHAPES[shape]
    r = np.random.RandomState(page + kv)
    n_pages = 7
    slots = [int(s) for s in r.permutation(n_pages * page)[:67]]
    slots[5:5] = [-1, n_pages * page, 2 ** 31 - 1, -(2 ** 31)]
    T = len(slots)
    gain = np.exp(2.5 * r.randn(T, 1, 1))
    sem, pos = (torch.from_numpy(r.randn(T, kv, d) * gain * np.exp(r.randn(d // 32).repeat(32) * 2)).bfloat16() for d in (d_sem, d_pos))
    check_write(B, shape, kv, page, slots, sem, pos, new_pool(shape, n_pages, page, 3, kv))


@pytest.mark.parametrize("shape,kv", [("mla512", 1), ("gqa128", 2), ("gqa64", 1), ("mla128", 1), ("gqa128", 8), ("gqa64", 8), ("gqa128", 3)])
def test_write_extreme_values(B, shape, kv):
    variant, d_sem, d_pos = SHAPES[shape]
    r = np.random.RandomState(5)
    T, page = 40, 16
    sem, pos = (torch.from_numpy(r.randn(T, kv, d)).float() for d in (d_sem, d_pos))
    for t, (a, b) in enumerate([(0.0, 0.0), (1e-38, 1e-38), (1e-40, 0.0), (3.0e37, 1.0), (1.0, 3.0e37), (2 ** -95, 2 ** -99), (2 ** -92, 2 ** -100), (0.0, 1.0)]):
        sem[t] *= a
        pos[t] *= b
    for t, top in enumerate([6.0, 6.03125, 3.0, 3.015625, 5.96875, 12.0]):      # on, above and below the border of a scale
        sem[8 + t] = sem[8 + t].clamp(-2, 2)
        sem[8 + t, :, 1] = -top
    grid = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0])          # ties
    for t in range(4):
        v = torch.cat([grid, -grid, torch.nextafter(grid.bfloat16(), torch.zeros(8).bfloat16()).float(),
                       torch.nextafter(grid.bfloat16(), torch.full((8,), 9.0).bfloat16()).float().clamp(max=6.0)])
        sem[14 + t] = v.repeat(d_sem // 32) * 2.0 ** (3 * t - 4)
        pos[14 + t] = -v.repeat(d_pos // 32) * 2.0 ** (3 * t - 4)
    for t in range(12):                                                        # blocks far below the row's largest
        sem[18 + t, :, 32:] *= 2.0 ** (-2 * t)
        pos[18 + t] *= 2.0 ** (-3 * t)
    sem[30, :, 3], sem[30, :, 5], sem[31, :, 40], pos[32, :, 33] = float("inf"), float("-inf"), float("nan"), float("nan")
    sem[33], pos[33] = float("inf"), float("nan")
    sem[34], pos[34, :, :32] = float("nan"), float("-inf")
    check_write(B, shape, kv, page, list(range(2, 2 + T)), sem.bfloat16(), pos.bfloat16(), new_pool(shape, 4, page, 4, kv))


@pytest.mark.parametrize("shape,n", [("mla512", 4097), ("mla512", 4106), ("mla128", 4099), ("mla128", 5000)])
def test_write_and_read_more_rows_than_a_warp_has_for_itself(B, shape, n):
    # several rows to a warp: neighbours of every kind side by side, rows without a slot among them, a last warp that is not full
    _, d_sem, d_pos = SHAPES[shape]
    r = np.random.RandomState(n)
    page, n_pages = 64, n // 64 + 3
    slots = r.permutation(n_pages * page)[:n]
    slots[r.permutation(n)[:n // 9]] = -1
    slots[[1, 6, n - 2]] = [n_pages * page, 2 ** 31 - 1, -(2 ** 31)]
    sem, pos = (torch.from_numpy(r.randn(n, 1, d) * np.exp(3 * r.randn(n, 1, 1)) * np.exp(r.randn(d // 32).repeat(32) * 2)).bfloat16() for d in (d_sem, d_pos))
    for x in (sem, pos):
        for value in (float("inf"), float("-inf"), float("nan"), 0.0, 1e-40, 3e38):
            x[torch.from_numpy(r.permutation(n)[:n // 20]), 0, r.randint(x.shape[-1])] = value
        x[torch.from_numpy(r.permutation(n)[:n // 20])] = 0.0
        x[torch.from_numpy(r.permutation(n)[:n // 50])] = float("nan")
    check_write(B, shape, 1, page, [int(s) for s in slots], sem, pos, new_pool(shape, n_pages, page, 3, 1))


def test_read_gives_what_the_bytes_say_for_every_byte(B):
    # every exponent, shift and code, also those that no write produces
    p = B.make_params("gqa", 1, 1, 1, 1, 64, 64, 64, 0, 1.0)
    pool = new_pool("gqa64", 16, 16, 0, 1)
    e = np.arange(256, dtype=np.int64).reshape(16, 1, 16)
    pool.exp_sem, pool.exp_pos = e.astype(np.uint8), ((e * 7 + 3) % 256).astype(np.uint8)
    pool.shift_sem[...] = ((e * 5) % 256)[..., None].astype(np.uint8)
    pool.shift_pos[...] = ((e * 11 + 1) % 256)[..., None].astype(np.uint8)
    pool.pages_sem[...] = np.random.RandomState(0).randint(0, 256, pool.pages_sem.shape)
    cache, _ = to_gpu(B, pool)
    sem, pos = B.paged4_read(p, cache, i32(list(range(256))))
    for x, w in ((sem, pool.sem()), (pos, pool.pos())):
        w = w.transpose(0, 2, 1, 3).reshape(256, 1, 64)
        ref = torch.from_numpy(w).float().bfloat16().double().numpy()          # 2^128 and more: infinity
        assert np.array_equal(x.double().cpu().numpy(), ref, equal_nan=True)


def test_many_rows_and_empty_calls(B):
    for shape, kv, n in (("mla512", 1, 70001), ("gqa128", 8, 9001), ("gqa64", 3, 33333)):
        variant, d_sem, d_pos = SHAPES[shape]
        p = B.make_params(variant, 1, 1, kv, kv, d_sem, d_pos, 64, 0, 1.0)
        page = 64
        n_pages = -(-n // page) + 1
        cache = B.new_paged4_cache(p, n_pages, page, 1, DEV)
        g = torch.Generator(device=DEV).manual_seed(1)
        # rows that the format holds exactly: codes times powers of two
        lev = torch.tensor([0.0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.5, -1, -1.5, -2, -3, -4, -6], device=DEV)
        make = lambda d: lev[torch.randint(0, 15, (n, kv, d), generator=g, device=DEV)] * torch.exp2(torch.randint(-3, 4, (n, kv, 1), generator=g, device=DEV).float())  # noqa: E731
        sem, pos = make(d_sem).bfloat16(), make(d_pos).bfloat16()
        sem[..., 0] = 6.0 * 2.0 ** 4                                           # the same exponent for all: nothing below 2^-14 of it
        pos[..., 0] = 6.0 * 2.0 ** 4
        slots = torch.randperm(n_pages * page, generator=g, device=DEV)[:n].int()
        B.paged4_write(p, cache, sem, pos, slots)
        a, b = B.paged4_read(p, cache, slots)
        keep = torch.ones(d_sem, dtype=torch.bool, device=DEV)
        keep[:32] = False                                                      # the first block carries the large element
        assert torch.equal(a[..., keep], sem[..., keep]) and torch.equal(a[..., 0], sem[..., 0])
        keep = torch.ones(d_pos, dtype=torch.bool, device=DEV)
        keep[:32] = False
        assert torch.equal(b[..., keep], pos[..., keep])
        B.paged4_write(p, cache, sem[:0], pos[:0], slots[:0])
        B.paged4_read(p, cache, slots[:0], sem[:0], pos[:0])


# ------------------------------------------------------------------------------------------------------------ attend
def build(shape, kv, page, states, g, seed, spare=3):
    """Cache of sequences in the given states [(n_rep, n_tok)]; every row that is not present is NaN."""
    r = np.random.RandomState(seed)
    width = max(1, -(-max(t for _, t in states) // page))
    need = [(b, e) for b, (n, t) in enumerate(states) for e in range(width)
            if any(R8.present(n, t, g, x) for x in range(e * page, (e + 1) * page))]
    n_pages = len(need) + spare
    ids = r.permutation(n_pages)[:len(need)]
    table = np.full((len(states), width), -1, dtype=np.int32)
    pool = new_pool(shape, n_pages, page, seed + 1, kv)
    keep = np.zeros((n_pages, page), dtype=bool)
    for (b, e), i in zip(need, ids):
        table[b, e] = i
        keep[i] = [R8.present(*states[b], g, x) for x in range(e * page, (e + 1) * page)]
    gone = np.broadcast_to(~keep[:, None], (n_pages, kv, page))
    for x in (pool.shift_sem, pool.shift_pos, pool.exp_sem, pool.exp_pos):
        if x is not None:
            x[gone] = 0xff
    return pool, table


def check_attend(B, shape, heads, kv, page, states, g, q_len, seed=0, bias=0.0, reps=True, impl=0, edit=None, q_gain=1.0, softmax_scale=None,
                 weight=2.0 ** -9, floor=2.0 ** -18):
    variant, d_sem, d_pos = SHAPES[shape]
    pool, table = build(shape, kv, page, states, g, seed)
    if edit:
        edit(pool, table)
    r = torch.Generator().manual_seed(seed)
    nb = len(states)
    scale = softmax_scale or 1.0 / math.sqrt(192.0 if variant == "mla" else d_pos)
    q_pos = (torch.randn((nb, q_len, heads, d_pos), generator=r) * q_gain).bfloat16()
    q_sem = (torch.randn((nb, q_len, heads, d_sem), generator=r) * q_gain).bfloat16() if variant == "mla" else None
    p = B.make_params(variant, nb, 1, heads, kv, d_sem, d_pos, g, 0, scale, rep_logit_bias=bias)
    cache, keep = to_gpu(B, pool, table)
    n_rep = i32([s[0] for s in states]) if reps else None
    old = B.lca_set_attention_impl(impl)
    try:
        out, lse = B.decode_attention_paged4(p, cache, None if q_sem is None else q_sem.to(DEV), q_pos.to(DEV), n_rep, i32([s[1] for s in states]),
                                             want_lse=True)
        torch.cuda.synchronize()
    finally:
        B.lca_set_attention_impl(old)
    want, want_lse, absv, big = R.attend(None if q_sem is None else q_sem.double().numpy(), q_pos.double().numpy(), pool, table,
                                         [s[0] for s in states] if reps else [0] * nb, [s[1] for s in states], g, scale, bias)
    compare(out, lse, want, want_lse, absv, big, n=max(t for _, t in states), weight=weight, floor=floor)
    return out, lse, want


def compare(out, lse, want, want_lse, absv, big, n, weight=2.0 ** -9, floor=2.0 ** -18):
    """Logit error e: a query element is off by 2^-17 of its row's largest, so the product sum by 2^-17 max|q| sum|k| (`big`, with
    the softmax scale); fp32 sums of up to 2 * 576 products (2^-24 each, worst order) add 2^-13 of the same; exp2 / log2 and
    the scale products 2^-20 of the logits, which `big` bounds as well.  The cached values enter exactly.  A weight is then off
    by the factor 2 e, its two terms by 2^-9, the result by the same of sum p|v| (numerator) and of |out| (row sum, logit part
    only); a weight's floor is half a step of 2^-13 where the largest is at least 2^5 (2^-19 of it), rounded with offsets that leave at most a
    few dozen steps of a tail (held here to one step for every 64 rows, and one more); bf16 rounds by 2^-8 |out| at most."""
    got, gl = out.double().cpu().numpy(), lse.double().cpu().numpy()
    e = big * (2.0 ** -17 + 2.0 ** -13 + 2.0 ** -20)
    empty = ~np.isfinite(want_lse)
    assert np.array_equal(np.isneginf(gl), empty) and np.all(got[empty] == 0)
    dl = np.abs(gl[~empty] - want_lse[~empty])
    assert np.all(dl <= e[~empty] + 1e-6 * np.abs(want_lse[~empty]) + 1e-6), dl.max()
    tol = absv * (weight + 4 * e[..., None]) + 2.0 ** -8 * np.abs(want) + floor * (1 + n / 64) * absv.max(initial=0) + 1e-30
    bad = np.abs(got - want) > tol
    assert not bad.any(), (int(bad.sum()), float(np.abs(got - want).max()), np.argwhere(bad)[:4])


STATES = [(0, 1), (0, 130), (3, 3 * 64 + 70), (0, 0), (5, 5 * 64 + 1), (17, 17 * 64 + 333)]


@pytest.mark.parametrize("impl", [1, 0])
@pytest.mark.parametrize("shape,heads,kv", [("mla512", 16, 1), ("mla512", 3, 1), ("mla512", 8, 1), ("mla512", 20, 1), ("mla512", 128, 1), ("mla512", 40, 1),
                                            ("mla128", 8, 1), ("mla128", 4, 1), ("mla128", 16, 1), ("mla128", 32, 1), ("mla128", 64, 1), ("gqa128", 8, 2),
                                            ("gqa128", 2, 2), ("gqa128", 15, 3), ("gqa128", 16, 1), ("gqa128", 32, 1), ("gqa128", 70, 1), ("gqa64", 8, 4), ("gqa64", 24, 1),
                                            ("gqa64", 24, 2), ("gqa64", 14, 2), ("gqa64", 64, 1)])
def test_attend_head_layouts(B, impl, shape, heads, kv):
    check_attend(B, shape, heads, kv, 64, STATES, 64, 1, seed=heads, bias=0.7, impl=impl)


@pytest.mark.parametrize("shape,heads,kv,q_len", [("mla512", 16, 1, 2), ("mla512", 24, 1, 5), ("gqa128", 8, 2, 4), ("gqa128", 6, 2, 7), ("gqa64", 4, 2, 33),
                                                  ("mla128", 2, 1, 16), ("mla512", 128, 1, 3), ("mla512", 2, 1, 2), ("gqa64", 6, 3, 3)])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_attend_several_queries_and_page_sizes(B, shape, heads, kv, q_len, page):
    # short sequences leave the first queries without a row
    states = [(0, 1), (0, 3), (2, 2 * 128 + 140), (1, 128 + q_len), (0, 257), (0, 0), (3, 3 * 128)]
    check_attend(B, shape, heads, kv, page, states, 128, q_len, seed=page + q_len, bias=-0.4)


@pytest.mark.parametrize("shape,heads,kv,rows,batch", [("mla512", 16, 1, 9000, 1), ("mla512", 33, 1, 21000, 1), ("mla512", 128, 1, 3000, 5), ("gqa128", 8, 2, 5003, 3),
                                                       ("mla512", 64, 1, 2600, 2), ("gqa64", 3, 1, 40001, 1), ("gqa128", 40, 2, 7000, 2)])
def test_attend_long_sequences_are_cut_and_merged(B, shape, heads, kv, rows, batch):
    check_attend(B, shape, heads, kv, 64, [(0, rows - 700 * i) for i in range(batch)], 64, 1, seed=rows, reps=False)


def test_attend_many_units_on_few_ctas(B):
    # more (sequence, KV head) units than CTAs, lengths from nothing to several tiles; more sequences than one warp's sums
    rng = np.random.RandomState(0)
    check_attend(B, "gqa128", 16, 8, 16, [(0, int(n)) for n in rng.randint(0, 400, 90)], 64, 1, seed=2)
    check_attend(B, "gqa64", 4, 2, 16, [(0, int(n)) for n in rng.randint(0, 200, 300)], 64, 1, seed=2)
    check_attend(B, "mla512", 16, 1, 16, [(0, int(n)) for n in rng.randint(0, 300, 310)], 64, 1, seed=2)


@pytest.mark.parametrize("shape,heads,kv", [("gqa128", 8, 1), ("gqa128", 4, 1), ("mla512", 16, 1), ("mla512", 20, 1), ("gqa64", 16, 1)])
def test_attend_growing_maximum(B, shape, heads, kv):
    # logits of tens, rising along the sequence: the running maximum is raised again and again, O rescaled
    def rise(pool, table):
        for e in range(table.shape[1]):
            for x in ([pool.exp_sem] if pool.mla else [pool.exp_pos, pool.exp_sem]):
                x[table[0, e]] = 119 + e // 3
    check_attend(B, shape, heads, kv, 64, [(0, 64 * 30)], 64, 1, seed=9, edit=rise, q_gain=0.05)
    check_attend(B, shape, heads, kv, 64, [(0, 64 * 30 + 5)], 64, 1, seed=9, q_gain=4.0)


def test_attend_exponents_and_shifts_of_every_size(B):
    def wild(pool, table):
        r = np.random.RandomState(7)
        pool.exp_sem[...] = r.choice([33, 60, 127, 160, 5], pool.exp_sem.shape)
        pool.shift_sem[...] = r.randint(0, 15, pool.shift_sem.shape) | (r.randint(0, 15, pool.shift_sem.shape) << 4)
        pool.shift_pos[...] = r.randint(0, 15, pool.shift_pos.shape) | (r.randint(0, 15, pool.shift_pos.shape) << 4)
    check_attend(B, "gqa128", 8, 2, 16, [(0, 16 * 23 + 3)], 64, 1, seed=11, edit=wild)

    def small(pool, table):                                                    # MLA: key and value share the exponent
        wild(pool, table)
        pool.exp_sem[...] = np.random.RandomState(8).choice([33, 60, 120, 127, 5], pool.exp_sem.shape)
    for heads in (16, 30):
        check_attend(B, "mla512", heads, 1, 16, [(0, 16 * 23 + 3)], 64, 1, seed=11, edit=small)


def test_attend_entries_that_are_no_pages(B):
    def edit(pool, table):
        table[0, 1], table[0, 3], table[1, 0], table[1, 2] = -1, 1 << 30, 2 ** 31 - 1, -(2 ** 31)
    for impl in (0, 1):
        check_attend(B, "gqa128", 8, 2, 32, [(0, 200), (0, 81), (0, 32)], 64, 2, seed=4, edit=edit, impl=impl)

    def none(pool, table):
        table[:] = -5
    check_attend(B, "mla512", 16, 1, 32, [(0, 200), (0, 81)], 64, 1, seed=4, edit=none)


@pytest.mark.parametrize("heads", [16, 40])
def test_attend_nan_and_infinity_stay_where_they_belong(B, heads):
    states = [(0, 50), (0, 260), (0, 140), (0, 40)]
    pool, table = build("mla512", 1, 64, states, 64, 3)
    pool.shift_sem[table[1, 2], 0, 3, 2] |= 0xf0                                # one block of a latent: key and value
    q = [torch.randn((4, 1, heads, d), generator=torch.Generator().manual_seed(1)).bfloat16() for d in (512, 64)]
    q[0][3, 0, 5, 11], q[1][3, 0, heads - 1, 0] = float("inf"), float("nan")
    p = B.make_params("mla", 4, 1, heads, 1, 512, 64, 64, 0, 0.07)
    cache, _ = to_gpu(B, pool, table)
    out, lse = B.decode_attention_paged4(p, cache, q[0].to(DEV), q[1].to(DEV), None, i32([s[1] for s in states]), want_lse=True)
    want = torch.zeros((4, heads), dtype=torch.bool)
    want[1] = True
    want[3, 5], want[3, heads - 1] = True, True
    assert torch.equal(torch.isnan(out[:, 0]).all(-1).cpu(), want) and torch.equal(torch.isnan(out[:, 0]).any(-1).cpu(), want)
    assert torch.equal(torch.isnan(lse[:, 0]).cpu(), want)


def test_attend_nan_in_values_of_one_head(B):
    states = [(0, 50), (0, 60), (0, 30)]
    pool, table = build("gqa128", 2, 16, states, 64, 3)
    pool.shift_sem[table[1, 0], 1, 3, 1] |= 0x0f                               # V of sequence 1, head 1, columns 64 .. 95
    pool.shift_pos[table[2, 1], 0, 2, 0] |= 0xf0                               # K of sequence 2, head 0
    q = torch.randn((3, 1, 8, 128), generator=torch.Generator().manual_seed(1)).bfloat16()
    p = B.make_params("gqa", 3, 1, 8, 2, 128, 128, 64, 0, 0.1)
    cache, _ = to_gpu(B, pool, table)
    out, lse = B.decode_attention_paged4(p, cache, None, q.to(DEV), None, i32([s[1] for s in states]), want_lse=True)
    want = torch.zeros((3, 8, 128), dtype=torch.bool)
    want[1, 4:, 64:96] = True
    want[2, :4] = True
    assert torch.equal(torch.isnan(out[:, 0]).cpu(), want)
    assert torch.equal(torch.isnan(lse[:, 0]).cpu(), want.all(-1))


def test_attend_counters_beyond_the_table_are_clamped(B):
    pool, table = build("mla128", 1, 16, [(0, 64), (4, 64)], 16, 3)
    p = B.make_params("mla", 2, 1, 8, 1, 128, 64, 16, 0, 0.1)
    cache, _ = to_gpu(B, pool, table)
    g = torch.Generator().manual_seed(1)
    q = [torch.randn((2, 1, 8, d), generator=g).bfloat16().to(DEV) for d in (128, 64)]
    a, _ = B.decode_attention_paged4(p, cache, *q, i32([0, 4]), i32([64, 64]))
    b, _ = B.decode_attention_paged4(p, cache, *q, i32([-3, 4]), i32([2 ** 31 - 1, 70]))
    assert torch.equal(a, b)
    c, l = B.decode_attention_paged4(p, cache, *q, i32([2 ** 31 - 1, 5]), i32([-7, -2 ** 31]), want_lse=True)
    assert torch.all(c == 0) and torch.all(torch.isneginf(l))


def test_attend_rows_behind_the_batch_stay_as_they_are(B):
    pool, table = build("gqa128", 2, 16, [(0, 50), (0, 0), (0, 333)], 64, 3)
    p = B.make_params("gqa", 3, 1, 6, 2, 128, 128, 64, 0, 0.1)
    cache, _ = to_gpu(B, pool, table)
    q = torch.randn((3, 2, 6, 128), device=DEV).bfloat16()
    out = torch.full((5, 2, 6, 128), 7.0, dtype=torch.bfloat16, device=DEV)
    lse = torch.full((5, 2, 6), 7.0, device=DEV)
    ws = torch.full((B.lca_paged4_workspace_bytes(p, cache, 2) + 64,), 0xff, dtype=torch.uint8, device=DEV)      # NaN everywhere
    n = ws.numel() - 64
    assert B.lca_decode_attention_paged4(p, cache, None, q, 2, None, i32([50, 0, 333]), out, lse, ws, n) == 0
    torch.cuda.synchronize()
    assert torch.all(out[3:] == 7) and torch.all(lse[3:] == 7) and torch.all(ws[n:] == 0xff)
    assert torch.isfinite(out).all()


def test_attend_flat_tail_behind_one_large_logit(B):
    # one key far above 120000 equal ones (all keys zero): the tail's share comes from weights below the floor of a single
    # one, which must not all round the same way.  The reference is the closed form; values of the tail are 1, of the peak 0.
    page, n = 128, 120000
    p = B.make_params("gqa", 1, 1, 4, 1, 64, 64, 64, 0, 1.0)
    n_pages = -(-n // page)
    cache = B.new_paged4_cache(p, n_pages, page, n_pages, DEV)
    slots = torch.arange(n, dtype=torch.int32, device=DEV)
    sem, pos = torch.ones((n, 1, 64), dtype=torch.bfloat16, device=DEV), torch.zeros((n, 1, 64), dtype=torch.bfloat16, device=DEV)
    sem[5] = 0
    pos[5] = 1
    B.paged4_write(p, cache, sem, pos, slots)
    cache.tensors[6].copy_(torch.arange(n_pages, dtype=torch.int32, device=DEV)[None])
    q = torch.zeros((1, 1, 4, 64), dtype=torch.bfloat16, device=DEV)
    for h, top in enumerate([4.0, 9.0, 12.0, 13.5]):
        q[0, 0, h] = top / 64
    out, lse = B.decode_attention_paged4(p, cache, None, q, None, i32([n]), want_lse=True)
    for h in range(4):
        t = float(q[0, 0, h].double().sum())
        l = math.exp(t) + n - 1
        share = (n - 1) / l
        # floor 2^-18 of the largest weight, exp(t), for at most 64 steps of the offsets in the range that holds the peak; elsewhere every
        # weight is the largest (2^-9), and bf16 rounds by 2^-8
        assert abs(float(out[0, 0, h, 0]) - share) <= (2.0 ** -9 + 2.0 ** -8) * share + 64 * 2.0 ** -18 * math.exp(t) / l
        assert abs(float(lse[0, 0, h]) - math.log(l)) < 1e-4


@pytest.mark.parametrize("shape,heads,kv", [("mla512", 16, 1), ("mla512", 128, 1), ("gqa128", 8, 2), ("gqa64", 32, 2)])
def test_whole_rows_are_as_exact_as_two_terms_make_them(B, shape, heads, kv):
    # bf16's rounding alone leaves about 2^-9 / sqrt(3) of a row; single 8-bit terms of queries or weights would leave over 2^-6
    out, _, want = check_attend(B, shape, heads, kv, 64, [(0, 3000), (0, 1111)], 64, 1, seed=1)
    d = out.double().cpu().numpy() - want
    assert np.all(np.linalg.norm(d, axis=-1) <= 2.0 ** -8 * np.linalg.norm(want, axis=-1))


def test_pages_behind_4_gb(B):
    page, kv = 128, 8
    p = B.make_params("gqa", 2, 1, 16, kv, 128, 128, 128, 0, 0.1)
    n_pages = (5 << 30) // (kv * page * 64)
    cache = B.new_paged4_cache(p, n_pages, page, 4, DEV)
    table = cache.tensors[6]
    table.copy_(i32([[n_pages - 1, 3, n_pages - 2, n_pages - 7], [n_pages - 4, n_pages // 2 + 1, 0, n_pages - 9]]))
    g = torch.Generator(device=DEV).manual_seed(1)
    n_tok = [500, 333]
    x = torch.cat([torch.arange(n, device=DEV) for n in n_tok])
    b = torch.cat([torch.full((n,), i, device=DEV) for i, n in enumerate(n_tok)])
    slots = (table[b, x // page].long() * page + x % page).int()
    sem, pos = (torch.randn((x.numel(), kv, 128), generator=g, device=DEV).bfloat16() for _ in range(2))
    B.paged4_write(p, cache, sem, pos, slots)
    v, k = B.paged4_read(p, cache, slots)
    assert float((v.float() - sem.float()).norm() / sem.float().norm()) < 0.15
    q = torch.randn((2, 1, 16, 128), generator=g, device=DEV).bfloat16()
    out, _ = B.decode_attention_paged4(p, cache, None, q, None, i32(n_tok))
    for i in range(2):
        z = torch.einsum("hrd,xhd->hrx", q[i, 0].view(kv, 2, 128).double(), k[b == i].double()) * 0.1
        want = torch.einsum("hrx,xhd->hrd", torch.softmax(z, -1), v[b == i].double()).reshape(16, 128)
        assert float((out[i, 0].double() - want).norm() / want.norm()) < 2.0 ** -8


# ------------------------------------------------------------------------------------------------------------ update
@pytest.mark.parametrize("shape,heads,kv,g,page", [("mla512", 16, 1, 64, 64), ("mla128", 4, 1, 16, 16), ("gqa128", 8, 2, 64, 16), ("gqa64", 6, 3, 32, 32),
                                                   ("mla512", 4, 1, 128, 32)])
def test_update_condenses_what_is_due(B, shape, heads, kv, g, page):
    variant, d_sem, d_pos = SHAPES[shape]
    w = 2 * g
    states = [(0, w + g), (2, 2 * g + w + g + 5), (1, g + w + g - 1), (0, 0), (3, 4 * g), (0, 3 * w)]
    pool, table = build(shape, kv, page, states, g, 5)
    table[5, 0] = -1                                                           # not wholly on pages: left alone
    p = B.make_params(variant, len(states), 1, heads, kv, d_sem, d_pos, g, w, 0.11)
    cache, _ = to_gpu(B, pool, table)
    r = torch.Generator().manual_seed(2)
    dk = d_pos + (d_sem if variant == "mla" else 0)
    n_rep, n_tok = i32([s[0] for s in states]), i32([s[1] for s in states])
    tails = [torch.randn((len(states), g, heads, d), generator=r).bfloat16() for d in (d_sem, d_pos)]
    qbar = torch.cat(tails, -1) if variant == "mla" else tails[1]
    qbar = qbar.double().view(len(states), g, kv, heads // kv, dk).mean((1, 3)).numpy()
    want = R.update(pool, table, [s[0] for s in states], [s[1] for s in states], qbar, g, w, 0.11)
    args = [(dict(qbar=torch.from_numpy(qbar).float().to(DEV)), (None, None)),
            (dict(), (tails[0].to(DEV) if variant == "mla" else None, tails[1].to(DEV)))]
    for kw, tail in args:
        new, sem, pos, anchor = B.decode_update_paged4(p, cache, *tail, n_rep, n_tok, **kw)
        assert new.cpu().tolist() == want[0].tolist() and anchor.cpu().tolist() == want[3].tolist()
        for b in range(len(states)):
            if b not in want[1]:
                assert torch.all(sem[b] == 0) and torch.all(pos[b] == 0)
                continue
            assert np.array_equal(pos[b].double().cpu().numpy(), want[2][b])
            # fp32 weights and sums of g terms: (g + 8) 2^-23 of sum |v|, which max |v| bounds; one bf16 rounding
            top = np.abs(R.gather(pool.sem(), table[b], list(range(states[b][0] * g, states[b][0] * g + g)), page)[0]).max()
            d = np.abs(sem[b].double().cpu().numpy() - want[1][b])
            assert np.all(d <= 2.0 ** -8 * np.abs(want[1][b]) + (g + 8) * 2.0 ** -23 * top)


# ------------------------------------------------------------------------------------------------- streams and graphs
@pytest.mark.parametrize("shape,heads,kv", [("mla512", 32, 1), ("gqa128", 8, 2)])
def test_calls_are_capturable_reproducible_and_independent_of_the_stream(B, shape, heads, kv):
    variant, d_sem, d_pos = SHAPES[shape]
    states = [(3, 3 * 64 + 200), (0, 700), (2, 2 * 64 + 90)]
    pool, table = build(shape, kv, 64, states, 64, 8)
    p = B.make_params(variant, 3, 1, heads, kv, d_sem, d_pos, 64, 0, 0.07)
    cache, t = to_gpu(B, pool, table)
    g = torch.Generator().manual_seed(1)
    q_pos = torch.randn((3, 1, heads, d_pos), generator=g).bfloat16().to(DEV)
    q_sem = torch.randn((3, 1, heads, d_sem), generator=g).bfloat16().to(DEV) if variant == "mla" else None
    rows = [torch.randn((3, kv, d), generator=g).bfloat16().to(DEV) for d in (d_sem, d_pos)]
    n_rep, n_tok = i32([s[0] for s in states]), i32([s[1] for s in states])
    slots = i32([int(table[b, (s[1] - 1) // 64]) * 64 + (s[1] - 1) % 64 for b, s in enumerate(states)])
    ws = B.workspace_paged4(p, cache, 1, DEV)

    def step(out, stream=None, ws=ws):
        B.paged4_write(p, cache, *rows, slots, stream=stream)
        B.decode_attention_paged4(p, cache, q_sem, q_pos, n_rep, n_tok, out=out, ws=ws, stream=stream)

    outs = [torch.zeros((3, 1, heads, d_sem), dtype=torch.bfloat16, device=DEV) for _ in range(4)]
    step(outs[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    step(outs[1], stream=side, ws=torch.empty_like(ws))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(outs[2])
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])
    rows[0].add_(0.5)                                                          # the graph reads what is there when it is replayed
    n_tok.copy_(i32([s[1] for s in states]) - 1)
    graph.replay()
    step(outs[3])
    torch.cuda.synchronize()
    assert torch.equal(outs[3], outs[2]) and not torch.equal(outs[3], outs[0])
