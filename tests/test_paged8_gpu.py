"""Paged 8-bit cache on the GPU against 64-bit statements of the same calls (tests/paged8_reference.py)."""
import math

import numpy as np
import pytest
import torch

from tests import paged8_reference as R

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
SHAPES = {"mla512": ("mla", 1, 512, 64), "mla128": ("mla", 1, 128, 64), "gqa128": ("gqa", 0, 128, 128), "gqa64": ("gqa", 0, 64, 64)}


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


# ------------------------------------------------------------------------------------------------------------- pages
class Tables:
    """The GPU state of a set of page tables beside the reference's."""

    def __init__(self, B, batch, width, n_pages, page, g, reps=True, seed=0):
        perm = np.random.RandomState(seed).permutation(n_pages)
        self.B, self.g, self.page, self.reps = B, g, page, reps
        self.p = B.make_params("mla", batch, 1, 16, 1, 512, 64, g, 0, 1.0)
        self.table = torch.full((batch, width), -1, dtype=torch.int32, device=DEV)
        self.cache = B.paged8_cache(None, None, None, None, self.table, page_size=page, n_pages=n_pages)
        self.free, self.n_free = i32(perm), i32([n_pages])
        self.held_rep = torch.zeros(batch, dtype=torch.int32, device=DEV) if reps else None
        self.held_tok = torch.zeros(batch, dtype=torch.int32, device=DEV)
        self.status = i32([-9])
        self.ref = R.Pages(self.table.cpu().numpy(), perm, n_pages, page, g, n_pages)

    def update(self, target, n_rows, per_seq=0, slots=True):
        Bn = len(target)
        n_rep = i32([t[0] for t in target]) if self.reps else None
        sm = torch.full((n_rows,), -7, dtype=torch.int32, device=DEV) if slots else None
        off = torch.full((Bn + 1,), -7, dtype=torch.int32, device=DEV)
        self.B.page_update(self.p, self.cache, n_rep, i32([t[1] for t in target]), self.held_rep, self.held_tok, self.free, self.n_free,
                           sm, off, self.status, rows_per_seq=per_seq)
        limit = None
        if slots:
            limit = (lambda rows: any(len(r) > per_seq for r in rows)) if per_seq else (lambda rows: sum(map(len, rows)) > n_rows)
        want, status = self.ref.update(target, limit)
        torch.cuda.synchronize()
        assert int(self.status) == status
        assert self.table.cpu().tolist() == self.ref.table
        assert int(self.n_free) == self.ref.top and self.free.cpu().tolist()[:self.ref.top] == self.ref.free[:self.ref.top]
        assert self.held_tok.cpu().tolist() == [h[1] for h in self.ref.held]
        if self.reps:
            assert self.held_rep.cpu().tolist() == [h[0] for h in self.ref.held]
        assert off.cpu().tolist() == np.concatenate([[0], np.cumsum([len(w) for w in want])]).astype(int).tolist()
        if slots:
            if per_seq:
                flat = [s for w in want for s in w + [-1] * (per_seq - len(w))]
            else:
                flat = [s for w in want for s in w]
                flat += [-1] * (n_rows - len(flat))
            assert sm.cpu().tolist() == flat
        return status


@pytest.mark.parametrize("batch,page,g", [(1, 16, 16), (5, 16, 64), (3, 64, 64), (7, 32, 64), (2, 128, 128), (600, 16, 16)])
def test_page_update_through_the_life_of_requests(B, batch, page, g):
    rng = np.random.RandomState(batch + page)
    w = 2 * g
    width = -(-40 * g // page)
    T = Tables(B, batch, width, batch * width, page, g, seed=batch)
    toks = rng.randint(0, 4 * g, batch)
    toks[0] = 0
    reps = np.maximum(0, (toks - w) // g)
    assert T.update(list(zip(reps.tolist(), toks.tolist())), int(batch * 6 * g)) == 0          # prompts, some of them empty
    for step in range(6):
        toks = np.minimum(toks + rng.randint(0, 3, batch) * (1 + step * g // 2), 39 * g)
        n = 40 * g
        reps = np.maximum(reps, np.maximum(0, (toks - w) // g) if step % 2 else reps)           # condensation lags
        assert T.update(list(zip(reps.tolist(), toks.tolist())), batch * n) == 0
        back = np.maximum(toks - rng.randint(0, g, batch), reps * g)                           # rejected tokens
        T.update(list(zip(reps.tolist(), back.tolist())), 0, slots=False)
        toks = back
        done = rng.rand(batch) < 0.2
        toks, reps = np.where(done, 0, toks), np.where(done, 0, reps)
        T.update(list(zip(reps.tolist(), toks.tolist())), 0, slots=False)
    T.update([(0, 0)] * batch, 8)
    assert int(T.n_free) == T.free.numel()                                                     # every page came back


def test_page_update_padded_slots_and_uncondensed_tables(B):
    T = Tables(B, 4, 8, 20, 32, 64, reps=False)
    assert T.update([(0, 5), (0, 0), (0, 33), (0, 64)], 4 * 64, per_seq=64) == 0
    assert T.update([(0, 6), (0, 1), (0, 33), (0, 65)], 4, per_seq=1) == 0
    assert T.update([(0, 6), (0, 1), (0, 33), (0, 65)], 4, per_seq=1) == 0                     # nothing new
    assert T.update([(0, 8), (0, 1), (0, 33), (0, 65)], 4, per_seq=1) == -2                    # two rows, one place
    U = Tables(B, 2, 40, 64, 16, 16)
    assert U.update([(0, 100), (0, 48)], 2 * 100, per_seq=100) == 0
    assert U.update([(2, 101), (1, 48)], 2 * 3, per_seq=3) == 0                                # representatives first, then the token


def test_page_update_refuses_as_a_whole(B):
    T = Tables(B, 3, 4, 5, 16, 16)
    assert T.update([(0, 40), (0, 3), (0, 0)], 64) == 0                                        # 3 + 1 pages of 5
    assert T.update([(0, 40), (0, 17), (0, 20)], 64) == 2                                      # 1 + 2 more: two are missing
    assert T.update([(0, 40), (0, 3), (0, 65)], 64) == -1                                      # behind the table
    assert T.update([(3, 40), (0, 3), (0, 1)], 64) == -1                                       # more condensed than there is
    assert T.update([(-1, 40), (0, 3), (0, 1)], 64) == -1
    assert T.update([(0, -5), (0, 3), (0, 1)], 64) == -1
    assert T.update([(0, 40), (0, 3), (0, 16)], 3) == -2                                       # 16 rows, 3 places
    assert T.update([(0, 40), (0, 3), (0, 16)], 0) == -2                                       # an empty slot map is one
    assert T.update([(0, 40), (0, 3), (0, 0)], 0) == 0                                         # ... and enough where there is nothing new
    assert T.update([(2, 40), (0, 3), (0, 16)], 64) == 0                                       # two pages come back, two are taken
    assert T.update([(1, 40), (0, 3), (0, 16)], 64) == -1                                      # a condensation is not undone
    T.held_tok[1] = 1 << 20                                                                    # a broken held state is refused too
    T.B.page_update(T.p, T.cache, i32([2, 0, 0]), i32([40, 3, 16]), T.held_rep, T.held_tok, T.free, T.n_free, None, None, T.status)
    assert int(T.status) == -1


# ------------------------------------------------------------------------------------------------------------- write
def pool(shape, n_pages, page, seed, kv):
    """Random codes (no NaN) and power-of-two scales as numpy arrays."""
    variant, _, d_sem, d_pos = SHAPES[shape]
    r = np.random.RandomState(seed)
    code = lambda d: R.encode(np.clip(r.randn(n_pages, kv, page, d) * 60, -448, 448))  # noqa: E731
    scale = lambda: (2.0 ** r.randint(-8, -4, (n_pages, kv))).astype(np.float32)       # noqa: E731
    return code(d_sem), code(d_pos), scale(), scale() if variant == "gqa" else None


def to_gpu(B, pool_, table=None):
    t = [None if x is None else torch.from_numpy(np.ascontiguousarray(x)).to(DEV) for x in pool_]
    return B.paged8_cache(*t, table), t


def check_write(B, shape, kv, page, slots, rows_sem, rows_pos, pool_, n_pages):
    variant, _, d_sem, d_pos = SHAPES[shape]
    p = B.make_params(variant, 1, 1, kv, kv, d_sem, d_pos, 64, 0, 1.0)
    cache, t = to_gpu(B, pool_)
    B.paged8_write(p, cache, rows_sem.to(DEV), rows_pos.to(DEV), i32(slots))
    torch.cuda.synchronize()
    want = R.write(*pool_, rows_sem.double().numpy(), rows_pos.double().numpy(), slots, page)
    for name, got, w in zip(("sem", "pos", "scale_sem", "scale_pos"), t, want):
        if w is not None:
            g = got.cpu().numpy()
            if w.dtype == np.uint8:                       # both zeros are the same value
                g, w = np.where(g == 128, 0, g), np.where(w == 128, 0, w)
            assert np.array_equal(g, w), (name, int((g != w).sum()), np.argwhere(g != w)[:3])


@pytest.mark.parametrize("shape,kv", [("mla512", 1), ("mla128", 1), ("gqa128", 3), ("gqa64", 2)])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_write_whole_pages_odd_runs_and_single_rows(B, shape, kv, page):
    variant, _, d_sem, d_pos = SHAPES[shape]
    r = np.random.RandomState(page + kv)
    n_pages = 9
    order = r.permutation(n_pages)
    slots = []
    for i, n in enumerate([page, 1, page - 1, 5, page]):                       # runs from place 0
        slots += [int(order[i]) * page + k for k in range(n)]
    slots += [-1, -1, n_pages * page, 2 ** 31 - 1]                             # padding, and slots behind the pool
    slots += [int(order[5]) * page + k for k in range(3, 9)]                   # a run that starts inside a page
    slots += [int(order[6]) * page + page - 1, int(order[7]) * page + 1]       # single rows
    T = len(slots)
    gain = np.exp(2.5 * r.randn(T, 1, 1))                                      # scales grow and do not
    sem, pos = (torch.from_numpy(r.randn(T, kv, d) * gain).bfloat16() for d in (d_sem, d_pos))
    check_write(B, shape, kv, page, slots, sem, pos, pool(shape, n_pages, page, 3, kv), n_pages)


@pytest.mark.parametrize("shape,kv", [("mla512", 1), ("gqa128", 2)])
def test_write_extreme_values(B, shape, kv):
    variant, _, d_sem, d_pos = SHAPES[shape]
    page, n_pages = 16, 12
    r = np.random.RandomState(5)
    slots = [p * page + k for p in range(n_pages) for k in (range(2) if p < 9 else range(3, 5))]
    T = len(slots)
    sem, pos = (torch.from_numpy(r.randn(T, kv, d)).float() for d in (d_sem, d_pos))
    for t, (a, b) in enumerate([(0.0, 0.0), (1e-38, 1e-38), (1e-40, 0.0), (3.3e38, 1.0), (448.0, 448.0), (449.0, 1.0), (2 ** -95, 2 ** -99)]):
        sem[2 * t:2 * t + 2] *= a
        pos[2 * t:2 * t + 2] *= b
    sem[8, :, 0] = 448.0; sem[8, :, 1:] = 0.25                                 # the maximum is exactly 448
    sem[14, :, 3], sem[14, :, 5], sem[15, :, 7] = float("inf"), float("-inf"), float("nan")
    pos[16, :, 3] = float("nan"); pos[16, :, 2] = float("inf")
    sem[17] = float("inf"); pos[17] = float("nan")
    check_write(B, shape, kv, page, slots, sem.bfloat16(), pos.bfloat16(), pool(shape, n_pages, page, 4, kv), n_pages)


def test_write_long_prompt_and_appended_rows_equal_one_write(B):
    # appending row by row gives the codes of one write wherever no code falls below the normal range
    shape, kv, page, n = "mla512", 1, 64, 64 * 7 + 13
    p = B.make_params("mla", 1, 1, 1, 1, 512, 64, 64, 0, 1.0)
    r = np.random.RandomState(1)
    sign = torch.from_numpy(r.choice([-1.0, 1.0], (n, 1, 576)))
    rows = sign * torch.from_numpy(r.uniform(1.0, 8.0, (n, 1, 576)))
    sem, pos = rows[..., :512].bfloat16().to(DEV), rows[..., 512:].bfloat16().to(DEV)
    slots = i32([(7 - i // page) * page + i % page for i in range(n)])
    got = []
    for step in (n, 1):
        cache, t = to_gpu(B, pool(shape, 8, page, 6, kv))
        for i in range(0, n, step):
            B.paged8_write(p, cache, sem[i:i + step], pos[i:i + step], slots[i:i + step])
        got.append(t)
    used = slots.cpu().long()
    one, many = (x[0].view(8 * page, 512)[used] for x in got), None
    a, b = (x[0].transpose(1, 2).reshape(8 * page, 512)[used].cpu() for x in got)
    sa, sb = (x[2][used.to(DEV) // page].cpu() for x in got)
    assert torch.equal(sa, sb) and torch.equal(a, b)


# ------------------------------------------------------------------------------------------------------------ attend
def build(B, shape, kv, page, states, g, seed, reps=True, hole_nan=True, spare=3):
    """Cache of sequences in the given states [(n_rep, n_tok)]; every byte that no present row holds is NaN."""
    variant, _, d_sem, d_pos = SHAPES[shape]
    r = np.random.RandomState(seed)
    width = max(1, -(-max(t for _, t in states) // page))
    need = [(b, e) for b, (n, t) in enumerate(states) for e in range(width)
            if any(R.present(n, t, g, x) for x in range(e * page, (e + 1) * page))]
    n_pages = len(need) + spare
    ids = r.permutation(n_pages)[:len(need)]
    table = np.full((len(states), width), -1, dtype=np.int32)
    for (b, e), i in zip(need, ids):
        table[b, e] = i
    cs, cp, ss, sp = pool(shape, n_pages, page, seed + 1, kv)
    if hole_nan:
        keep = np.zeros((n_pages, page), dtype=bool)
        for (b, e), i in zip(need, ids):
            keep[i] = [R.present(*states[b], g, x) for x in range(e * page, (e + 1) * page)]
        cs[~keep[:, None].repeat(kv, 1)] = 0x7f
        cp[~keep[:, None].repeat(kv, 1)] = 0xff
        unused = np.setdiff1d(np.arange(n_pages), ids)
        ss[unused] = np.nan
    return (cs, cp, ss, sp), table


def check_attend(B, shape, heads, kv, page, states, g, q_len, seed=0, bias=0.0, reps=True, impl=0, table_edit=None, q_gain=1.0, pool_edit=None,
                 softmax_scale=None):
    variant, _, d_sem, d_pos = SHAPES[shape]
    pool_, table = build(B, shape, kv, page, states, g, seed)
    if pool_edit:
        pool_edit(pool_, table)
    if table_edit:
        table_edit(table)
    r = torch.Generator().manual_seed(seed)
    nb = len(states)
    scale = softmax_scale or 1.0 / math.sqrt(192.0 if variant == "mla" else d_pos)
    q_pos = (torch.randn((nb, q_len, heads, d_pos), generator=r) * q_gain).bfloat16()
    q_sem = (torch.randn((nb, q_len, heads, d_sem), generator=r) * q_gain).bfloat16() if variant == "mla" else None
    p = B.make_params(variant, nb, 1, heads, kv, d_sem, d_pos, g, 0, scale, rep_logit_bias=bias)
    cache, keep = to_gpu(B, pool_, torch.from_numpy(table).to(DEV))
    n_rep = i32([s[0] for s in states]) if reps else None
    old = B.lca_set_attention_impl(impl)
    try:
        out, lse = B.decode_attention_paged8(p, cache, None if q_sem is None else q_sem.to(DEV), q_pos.to(DEV), n_rep, i32([s[1] for s in states]),
                                             want_lse=True)
        torch.cuda.synchronize()
    finally:
        B.lca_set_attention_impl(old)
    want, want_lse, absv, big = R.attend(None if q_sem is None else q_sem.double().numpy(), q_pos.double().numpy(), *pool_, table,
                                         [s[0] for s in states] if reps else [0] * nb, [s[1] for s in states], g, page, scale, bias)
    compare(out, lse, want, want_lse, absv, big, n=max(t for _, t in states), top=np.nanmax(np.abs(want)) if want.size else 0.0)
    return out, lse


def compare(out, lse, want, want_lse, absv, big, n, top):
    """Logit error e: a query element is off by 2^-17 of its row's largest, so the product sum by 2^-17 max|q| sum|k| (`big`, with
    the softmax scale); fp32 sums of up to 2 * 576 products (2^-24 each, worst order) add 2^-13 of the same; exp2 / log2 and
    the scale products 2^-21 of the logits, which `big` bounds as well.  A weight is then off by the factor 2 e, its two terms
    by 2^-8, the result by the same of sum p|v| (numerator) and of |out| (row sum, logit part only); the floor of a weight, 2^-10
    where the largest is at least 2^5, i.e. 2^-15 of it, is dithered: 1/64 of it for every key in one direction, and what the
    offsets do not cancel within one round of 32 keys, 32 times it at most per round of different weights, i.e. the mean error
    of independent roundings; bf16 rounds by 2^-8 |out| at most."""
    got, gl = out.double().cpu().numpy(), lse.double().cpu().numpy()
    e = big * (2.0 ** -17 + 2.0 ** -13 + 2.0 ** -20)
    empty = ~np.isfinite(want_lse)
    assert np.array_equal(np.isneginf(gl), empty) and np.all(got[empty] == 0)
    dl = np.abs(gl[~empty] - want_lse[~empty])
    assert np.all(dl <= e[~empty] + 1e-6 * np.abs(want_lse[~empty]) + 1e-6), dl.max()
    tol = absv * (2.0 ** -8 + 4 * e[..., None]) + 2.0 ** -8 * np.abs(want) + 2.0 ** -15 * (1 + n / 64) * absv.max(initial=0) + 1e-30
    bad = np.abs(got - want) > tol
    assert not bad.any(), (int(bad.sum()), float(np.abs(got - want).max()), np.argwhere(bad)[:4])
    if (~empty).any():
        print("lse err %.2e  out rel %.2e" % (dl.max(), np.linalg.norm(got - want) / max(np.linalg.norm(want), 1e-300)))


STATES = [(0, 1), (0, 130), (3, 3 * 64 + 70), (0, 0), (5, 5 * 64 + 1), (17, 17 * 64 + 333)]


@pytest.mark.parametrize("impl", [1, 0])
@pytest.mark.parametrize("shape,heads,kv", [("mla512", 16, 1), ("mla512", 3, 1), ("mla512", 20, 1), ("mla512", 128, 1), ("mla512", 40, 1), ("mla128", 8, 1),
                                            ("mla128", 32, 1), ("mla128", 64, 1), ("gqa128", 8, 2), ("gqa128", 2, 2), ("gqa128", 32, 1), ("gqa128", 70, 1),
                                            ("gqa64", 8, 4), ("gqa64", 24, 1), ("gqa64", 64, 1)])
def test_attend_head_layouts(B, impl, shape, heads, kv):
    check_attend(B, shape, heads, kv, 64, STATES, 64, 1, seed=heads, bias=0.7, impl=impl)


@pytest.mark.parametrize("shape,heads,kv,q_len", [("mla512", 16, 1, 2), ("mla512", 24, 1, 5), ("gqa128", 8, 2, 4), ("gqa128", 6, 2, 7), ("gqa64", 4, 2, 33),
                                                  ("mla128", 2, 1, 16), ("mla512", 128, 1, 3), ("mla512", 80, 1, 1), ("mla512", 48, 1, 2)])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_attend_several_queries_and_page_sizes(B, shape, heads, kv, q_len, page):
    # short sequences leave the first queries without a row
    states = [(0, 1), (0, 3), (2, 2 * 128 + 140), (1, 128 + q_len), (0, 257), (0, 0), (3, 3 * 128)]
    check_attend(B, shape, heads, kv, page, states, 128, q_len, seed=page + q_len, bias=-0.4)


@pytest.mark.parametrize("shape,heads,kv,rows,batch", [("mla512", 16, 1, 9000, 1), ("mla512", 33, 1, 21000, 1), ("mla512", 128, 1, 3000, 5), ("gqa128", 8, 2, 5003, 3), ("mla512", 64, 1, 2600, 2), ("gqa64", 3, 1, 40001, 1)])
def test_attend_long_sequences_are_cut_and_merged(B, shape, heads, kv, rows, batch):
    check_attend(B, shape, heads, kv, 64, [(0, rows - 700 * i) for i in range(batch)], 64, 1, seed=rows, reps=False)


def test_attend_many_units_on_few_ctas(B):
    # more (sequence, KV head) units than CTAs, lengths from nothing to several tiles
    rng = np.random.RandomState(0)
    states = [(0, int(n)) for n in rng.randint(0, 400, 90)]
    check_attend(B, "gqa128", 16, 8, 16, states, 64, 1, seed=2)


def test_attend_growing_maximum(B):
    # logits of tens, rising along the sequence: the running maximum is raised again and again, O rescaled
    def rise(pool_, table):
        cs, cp, ss, sp = pool_
        for e in range(table.shape[1]):
            sp[table[0, e]] = 2.0 ** (-8 + e / 3.0)
            ss[table[0, e]] = 2.0 ** (-4 - e / 4.0) * 1.3                     # scales need not be powers of two
    check_attend(B, "gqa128", 8, 1, 64, [(0, 64 * 30)], 64, 1, seed=9, pool_edit=rise, q_gain=0.05)
    check_attend(B, "gqa128", 8, 1, 64, [(0, 64 * 30)], 64, 1, seed=9, q_gain=4.0)
    check_attend(B, "mla512", 64, 1, 64, [(0, 64 * 20 + 5)], 64, 1, seed=10, q_gain=3.0)

    def rise_mla(pool_, table):
        for e in range(table.shape[1]):
            pool_[2][table[0, e]] = 2.0 ** (-9 + e / 3.0)                     # keys and values grow together
    for heads in (16, 20, 72):
        check_attend(B, "mla512", heads, 1, 64, [(0, 64 * 30)], 64, 1, seed=12, pool_edit=rise_mla, q_gain=0.05)


def test_attend_scales_of_every_size(B):
    def edit(pool_, table):
        for e in range(table.shape[1]):
            pool_[2][table[0, e]] = [2.0 ** -100, 2.0 ** 40, 1.0, 2.0 ** -60][e % 4]
    check_attend(B, "gqa128", 8, 2, 16, [(0, 16 * 23 + 3)], 64, 1, seed=11, pool_edit=edit)

    def small(pool_, table):                                                   # MLA: key and value share the scale
        for e in range(table.shape[1]):
            pool_[2][table[0, e]] = [2.0 ** -100, 2.0 ** -7, 2.0 ** -60][e % 3]
    for heads in (16, 70):
        check_attend(B, "mla512", heads, 1, 16, [(0, 16 * 23 + 3)], 64, 1, seed=11, pool_edit=small)


def test_attend_flat_tail_behind_one_large_logit(B):
    # one key far above 120000 equal ones (all codes zero): the tail's share comes from weights below the floor of a single
    # one, which must not all round the same way.  The reference is the closed form; values of the tail are 1, of the peak 0.
    page, n = 128, 120000
    p = B.make_params("gqa", 1, 1, 4, 1, 64, 64, 64, 0, 1.0)
    n_pages = -(-n // page)
    cache = B.new_paged8_cache(p, n_pages, page, n_pages, DEV)
    sem, pos, ss, sp, table = cache.tensors
    table.copy_(torch.arange(n_pages, dtype=torch.int32, device=DEV)[None])
    sem.fill_(0x38)                                                            # 1.0
    sem[0, 0, 5] = 0
    pos[0, 0, 5] = 0x38                                                        # key (1, ..., 1)
    q = torch.zeros((1, 1, 4, 64), dtype=torch.bfloat16, device=DEV)
    tops = [4.0, 9.0, 12.0, 13.5]
    for h, top in enumerate(tops):
        q[0, 0, h] = top / 64
    out, lse = B.decode_attention_paged8(p, cache, None, q, None, i32([n]), want_lse=True)
    for h in range(4):
        t = float(q[0, 0, h].double().sum())
        l = math.exp(t) + n - 1
        share = (n - 1) / l
        # floor 2^-15 of the largest weight, exp(t): the 938 tiles are cut into at least 148 ranges with a maximum of their own, so
        # that at most 8 tiles share the peak's, and there the 32 offsets leave at most 1/64 of it for each of 1024 equal keys;
        # elsewhere every weight is the largest (2^-9), and bf16 rounds by 2^-8
        assert abs(float(out[0, 0, h, 0]) - share) <= 2.0 ** -7 * share + 1024 * 2.0 ** -21 * math.exp(t) / l
        assert abs(float(lse[0, 0, h]) - math.log(l)) < 1e-4


def test_attend_entries_that_are_no_pages(B):
    def edit(table):
        table[0, 1], table[0, 3], table[1, 0], table[1, 2] = -1, 1 << 30, 2 ** 31 - 1, -(2 ** 31)
    for impl in (0, 1):
        check_attend(B, "gqa128", 8, 2, 32, [(0, 200), (0, 81), (0, 32)], 64, 2, seed=4, table_edit=edit, impl=impl)
    def none(table):
        table[:] = -5
    check_attend(B, "mla512", 16, 1, 32, [(0, 200), (0, 81)], 64, 1, seed=4, table_edit=none)


def test_attend_nan_and_infinity_stay_where_they_belong(B):
    def edit(pool_, table):
        pool_[0][table[1, 0], 1, 3, 7] = 0x7f                                  # V of sequence 1, head 1
        pool_[1][table[2, 1], 0, 2, 9] = 0xff                                  # K of sequence 2, head 0
    shape, kv, page, states, g = "gqa128", 2, 16, [(0, 50), (0, 60), (0, 30), (0, 40)], 64
    pool_, table = build(B, shape, kv, page, states, g, 3)
    edit(pool_, table)
    q = torch.randn((4, 1, 8, 128), generator=torch.Generator().manual_seed(1)).bfloat16()
    q[3, 0, 5, 11], q[3, 0, 1, 0] = float("inf"), float("nan")
    p = B.make_params("gqa", 4, 1, 8, kv, 128, 128, g, 0, 0.1)
    cache, _ = to_gpu(B, pool_, torch.from_numpy(table).to(DEV))
    out, lse = B.decode_attention_paged8(p, cache, None, q.to(DEV), None, i32([s[1] for s in states]), want_lse=True)
    bad = torch.isnan(out[:, 0]).cpu()
    want = torch.zeros((4, 8, 128), dtype=torch.bool)
    want[1, 4:, 7] = True                                                      # one column of the values
    want[2, :4] = True
    want[3, 5], want[3, 1] = True, True
    assert torch.equal(bad, want)
    assert torch.equal(torch.isnan(lse[:, 0]).cpu(), want.all(-1))


@pytest.mark.parametrize("heads", [16, 96])
def test_attend_nan_and_infinity_in_latents_and_queries(B, heads):
    states = [(0, 50), (0, 260), (0, 140), (0, 40)]
    pool_, table = build(B, "mla512", 1, 64, states, 64, 3)
    pool_[0][table[1, 2], 0, 3, 7] = 0x7f                                      # one latent element: key and value
    q = [torch.randn((4, 1, heads, d), generator=torch.Generator().manual_seed(1)).bfloat16() for d in (512, 64)]
    q[0][3, 0, 5, 11], q[1][3, 0, heads - 1, 0] = float("inf"), float("nan")
    p = B.make_params("mla", 4, 1, heads, 1, 512, 64, 64, 0, 0.07)
    cache, _ = to_gpu(B, pool_, torch.from_numpy(table).to(DEV))
    out, lse = B.decode_attention_paged8(p, cache, q[0].to(DEV), q[1].to(DEV), None, i32([s[1] for s in states]), want_lse=True)
    want = torch.zeros((4, heads), dtype=torch.bool)
    want[1] = True
    want[3, 5], want[3, heads - 1] = True, True
    assert torch.equal(torch.isnan(out[:, 0]).all(-1).cpu(), want) and torch.equal(torch.isnan(out[:, 0]).any(-1).cpu(), want)
    assert torch.equal(torch.isnan(lse[:, 0]).cpu(), want)


def test_attend_counters_beyond_the_table_are_clamped(B):
    pool_, table = build(B, "mla128", 1, 16, [(0, 64), (4, 64)], 16, 3)
    p = B.make_params("mla", 2, 1, 8, 1, 128, 64, 16, 0, 0.1)
    cache, _ = to_gpu(B, pool_, torch.from_numpy(table).to(DEV))
    g = torch.Generator().manual_seed(1)
    q = [torch.randn((2, 1, 8, d), generator=g).bfloat16().to(DEV) for d in (128, 64)]
    a, _ = B.decode_attention_paged8(p, cache, *q, i32([0, 4]), i32([64, 64]))
    b, _ = B.decode_attention_paged8(p, cache, *q, i32([-3, 4]), i32([2 ** 31 - 1, 70]))
    assert torch.equal(a, b)
    c, l = B.decode_attention_paged8(p, cache, *q, i32([2 ** 31 - 1, 5]), i32([-7, -2 ** 31]), want_lse=True)
    assert torch.all(c == 0) and torch.all(torch.isneginf(l))


def test_attend_rows_behind_the_batch_stay_as_they_are(B):
    pool_, table = build(B, "gqa128", 2, 16, [(0, 50), (0, 0), (0, 333)], 64, 3)
    p = B.make_params("gqa", 3, 1, 6, 2, 128, 128, 64, 0, 0.1)
    cache, _ = to_gpu(B, pool_, torch.from_numpy(table).to(DEV))
    q = torch.randn((3, 2, 6, 128), device=DEV).bfloat16()
    out = torch.full((5, 2, 6, 128), 7.0, dtype=torch.bfloat16, device=DEV)
    lse = torch.full((5, 2, 6), 7.0, device=DEV)
    ws = torch.full((B.lca_paged8_workspace_bytes(p, cache, 2) + 64,), 0xff, dtype=torch.uint8, device=DEV)      # NaN everywhere
    n = ws.numel() - 64
    assert B.lca_decode_attention_paged8(p, cache, None, q, 2, None, i32([50, 0, 333]), out, lse, ws, n) == 0
    torch.cuda.synchronize()
    assert torch.all(out[3:] == 7) and torch.all(lse[3:] == 7) and torch.all(ws[n:] == 0xff)
    assert torch.isfinite(out).all()


@pytest.mark.parametrize("heads", [32, 128])
def test_calls_are_capturable_reproducible_and_independent_of_the_stream(B, heads):
    states = [(3, 3 * 64 + 200), (0, 700), (2, 2 * 64 + 90)]
    pool_, table = build(B, "mla512", 1, 64, states, 64, 8, hole_nan=False)
    p = B.make_params("mla", 3, 1, heads, 1, 512, 64, 64, 0, 0.07)
    cache, t = to_gpu(B, pool_, torch.from_numpy(table).to(DEV))
    g = torch.Generator().manual_seed(1)
    q_sem, q_pos = (torch.randn((3, 1, heads, d), generator=g).bfloat16().to(DEV) for d in (512, 64))
    rows = [torch.randn((3, 1, d), generator=g).bfloat16().to(DEV) for d in (512, 64)]
    n_rep, n_tok = i32([s[0] for s in states]), i32([s[1] for s in states])
    slots = i32([int(table[b, (s[1] - 1) // 64]) * 64 + (s[1] - 1) % 64 for b, s in enumerate(states)])
    ws = B.workspace_paged8(p, cache, 1, DEV)

    def step(out, stream=None):
        B.paged8_write(p, cache, *rows, slots, stream=stream)
        B.decode_attention_paged8(p, cache, q_sem, q_pos, n_rep, n_tok, out=out, ws=ws, stream=stream)

    outs = [torch.zeros((3, 1, heads, 512), dtype=torch.bfloat16, device=DEV) for _ in range(4)]
    step(outs[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    step(outs[1], stream=side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(outs[2])
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])
    # the captured calls read their inputs at replay: other queries, another row, one token more in one sequence
    q_sem.mul_(0.5); rows[0].add_(1.0)
    n_tok.add_(i32([0, -1, 0]))
    graph.replay()
    step(outs[3])
    torch.cuda.synchronize()
    assert torch.equal(outs[2], outs[3]) and not torch.equal(outs[0], outs[3])


# ------------------------------------------------------------------------------------------------------------ update
@pytest.mark.parametrize("shape,heads,kv,g,page,w", [("mla512", 16, 1, 64, 64, 64), ("mla512", 16, 1, 16, 16, 0), ("gqa128", 8, 2, 32, 16, 40),
                                                     ("mla128", 4, 1, 128, 32, 7), ("gqa64", 4, 4, 64, 64, 64),
                                                     ("mla512", 16, 1, 208, 16, 3), ("gqa128", 9, 3, 80, 16, 0), ("gqa64", 4, 2, 48, 16, 5)])
def test_update_against_the_definition(B, shape, heads, kv, g, page, w):
    variant, _, d_sem, d_pos = SHAPES[shape]
    states = [(0, w + g), (0, w + g - 1), (3, 3 * g + w + g), (2, 2 * g + w + g + 5), (0, 0), (1, g), (1, g + w + g)]
    pool_, table = build(B, shape, kv, page, states, g, 5)
    table[6, (2 * g - 1) // page] = -1                                         # a group that is not wholly on pages
    p = B.make_params(variant, len(states), 1, heads, kv, d_sem, d_pos, g, w, 0.08)
    cache, _ = to_gpu(B, pool_, torch.from_numpy(table).to(DEV))
    dk = d_pos + (d_sem if variant == "mla" else 0)
    gen = torch.Generator().manual_seed(2)
    qbar = torch.randn((len(states), kv, dk), generator=gen)
    qbar[2] = 0.0                                                              # all scores equal: the lowest index
    n_rep, n_tok = i32([s[0] for s in states]), i32([s[1] for s in states])
    sem = torch.full((len(states), kv, d_sem), 7.0, dtype=torch.bfloat16, device=DEV)
    pos = torch.full((len(states), kv, d_pos), 7.0, dtype=torch.bfloat16, device=DEV)
    new, sem, pos, anchor = B.decode_update_paged8(p, cache, None, None, n_rep, n_tok, rep_sem=sem, rep_pos=pos, qbar=qbar.to(DEV))
    torch.cuda.synchronize()
    want_new, want_sem, want_pos, want_anchor = R.update(*pool_, table, [s[0] for s in states], [s[1] for s in states], qbar.numpy(), g, w, page, 0.08)
    assert new.cpu().tolist() == want_new.tolist() and anchor.cpu().tolist() == want_anchor.tolist()
    assert n_rep.cpu().tolist() == [s[0] for s in states]
    for b in range(len(states)):
        for h in range(kv):
            if (b, h) not in want_sem:
                assert torch.all(sem[b, h] == 7) and torch.all(pos[b, h] == 7)
                continue
            # fp32 weights and sums: (g + 8) roundings of 2^-24 relative to the largest value; one rounding to bf16 (2^-8)
            ref = want_sem[b, h]
            err = np.abs(sem[b, h].double().cpu().numpy() - ref)
            vmax = np.nanmax(np.abs(R.decode(torch.from_numpy(pool_[0])))) * np.nanmax(pool_[2])
            assert np.all(err <= 2.0 ** -8 * np.abs(ref) + (g + 8) * 2.0 ** -23 * vmax)
            assert np.array_equal(pos[b, h].double().cpu().numpy(), want_pos[b, h])      # code * 2^e: exact in bf16


def test_update_with_a_query_tail_equals_the_ready_query(B):
    states = [(0, 128), (1, 64 + 128), (0, 60)]
    pool_, table = build(B, "gqa128", 2, 16, states, 64, 5)
    p = B.make_params("gqa", 3, 1, 8, 2, 128, 128, 64, 64, 0.08, n_summary_q=10)
    cache, _ = to_gpu(B, pool_, torch.from_numpy(table).to(DEV))
    tail = torch.randn((3, 10, 8, 128), generator=torch.Generator().manual_seed(3)).bfloat16()
    qbar = tail.double().view(3, 10, 2, 4, 128).mean((1, 3)).float()
    n_rep, n_tok = i32([s[0] for s in states]), i32([s[1] for s in states])
    a = B.decode_update_paged8(p, cache, None, tail.to(DEV), n_rep, n_tok)
    b = B.decode_update_paged8(p, cache, None, None, n_rep, n_tok, qbar=qbar.to(DEV))
    assert torch.equal(a[0], b[0]) and torch.equal(a[3], b[3]) and torch.equal(a[2], b[2])
    # the fp32 summary query differs from the fp64 one by 2^-24: the weights by 2^-24 sum|q k| < 2^-17, the result by one bf16 step
    assert torch.all((a[1].float() - b[1].float()).abs() <= 2.0 ** -7 * b[1].float().abs() + 2.0 ** -15 * 30)


# -------------------------------------------------------------------------------------------------------- large pools
@pytest.mark.parametrize("shape,heads,kv,n_pages", [("mla512", 16, 1, 140000), ("mla512", 128, 1, 140000), ("gqa128", 16, 8, 70000)])
def test_pages_behind_four_gigabytes(B, shape, heads, kv, n_pages):
    """The last pages of a pool of 4.6 GB give what the same pages of a small pool give, bit for bit."""
    variant, _, d_sem, d_pos = SHAPES[shape]
    states = [(1, 64 + 200), (0, 130)]
    pool_, table = build(B, shape, kv, 64, states, 64, 9, hole_nan=False)
    small, t = to_gpu(B, pool_, torch.from_numpy(table).to(DEV))
    first = n_pages - t[0].shape[0]
    large = [None if x is None else torch.empty((n_pages,) + x.shape[1:], dtype=x.dtype, device=DEV) for x in t]
    for x, y in zip(t, large):
        if x is not None:
            y[first:] = x
    big = B.paged8_cache(*large, torch.from_numpy(np.where(table < 0, table, table + first).astype(np.int32)).to(DEV))
    p = B.make_params(variant, 2, 1, heads, kv, d_sem, d_pos, 64, 64, 0.07)
    g = torch.Generator().manual_seed(2)
    q_sem = torch.randn((2, 1, heads, d_sem), generator=g).bfloat16().to(DEV) if variant == "mla" else None
    q_pos = torch.randn((2, 1, heads, d_pos), generator=g).bfloat16().to(DEV)
    qbar = torch.randn((2, kv, d_pos + (d_sem if variant == "mla" else 0)), generator=g).to(DEV)
    rows = [torch.randn((70, kv, d), generator=g).bfloat16().to(DEV) for d in (d_sem, d_pos)]
    n_rep, n_tok = i32([s[0] for s in states]), i32([s[1] for s in states])
    slots = torch.cat([torch.arange(64, 128), torch.arange(10, 16)]).int().to(DEV)
    got = []
    for cache, at in ((small, 0), (big, first)):
        out, lse = B.decode_attention_paged8(p, cache, q_sem, q_pos, n_rep, n_tok, want_lse=True)
        up = B.decode_update_paged8(p, cache, None, None, n_rep, n_tok, qbar=qbar)
        B.paged8_write(p, cache, *rows, slots + 64 * at)
        got.append([out, lse, *up])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(*got))
    assert all(x is None or torch.equal(x, y[first:]) for x, y in zip(t, large))


# ------------------------------------------------------------------------------------------- streams, graphs, refusals
def decode_case(B, heads, seed, variant="mla512", kv=1):
    states = [(3, 3 * 64 + 200), (0, 700), (2, 2 * 64 + 90)]
    pool_, table = build(B, variant, kv, 64, states, 64, seed, hole_nan=False)
    _, _, d_sem, d_pos = SHAPES[variant]
    p = B.make_params(SHAPES[variant][0], 3, 1, heads, kv, d_sem, d_pos, 64, 64, 0.07)
    cache, _ = to_gpu(B, pool_, torch.from_numpy(table).to(DEV))
    g = torch.Generator().manual_seed(seed)
    q_sem = torch.randn((3, 1, heads, d_sem), generator=g).bfloat16().to(DEV) if variant[:3] == "mla" else None
    q_pos = torch.randn((3, 1, heads, d_pos), generator=g).bfloat16().to(DEV)
    qbar = torch.randn((3, kv, d_pos + (d_sem if q_sem is not None else 0)), generator=g).to(DEV)
    return p, cache, q_sem, q_pos, i32([s[0] for s in states]), i32([s[1] for s in states]), qbar


def test_results_made_on_another_stream(B):
    """Outputs and workspaces that a call makes itself belong to the stream it runs on."""
    p, cache, q_sem, q_pos, n_rep, n_tok, qbar = decode_case(B, 40, 3)
    want = B.decode_attention_paged8(p, cache, q_sem, q_pos, n_rep, n_tok, want_lse=True)
    up = B.decode_update_paged8(p, cache, None, None, n_rep, n_tok, qbar=qbar)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for stream in (side, side.cuda_stream):
        for _ in range(3):
            x = torch.full((1 << 28,), 7, dtype=torch.uint8, device=DEV)       # written, and free for reuse, on the current stream
            x = x + 1
            del x
            out, lse = B.decode_attention_paged8(p, cache, q_sem, q_pos, n_rep, n_tok, want_lse=True, stream=stream)
            got = B.decode_update_paged8(p, cache, None, None, n_rep, n_tok, qbar=qbar, stream=stream)
            torch.cuda.synchronize()
            assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
            assert all(torch.equal(a, b) for a, b in zip(got, up))


def test_two_calls_at_once(B):
    """Two streams, each with its own cache and workspace, in flight together; then two graphs that share one workspace."""
    cases = [decode_case(B, 128, 5), decode_case(B, 16, 6, "gqa128", 2)]
    want = [B.decode_attention_paged8(*c[:6], want_lse=True) for c in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    got = [[] for _ in cases]
    for _ in range(20):
        for c, st, o in zip(cases, streams, got):
            o.append(B.decode_attention_paged8(*c[:6], want_lse=True, stream=st))
    torch.cuda.synchronize()
    for w, o in zip(want, got):
        assert all(torch.equal(x[0], w[0]) and torch.equal(x[1], w[1]) for x in o)
    ws = torch.empty(max(B.lca_paged8_workspace_bytes(c[0], c[1], 1) for c in cases), dtype=torch.uint8, device=DEV)
    outs = [torch.zeros_like(w[0]) for w in want]
    graphs = [torch.cuda.CUDAGraph() for _ in cases]
    for c, o, gr in zip(cases, outs, graphs):
        with torch.cuda.graph(gr):
            B.decode_attention_paged8(*c[:6], out=o, ws=ws)
    ws.fill_(0xff)
    for gr in graphs + graphs[::-1]:
        gr.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(o, w[0]) for o, w in zip(outs, want))


@pytest.mark.parametrize("shape,heads,kv,nb", [("mla512", 16, 1, 3), ("mla512", 128, 1, 40), ("gqa128", 8, 2, 300)])
def test_calls_in_a_row_equal_calls_one_by_one(B, shape, heads, kv, nb):
    """A decode loop of these calls and nothing between them, every one reading what the one before it wrote: as it comes, with
    a synchronisation after each call, and as a replayed graph, bit for bit."""
    variant, _, d_sem, d_pos = SHAPES[shape]
    g, w, page, steps = 16, 16, 16, 10
    width = 12
    p = B.make_params(variant, nb, 1, heads, kv, d_sem, d_pos, g, w, 0.07)
    gen = torch.Generator().manual_seed(11)
    rnd = lambda *x: torch.randn(x, generator=gen).bfloat16().to(DEV)          # noqa: E731
    start = torch.randint(0, 120, (nb,), generator=gen)
    n_tok = [(start + i).int().to(DEV) for i in range(steps + 1)]
    prompt = [rnd(int(start.sum()), kv, d) for d in (d_sem, d_pos)]
    new_rows = [[rnd(nb, kv, d) for d in (d_sem, d_pos)] for _ in range(steps)]
    q = [(rnd(nb, 1, heads, d_sem) if variant == "mla" else None, rnd(nb, 1, heads, d_pos)) for _ in range(steps)]
    qbar = torch.randn((nb, kv, d_pos + (d_sem if variant == "mla" else 0)), generator=gen).to(DEV)

    def state():
        cache = B.new_paged8_cache(p, nb * width, page, width, DEV)
        z = lambda n=nb, v=0, t=torch.int32: torch.full((n,), v, dtype=t, device=DEV)                       # noqa: E731
        n_rep = [z() for _ in range(steps + 1)]
        return dict(cache=cache, free=torch.arange(nb * width, dtype=torch.int32, device=DEV), n_free=z(1, nb * width), held=(z(), z()), n_rep=n_rep,
                    slots=z(max(1, int(start.sum()))), off=z(nb + 1), one=[z() for _ in range(2 * steps)], status=[z(1, -9) for _ in range(2 * steps + 1)],
                    out=[torch.zeros((nb, 1, heads, d_sem), dtype=torch.bfloat16, device=DEV) for _ in range(steps)],
                    rep=[[torch.zeros((nb, kv, d), dtype=torch.bfloat16, device=DEV) for d in (d_sem, d_pos)] for _ in range(steps)],
                    anchor=[torch.zeros((nb, kv), dtype=torch.int32, device=DEV) for _ in range(steps)],
                    ws=B.workspace_paged8(p, cache, 1, DEV), ws2=B.workspace(p, B.LCA_WS_UPDATE, DEV))

    def run(s, after):
        c, pages = s["cache"], (*s["held"], s["free"], s["n_free"])
        B.page_update(p, c, s["n_rep"][0], n_tok[0], *pages, s["slots"], s["off"], s["status"][-1]); after()
        B.paged8_write(p, c, *prompt, s["slots"]); after()
        for i in range(steps):
            B.page_update(p, c, s["n_rep"][i], n_tok[i + 1], *pages, s["one"][2 * i], None, s["status"][2 * i], rows_per_seq=1); after()
            B.paged8_write(p, c, *new_rows[i], s["one"][2 * i]); after()
            B.decode_attention_paged8(p, c, *q[i], s["n_rep"][i], n_tok[i + 1], out=s["out"][i], ws=s["ws"]); after()
            B.decode_update_paged8(p, c, None, None, s["n_rep"][i], n_tok[i + 1], s["n_rep"][i + 1], *s["rep"][i], qbar=qbar,
                                   anchor=s["anchor"][i], ws=s["ws2"]); after()
            B.page_update(p, c, s["n_rep"][i + 1], n_tok[i + 1], *pages, s["one"][2 * i + 1], None, s["status"][2 * i + 1], rows_per_seq=1); after()
            B.paged8_write(p, c, *s["rep"][i], s["one"][2 * i + 1]); after()

    states = [state() for _ in range(3)]
    run(states[0], torch.cuda.synchronize)
    run(states[1], lambda: None)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(states[2], lambda: None)
    graph.replay()
    torch.cuda.synchronize()

    def flat(s):
        return [*s["cache"].tensors, s["free"], s["n_free"], *s["held"], *s["n_rep"], s["slots"], *s["one"], *s["status"], *s["out"],
                *(x for r in s["rep"] for x in r), *s["anchor"]]
    assert all(int(x) == 0 for x in states[0]["status"]) and int((states[0]["n_rep"][-1] > 0).sum()) > 0
    for other in states[1:]:
        assert all(a is b or torch.equal(a, b) for a, b in zip(flat(states[0]), flat(other)))


def test_helpers_refuse_tensors_that_do_not_fit(B):
    p, cache, q_sem, q_pos, n_rep, n_tok, qbar = decode_case(B, 16, 4)
    before = B.lca_launch_count()
    more = B.make_params("mla", 4, 1, 16, 1, 512, 64, 64, 64, 0.07)             # a sequence more than the table has rows
    other = B.make_params("gqa", 3, 1, 16, 1, 128, 128, 64, 64, 0.07)
    calls = [lambda: B.decode_attention_paged8(p, cache, q_sem.half(), q_pos, n_rep, n_tok),
             lambda: B.decode_attention_paged8(p, cache, q_sem, q_pos[:2], n_rep, n_tok),
             lambda: B.decode_attention_paged8(p, cache, q_sem, q_pos.transpose(0, 2), n_rep, n_tok),
             lambda: B.decode_attention_paged8(p, cache, q_sem, q_pos, n_rep, n_tok.long()),
             lambda: B.decode_attention_paged8(p, cache, q_sem, q_pos, n_rep.cpu(), n_tok),
             lambda: B.decode_attention_paged8(p, cache, q_sem, q_pos, n_rep, n_tok, out=q_sem[:1]),
             lambda: B.decode_attention_paged8(more, cache, q_sem, q_pos, n_rep, n_tok),
             lambda: B.decode_attention_paged8(other, cache, None, q_pos, n_rep, n_tok),
             lambda: B.decode_update_paged8(p, cache, None, None, n_rep, n_tok, qbar=qbar.double()),
             lambda: B.decode_update_paged8(p, cache, None, None, n_rep, n_tok, qbar=qbar[:2]),
             lambda: B.decode_update_paged8(p, cache, q_sem, q_pos, n_rep, n_tok),                   # one position, not group_size
             lambda: B.paged8_write(p, cache, q_sem, q_pos, torch.zeros(100, dtype=torch.int32, device=DEV)),
             lambda: B.paged8_write(p, cache, q_sem, q_pos, torch.zeros(3, device=DEV)),
             lambda: B.page_update(p, cache, n_rep, n_tok, n_rep, n_tok, n_tok[:1], n_tok, None, None, n_tok)]
    for k, call in enumerate(calls):
        with pytest.raises(ValueError):
            call()
            pytest.fail("call %d was not refused" % k)
    assert B.lca_launch_count() == before


# --------------------------------------------------------------------------------------------------- the run of calls
@pytest.mark.parametrize("variant,kv,page", [("mla", 1, 16), ("gqa", 2, 16)])
def test_prompt_decode_and_condensation_together(B, variant, kv, page):
    """Prompts through lca_condense into pages, then a decode loop: every step a row per sequence, attention over the pages
    (against the 64-bit definition on the cache as it is), and the online update whenever a sequence is due."""
    g, w, heads = 16, 32, 8 * kv
    d_sem, d_pos = (512, 64) if variant == "mla" else (128, 128)
    shape = "mla512" if variant == "mla" else "gqa128"
    scale = 0.06
    lens = [70, 1, 200]
    nb = len(lens)
    gen = torch.Generator().manual_seed(7)
    rnd = lambda *s: torch.randn(s, generator=gen).bfloat16().to(DEV)          # noqa: E731
    p = B.make_params(variant, nb, max(lens), heads, kv, d_sem, d_pos, g, w, scale)
    T = sum(lens)
    q_sem, q_pos = (rnd(T, heads, d_sem) if variant == "mla" else None), rnd(T, heads, d_pos)
    cond = B.condense_varlen(p, lens, q_sem, q_pos, rnd(T, kv, d_sem), rnd(T, kv, d_pos))
    m = [int(b - a) for a, b in zip(cond["group_offsets"], cond["group_offsets"][1:])]
    n_pages = 48
    cache = B.new_paged8_cache(p, n_pages, page, 32, DEV)
    sem_p, pos_p, ss, sp, table = cache.tensors
    sem_p.fill_(0x7f); pos_p.fill_(0x7f); ss.fill_(float("nan"))              # what an earlier owner left
    free, n_free = i32(list(range(n_pages))), i32([n_pages])
    held_rep, held_tok, status = i32([0] * nb), i32([0] * nb), i32([5])
    n_rep, n_tok = i32(m), i32(lens)
    rows = cond["cache_row_offsets"][-1]
    slots = torch.empty(rows, dtype=torch.int32, device=DEV)
    offsets = torch.empty(nb + 1, dtype=torch.int32, device=DEV)
    B.page_update(p, cache, n_rep, n_tok, held_rep, held_tok, free, n_free, slots, offsets, status)
    B.paged8_write(p, cache, cond["cache_sem"], cond["cache_pos"], slots)
    assert int(status) == 0 and offsets.cpu().tolist() == [int(x) for x in cond["cache_row_offsets"]]
    one = torch.empty(nb, dtype=torch.int32, device=DEV)
    qbar = torch.randn((nb, kv, d_pos + (d_sem if variant == "mla" else 0)), generator=gen).to(DEV)
    updates = 0
    for step in range(60):
        n_tok += 1
        B.page_update(p, cache, n_rep, n_tok, held_rep, held_tok, free, n_free, one, None, status, rows_per_seq=1)
        B.paged8_write(p, cache, rnd(nb, kv, d_sem), rnd(nb, kv, d_pos), one)
        qs, qp = (rnd(nb, 1, heads, d_sem) if variant == "mla" else None), rnd(nb, 1, heads, d_pos)
        out, lse = B.decode_attention_paged8(p, cache, qs, qp, n_rep, n_tok, want_lse=True)
        assert int(status) == 0
        pools = [None if x is None else x.cpu().numpy() for x in (sem_p, pos_p, ss, sp)]
        if step % 7 == 0 or step > 50:
            want = R.attend(None if qs is None else qs.double().cpu().numpy(), qp.double().cpu().numpy(), *pools, table.cpu().numpy(),
                            n_rep.cpu().tolist(), n_tok.cpu().tolist(), g, page, scale)
            compare(out, lse, *want, n=300, top=1.0)
        new, rsem, rpos, anchor = B.decode_update_paged8(p, cache, None, None, n_rep, n_tok, qbar=qbar)
        ref = R.update(*pools, table.cpu().numpy(), n_rep.cpu().tolist(), n_tok.cpu().tolist(), qbar.cpu().numpy(), g, w, page, scale)
        assert new.cpu().tolist() == ref[0].tolist() and anchor.cpu().tolist() == ref[3].tolist()
        updates += int((new != n_rep).sum())
        n_rep.copy_(new)
        B.page_update(p, cache, n_rep, n_tok, held_rep, held_tok, free, n_free, one, None, status, rows_per_seq=1)
        B.paged8_write(p, cache, rsem, rpos, one)
        assert int(status) == 0
        # no more pages are held than the present rows need
        need = sum(-(-int(r) // page) + -(-int(t) // page) - int(r) * g // page for r, t in zip(n_rep.cpu(), n_tok.cpu()))
        assert int(n_free) == n_pages - need
    assert updates >= 8
