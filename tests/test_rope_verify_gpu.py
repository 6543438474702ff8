"""Rotary positions and draft verification on the GPU against 64-bit statements, and a speculative decode loop on the paged
4-bit cache in which all the calls work together."""
import math

import numpy as np
import pytest
import torch

from tests import paged4_reference as R

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


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


# --------------------------------------------------------------------------------------------------------------- rope
def check_rope(B, x, out, positions, freqs, **kw):
    """Angles are exact but for one fp32 rounding of less than half a turn (2^-25 turns: an angle of 2 pi 2^-25), cosine and sine are off by
    2 ulp (2^-22), the factor's and the two products and their sum by four roundings of 2^-24, the result by one of its type: half a step, which is
    2^-8 of a bf16 value (8 significant bits) and 2^-24 of an fp32 one."""
    want = R.rope(x.double().cpu().numpy(), positions.cpu().numpy(), freqs.cpu().numpy(), kw.get("interleaved", False), kw.get("inverse", False),
                  kw.get("factor", 1.0))
    rot, d = 2 * freqs.numel(), x.shape[-1]
    got = out.double().cpu().numpy()
    assert np.array_equal(got[..., rot:], x.double().cpu().numpy()[..., rot:])
    half = 2.0 ** -8 if x.dtype is torch.bfloat16 else 2.0 ** -24
    xs = np.abs(x.double().cpu().numpy()[..., :rot])
    other = np.stack([xs[..., 1::2], xs[..., 0::2]], -1).reshape(xs.shape) if kw.get("interleaved") else np.roll(xs, rot // 2, -1)
    tol = half * np.abs(want[..., :rot]) * (1 + 2.0 ** -7) + abs(kw.get("factor", 1.0)) * (xs + other) * (2 * math.pi * 2.0 ** -25 + 2.0 ** -22 + 4 * 2.0 ** -24)
    bad = np.abs(got[..., :rot] - want[..., :rot]) > tol + 1e-38
    assert not bad.any(), (int(bad.sum()), np.abs(got[..., :rot] - want[..., :rot]).max())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("T,heads,kv,d,rot", [(1, 1, 1, 64, 64), (7, 16, 1, 64, 64), (300, 5, 2, 128, 64), (33, 3, 1, 80, 32), (17, 2, 2, 10, 6), (5, 3, 1, 7, 2),
                                              (2, 130, 8, 128, 128), (9, 1, 1, 9000, 8192), (1000, 4, 4, 24, 16)])
def test_rope_layouts(B, dtype, interleaved, T, heads, kv, d, rot):
    g = torch.Generator(device=DEV).manual_seed(T + d)
    q, k = (torch.randn((T, h, d), generator=g, device=DEV).to(dtype) for h in (heads, kv))
    pos = torch.randint(0, 200000, (T,), generator=g, device=DEV, dtype=torch.int32)
    freqs, _ = B.rope_frequencies(rot, 10000.0, device=DEV)
    for kw in (dict(interleaved=interleaved), dict(interleaved=interleaved, inverse=True, factor=1.35)):
        qo, ko = B.rope(q, k, pos, freqs, **kw)
        check_rope(B, q, qo, pos, freqs, **kw)
        check_rope(B, k, ko, pos, freqs, **kw)
    only, none = B.rope(q, None, pos, freqs, interleaved=interleaved)
    assert none is None and torch.equal(only, B.rope(q, k, pos, freqs, interleaved=interleaved)[0])
    assert torch.equal(B.rope(None, k, pos, freqs, interleaved=interleaved)[1], B.rope(q, k, pos, freqs, interleaved=interleaved)[1])
    # in place
    q2, k2 = q.clone(), k.clone()
    B.rope(q2, k2, pos, freqs, interleaved=interleaved, q_out=q2, k_out=k2)
    qo, ko = B.rope(q, k, pos, freqs, interleaved=interleaved)
    assert torch.equal(q2, qo) and torch.equal(k2, ko)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("shift", [0, 8, 3])
def test_rope_on_slices_of_projections(B, interleaved, shift):
    # the last 64 of 192 columns of 16 heads, and the rope key behind a latent; `shift` moves the rows off their alignment
    g = torch.Generator(device=DEV).manual_seed(1)
    T = 37
    proj = torch.randn((T, 16 * 192 + 16), generator=g, device=DEV).bfloat16()
    q = proj[:, shift:shift + 16 * 192].view(T, 16, 192)[:, :, 128:] if shift == 0 else proj[:, shift:shift + 16 * 192].unflatten(1, (16, 192))[:, :, 128:]
    k = torch.randn((T, 1, 576 + shift), generator=g, device=DEV).bfloat16()[:, :, 512 + shift:]
    pos = torch.arange(T, device=DEV, dtype=torch.int32) * 3001
    freqs, factor = B.rope_frequencies(64, 10000.0, B.ROPE_RAMP, 32.0, 4096.0, device=DEV)
    before = proj.clone()
    qo, ko = B.rope(q, k, pos, freqs, interleaved=interleaved, factor=factor)
    check_rope(B, q, qo, pos, freqs, interleaved=interleaved, factor=factor)
    check_rope(B, k, ko, pos, freqs, interleaved=interleaved, factor=factor)
    assert torch.equal(proj, before)
    # into a slice of a larger buffer: what is around it stays
    buf = torch.full((T, 16, 200), 7.0, dtype=torch.bfloat16, device=DEV)
    B.rope(q, None, pos, freqs, interleaved=interleaved, factor=factor, q_out=buf[:, :, 70 + shift:134 + shift])
    assert torch.equal(buf[:, :, 70 + shift:134 + shift], qo) and torch.all(buf[:, :, :70 + shift] == 7) and torch.all(buf[:, :, 134 + shift:] == 7)


def test_rope_far_and_negative_positions(B):
    pos = i32([0, 1, 999983, 2 ** 31 - 1, -1, -(2 ** 31), 16777217])
    x = torch.ones((7, 2, 64), device=DEV)
    freqs, _ = B.rope_frequencies(64, 10000.0, device=DEV)
    # the reference's own angle, a product rounded to 64 bits, is off by up to 2^31 * 2^-53, and its reduction by as much: 2^-20 in all
    out, _ = B.rope(x, None, pos, freqs)
    want = R.rope(x.double().cpu().numpy(), pos.cpu().numpy(), freqs.cpu().numpy(), False, False, 1.0)
    assert np.abs(out.double().cpu().numpy() - want).max() < 4e-6


@pytest.mark.parametrize("interleaved", [False, True])
def test_rope_gradient_is_the_inverse(B, interleaved):
    # of f(x) = <w, rope(x)>: the formula's gradient is the inverse rotation of w, and so are differences of f (which is linear)
    g = torch.Generator(device=DEV).manual_seed(3)
    x, w = (torch.randn((6, 2, 32), generator=g, device=DEV) for _ in range(2))
    pos = i32([0, 5, 100, 4000, 70000, 123456])
    freqs, _ = B.rope_frequencies(16, 10000.0, device=DEV)
    kw = dict(interleaved=interleaved, factor=1.1)
    grad, _ = B.rope(w, None, pos, freqs, inverse=True, **kw)
    xr = x.double().cpu().numpy()
    f = lambda y: (R.rope(y, pos.cpu().numpy(), freqs.cpu().numpy(), interleaved, False, 1.1)[..., :16] * w.double().cpu().numpy()[..., :16]).sum()  # noqa: E731
    for at in [(0, 0, 0), (1, 1, 3), (2, 0, 9), (4, 1, 15), (5, 0, 8)]:
        h = np.zeros_like(xr)
        h[at] = 0.5
        assert abs((f(xr + h) - f(xr - h)) - float(grad[at])) < 1e-5
    # there and back with factor 1: two roundings of 2^-22 each and those of the products
    y, _ = B.rope(x, None, pos, freqs, interleaved=interleaved)
    z, _ = B.rope(y, None, pos, freqs, interleaved=interleaved, inverse=True)
    assert float((z - x).abs().max()) < 16 * 2.0 ** -22 * float(x.abs().max())


def test_rope_refuses_what_does_not_fit(B):
    x = torch.zeros((4, 2, 64), dtype=torch.bfloat16, device=DEV)
    pos, f = torch.zeros(4, dtype=torch.int32, device=DEV), torch.zeros(32, dtype=torch.float64, device=DEV)
    for bad in (dict(q=x.half()), dict(positions=pos[:3]), dict(positions=pos.long()), dict(freqs=f.float()), dict(k=x[:3]), dict(k=x.float()),
                dict(q=x.transpose(1, 2)), dict(q_out=x[:, :1]), dict(q_out=x[:, :1].expand(4, 2, 64)), dict(q_out=x[:1].expand(4, 2, 64)),
                dict(k=torch.zeros((4, 2, 32), dtype=torch.bfloat16, device=DEV))):
        a = dict(q=x, k=None, positions=pos, freqs=f)
        a.update(bad)
        with pytest.raises(ValueError):
            B.rope(**a)
    with pytest.raises(B.LcaError):
        B.rope(x, None, pos, torch.zeros(40, dtype=torch.float64, device=DEV))         # 80 rotated columns of 64
    B.rope(x[:0], None, pos[:0], f)


# ------------------------------------------------------------------------------------------------------------- verify
def check_verify(B, target, draft, tokens, u_accept, u_sample, n_draft=None, n_tok=None):
    acc, out, left = B.verify_drafts(target, draft, tokens, u_accept, u_sample, n_draft=n_draft, n_tok=n_tok)
    nb, n1, V = target.shape
    t, d = target.double().cpu().numpy(), None if draft is None else draft.double().cpu().numpy()
    for b in range(nb):
        n = n1 - 1 if n_draft is None else int(n_draft[b])
        k, want = R.verify(t[b], None if d is None else d[b], tokens[b].tolist(), u_accept[b].tolist(), float(u_sample[b]), n)
        assert int(acc[b]) == k and out[b].tolist() == want.tolist(), (b, int(acc[b]), k, out[b].tolist(), want.tolist())
        if n_tok is not None:
            assert int(left[b]) == int(n_tok[b]) - (min(max(n, 0), n1 - 1) - k)
    return acc, out


def make(nb, n, V, seed, dtype, sharp=2.5):
    g = torch.Generator(device=DEV).manual_seed(seed)
    z = torch.randn((nb, n + 1, V), generator=g, device=DEV) * sharp
    target = torch.softmax(z, -1).to(dtype)
    q = torch.softmax(z[:, :n] + torch.randn((nb, n, V), generator=g, device=DEV) * 0.7, -1).to(dtype)
    tokens = (q.float() / -torch.log(torch.rand((nb, n, V), generator=g, device=DEV).clamp(min=1e-30))).argmax(-1).int() if n else i32([[]] * nb)
    return target, q, tokens, torch.rand((nb, n), generator=g, device=DEV), torch.rand((nb,), generator=g, device=DEV)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("nb,n,V", [(1, 1, 1), (2, 3, 2), (5, 4, 7), (3, 0, 100), (1, 7, 32001), (40, 3, 4099), (500, 2, 130), (7, 40, 1000), (3, 2, 128000), (1, 1, 1000003)])
def test_verify_against_the_definition(B, dtype, nb, n, V):
    target, q, tokens, ua, us = make(nb, n, V, nb + V, dtype)
    n_tok = torch.arange(100, 100 + nb, dtype=torch.int32, device=DEV)
    check_verify(B, target, q, tokens, ua, us, n_tok=n_tok)
    check_verify(B, target, None, tokens, ua, us)
    g = torch.Generator(device=DEV).manual_seed(9)
    check_verify(B, target, q, tokens, ua, us, n_draft=torch.randint(-1, n + 3, (nb,), generator=g, device=DEV, dtype=torch.int32), n_tok=n_tok)


def test_verify_at_the_ends_of_the_random_numbers(B):
    target, q, tokens, ua, us = make(6, 3, 977, 5, torch.float32)
    last = 1.0 - 2.0 ** -24
    for a, s in ((0.0, 0.0), (last, last), (0.0, last), (last, 0.0)):
        check_verify(B, target, q, tokens, torch.full_like(ua, a), torch.full_like(us, s))
    # zero probabilities before the first and behind the last possible token: never drawn
    target[:, :, :100] = 0
    target[:, :, 900:] = 0
    for s in (0.0, last, 0.5):
        acc, out = check_verify(B, target, q, tokens, torch.full_like(ua, last), torch.full_like(us, s))
        new = out.gather(1, acc[:, None].long())
        assert torch.all((new >= 100) & (new < 900))


def test_verify_equal_distributions_accept_everything_and_disjoint_ones_nothing(B):
    target, q, tokens, ua, us = make(8, 5, 500, 6, torch.float32)
    ua = ua * 0.999
    acc, out = check_verify(B, target, target[:, :5].contiguous(), tokens, ua, us)
    ok = target[:, :5].gather(2, tokens[..., None].long())[..., 0] > 0
    assert torch.equal(acc, torch.cumprod(ok.int(), 1).sum(1).int())
    p, d = torch.zeros_like(target), torch.zeros_like(q)
    p[..., 250:], d[..., :250] = target[..., 250:], q[..., :250]
    low = d.argmax(-1).int()
    acc, out = check_verify(B, p, d, low, ua, us)
    assert torch.all(acc == 0) and torch.all(out[:, 0] >= 250) and torch.all(out[:, 1:] == -1)


def test_verify_odd_inputs(B):
    target, q, tokens, ua, us = make(9, 2, 300, 7, torch.float32)
    tokens[0, 0], tokens[1, 0], tokens[2, 1] = -1, 300, 2 ** 31 - 1           # no such token: rejected
    target[3, :, 5], target[3, :, 7], q[3, :, 9] = float("nan"), float("inf"), float("nan")
    target[4] = 0                                                              # nothing to draw from
    target[5, 0] = q[5, 0] * 0.5                                               # the rest is empty: drawn from p
    tokens[5, 0] = int(q[5, 0].argmax())
    ua[5, 0] = 0.9
    target[6] = -1.0
    target[7] *= 1e-30                                                         # sums far from 1
    target[8, 0], q[8, 0] = q[8, 0] * 3e38, q[8, 0]
    check_verify(B, target, q, tokens, ua, us)
    check_verify(B, target, None, tokens, ua, us)


def test_verify_unaligned_rows_streams_and_graphs(B):
    # rows of odd length in a buffer that starts at any element
    V, n, nb = 1237, 3, 4
    target, q, tokens, ua, us = make(nb, n, V, 8, torch.bfloat16)
    buf = torch.zeros(target.numel() + q.numel() + 8, dtype=torch.bfloat16, device=DEV)
    t2 = buf[1:1 + target.numel()].view_as(target).copy_(target)
    q2 = buf[5 + target.numel():5 + target.numel() + q.numel()].view_as(q).copy_(q)
    want = check_verify(B, target, q, tokens, ua, us)
    got = check_verify(B, t2, q2, tokens, ua, us)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    a, o, _ = B.verify_drafts(target, q, tokens, ua, us, stream=side)
    side.synchronize()
    assert torch.equal(a, want[0]) and torch.equal(o, want[1])
    n_tok = i32([50] * nb)
    acc, out = torch.empty_like(want[0]), torch.empty_like(want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.verify_drafts(target, q, tokens, ua, us, n_tok=n_tok, accepted=acc, out=out, n_tok_out=n_tok)      # in place
    n_tok.fill_(50)
    graph.replay()
    graph.replay()
    assert torch.equal(acc, want[0]) and torch.equal(out, want[1]) and n_tok.tolist() == [50 - 2 * (n - int(x)) for x in want[0]]


def test_verify_refuses_what_does_not_fit(B):
    target, q, tokens, ua, us = make(2, 3, 50, 1, torch.float32)
    for bad in (dict(target_probs=target.half()), dict(draft_probs=q[:1]), dict(draft_probs=q.bfloat16()), dict(draft_tokens=tokens.long()),
                dict(draft_tokens=tokens[:1]), dict(u_accept=ua.double()), dict(u_sample=us[:1]), dict(n_draft=tokens[0, :1]),
                dict(target_probs=target.transpose(0, 1))):
        a = dict(target_probs=target, draft_probs=q, draft_tokens=tokens, u_accept=ua, u_sample=us)
        a.update(bad)
        with pytest.raises(ValueError):
            B.verify_drafts(**a)


# ------------------------------------------------------------------------------------------------------- all together
@pytest.mark.parametrize("variant", ["mla", "gqa"])
def test_speculative_decode_loop(B, variant):
    """Prompts into pages, then steps of drafts: rotate, take slots, write, attend, verify, roll back, condense.  Every step's outputs
    are compared with 64-bit statements over the values that the cache holds."""
    g, w, page, nb, k = 32, 64, 16, 3, 2
    H, kv, ds, dp = (16, 1, 512, 64) if variant == "mla" else (4, 2, 64, 64)
    scale = 1.0 / math.sqrt(192.0 if variant == "mla" else dp)
    p = B.make_params(variant, nb, 1, H, kv, ds, dp, g, w, scale)
    n_pages, width, V = 60, 20, 60
    cache = B.new_paged4_cache(p, n_pages, page, width, DEV)
    free, n_free, status = torch.randperm(n_pages, device=DEV).int(), i32([n_pages]), i32([0])
    held_rep, held_tok, n_rep, n_tok = (i32([0] * nb) for _ in range(4))
    gen = torch.Generator(device=DEV).manual_seed(4)
    rnd = lambda *s: torch.randn(s, generator=gen, device=DEV)  # noqa: E731
    freqs, factor = B.rope_frequencies(dp, 10000.0, B.ROPE_LINEAR, 4.0, device=DEV)
    state = (held_rep, held_tok, free, n_free)
    # prompts
    lens = [90, 17, 130]
    n_tok.copy_(i32(lens))
    T = sum(lens)
    slots, offsets = torch.empty(T, dtype=torch.int32, device=DEV), torch.empty(nb + 1, dtype=torch.int32, device=DEV)
    B.page_update(p, cache, n_rep, n_tok, *state, slots, offsets, status)
    at = torch.cat([torch.arange(n, dtype=torch.int32, device=DEV) for n in lens])
    sem, raw = rnd(T, kv, ds).bfloat16(), rnd(T, kv, dp).bfloat16()
    _, pos = B.rope(None, raw, at, freqs, factor=factor)
    B.paged4_write(p, cache, sem, pos, slots)
    condensed = 0
    for step in range(14):
        q_len = k + 1
        n_tok += q_len
        slot = torch.empty(nb * q_len, dtype=torch.int32, device=DEV)
        B.page_update(p, cache, n_rep, n_tok, *state, slot, None, status, rows_per_seq=q_len)
        at = (n_tok[:, None] - q_len + torch.arange(q_len, dtype=torch.int32, device=DEV)).reshape(-1).int()
        q_raw, k_raw = rnd(nb * q_len, H, dp).bfloat16(), rnd(nb * q_len, kv, dp).bfloat16()
        q_pos, k_pos = B.rope(q_raw, k_raw, at, freqs, factor=factor)
        check_rope(B, q_raw, q_pos, at, freqs, factor=factor)
        v_new = rnd(nb * q_len, kv, ds).bfloat16()
        B.paged4_write(p, cache, v_new, k_pos, slot)
        q_sem = rnd(nb, q_len, H, ds).bfloat16() if variant == "mla" else None
        out, lse = B.decode_attention_paged4(p, cache, q_sem, q_pos.view(nb, q_len, H, dp), n_rep, n_tok, want_lse=True)
        assert int(status) == 0
        pool = R.Pool(n_pages, kv, page, ds, dp, variant == "mla", 0)
        names = ("pages_sem", "pages_pos", "shift_sem", "shift_pos", "exp_sem", "exp_pos")
        for name, t in zip(names, cache.tensors):
            setattr(pool, name, None if t is None else t.cpu().numpy())
        table = cache.tensors[6].cpu().numpy()
        want, want_lse, _, _ = R.attend(None if q_sem is None else q_sem.double().cpu().numpy(), q_pos.view(nb, q_len, H, dp).double().cpu().numpy(), pool,
                                        table, n_rep.tolist(), n_tok.tolist(), g, scale)
        got = out.double().cpu().numpy()
        assert np.all(np.linalg.norm(got - want, axis=-1) <= 2.0 ** -8 * np.linalg.norm(want, axis=-1))
        assert np.abs(lse.double().cpu().numpy() - want_lse).max() < 1e-4
        # verification: the rejected drafts leave the cache
        target, q, tokens, ua, us = make(nb, k, V, 100 + step, torch.float32, sharp=1.0)
        before = n_tok.clone()
        acc, _, _ = B.verify_drafts(target, q, tokens, ua, us, n_tok=n_tok, n_tok_out=n_tok)
        check_verify(B, target, q, tokens, ua, us)
        assert torch.equal(n_tok, before - (k - acc))
        B.page_update(p, cache, n_rep, n_tok, *state, None, None, status)
        # condensation of the groups that are due
        dk = dp + (ds if variant == "mla" else 0)
        qbar = rnd(nb, kv, dk) * 0.3
        new, rs, rp, anchor = B.decode_update_paged4(p, cache, None, None, n_rep, n_tok, qbar=qbar)
        ref = R.update(pool, cache.tensors[6].cpu().numpy(), n_rep.tolist(), n_tok.tolist(), qbar.cpu().numpy(), g, w, scale)
        assert new.tolist() == ref[0].tolist() and anchor.tolist() == ref[3].tolist()
        condensed += int((new - n_rep).sum())
        n_rep.copy_(new)
        slot = torch.empty(nb, dtype=torch.int32, device=DEV)
        B.page_update(p, cache, n_rep, n_tok, *state, slot, None, status, rows_per_seq=1)
        B.paged4_write(p, cache, rs, rp, slot)
        due = [b for b in range(nb) if b in ref[1]]
        if due:
            s, r = B.paged4_read(p, cache, slot)
            for b in due:                                                      # a representative is quantised like any row: a third of a block's largest
                top = np.abs(ref[1][b]).max()
                assert np.abs(s[b].double().cpu().numpy() - ref[1][b]).max() <= top * (1 / 3 + 2.0 ** -7)
        assert int(status) == 0
    assert condensed >= 3
    n_rep.zero_(), n_tok.zero_()
    B.page_update(p, cache, n_rep, n_tok, *state, None, None, status)
    assert int(n_free) == n_pages and int(status) == 0
