"""Paged 4-bit cache, rotary positions and draft verification, host side: invalid calls are refused before anything is
launched, frequencies, and the 64-bit references against themselves (no GPU needed)."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from tests import paged4_reference as R


@pytest.fixture(scope="module")
def B():
    from paper_2604_12452_b200 import build
    build.build()
    from paper_2604_12452_b200 import binding
    return binding


def cache(B, **kw):
    c = B.LcaPaged4(16, 16, 16, 16, 16, None, 16, 8, 16, 4)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


@pytest.fixture()
def p(B):
    return B.make_params("mla", 2, 1, 16, 1, 512, 64, 64, 64, 0.07)


def test_write_and_read_refusals(B, p):
    before = B.lca_launch_count()
    for fn in (B.lca_paged4_write, B.lca_paged4_read):
        call = lambda c=None, sem=16, pos=16, slots=16, n=8, q=None: fn(q or p, c or cache(B), sem, pos, slots, n)  # noqa: E731
        assert call(sem=None) == -1 and call(pos=None) == -1 and call(slots=None) == -1 and call(n=-1) == -1 and call(n=1 << 31) == -1
        assert call(n=0) == 0
        assert call(sem=24) == -3 and call(pos=24) == -3 and call(c=cache(B, pages_sem=24)) == -3 and call(c=cache(B, shift_pos=20)) == -3 and call(c=cache(B, exp_sem=24)) == -3
        for k in ("pages_sem", "pages_pos", "shift_sem", "shift_pos", "exp_sem"):
            assert call(c=cache(B, **{k: None})) == -1, k
        assert call(c=cache(B, exp_pos=16)) == -1                             # MLA: one exponent for both
        gqa = B.make_params("gqa", 2, 1, 16, 2, 128, 128, 64, 64, 0.07)
        assert call(q=gqa) == -1                                              # GQA: two
        assert call(q=B.make_params("mla", 2, 1, 16, 1, 256, 64, 64, 64, 0.07)) == -2
        assert call(c=cache(B, page_size=48)) == -2 and call(c=cache(B, n_pages=0)) == -1 and call(c=cache(B, n_pages=1 << 28)) == -1
    assert B.lca_launch_count() == before


def test_attention_and_update_refusals(B, p):
    before = B.lca_launch_count()
    big = 1 << 40
    call = lambda c=None, qs=16, qp=16, n=1, nr=16, nt=16, out=16, ws=16, wsb=big, q=None: B.lca_decode_attention_paged4(  # noqa: E731
        q or p, c or cache(B), qs, qp, n, nr, nt, out, None, ws, wsb)
    assert call(qs=None) == -1 and call(qp=None) == -1 and call(nt=None) == -1 and call(out=None) == -1 and call(n=0) == -1
    assert call(ws=None) == -1 and call(ws=24) == -1 and call(wsb=64) == -4
    assert call(qs=24) == -3 and call(qp=24) == -3 and call(out=24) == -3
    assert call(c=cache(B, page_size=128)) == -1                              # with representatives: group % page
    assert call(c=cache(B, block_table=None)) == -1 and call(c=cache(B, page_size=8)) == -2
    assert call(n=1 << 30) == -1                                              # 2^35 query rows
    need = B.lca_paged4_workspace_bytes(p, cache(B), 1)
    assert need > 0 and call(wsb=need - 1) == -4
    assert B.lca_paged4_workspace_bytes(p, cache(B), 0) == 0 and B.lca_paged4_workspace_bytes(p, cache(B, page_size=5), 1) == 0
    up = lambda c=None, tail=16, qbar=None, nr=16, nt=16, new=32, sem=16, pos=16, an=16, ws=16, wsb=big, stride=64, q=None: B.lca_decode_update_paged4(  # noqa: E731
        q or p, c or cache(B), tail, tail, stride, qbar, nr, nt, new, sem, pos, an, ws, wsb)
    assert up(nr=None) == -1 and up(nt=None) == -1 and up(new=None) == -1 and up(new=16) == -1      # n_rep_new is another array
    assert up(sem=None) == -1 and up(pos=None) == -1 and up(an=None) == -1 and up(tail=None) == -1
    assert up(stride=63) == -1 and up(ws=None) == -1 and up(wsb=8) == -4 and up(sem=24) == -3 and up(tail=24) == -3
    wide = B.make_params("mla", 2, 1, 16, 1, 512, 64, 512, 64, 0.07)
    assert up(q=wide, stride=512) == -2                                       # 512 rows of 576 bytes exceed shared memory
    assert B.lca_launch_count() == before


def rope_args(B, **kw):
    a = B.LcaRopeArgs(0, 0, 0, 4, 2, 64, 64, 1.0, 8, 16, 16, 16, 256, 64, 16, 256, 64, 16, 128, 64, 16, 128, 64)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def test_rope_refusals(B):
    before = B.lca_launch_count()
    call = lambda **kw: B.lca_rope(rope_args(B, **kw))  # noqa: E731
    assert B._lib.lca_rope(None, None) == -1
    for kw in (dict(dtype=2), dict(interleaved=2), dict(inverse=-1), dict(q=None), dict(k_out=None), dict(q=None, q_out=None, k=None, k_out=None),
               dict(n_q_heads=0), dict(n_k_heads=-1), dict(n_tokens=-1), dict(head_dim=0), dict(rot_dim=0), dict(rot_dim=7), dict(rot_dim=66),
               dict(factor=float("nan")), dict(factor=float("inf")), dict(positions=None), dict(freqs=None), dict(head_dim=70000, rot_dim=64),
               dict(head_dim=16384, rot_dim=16384)):
        assert call(**kw) == -1, kw
    assert call(q=17) == -3 and call(k_out=17) == -3 and call(dtype=1, q_out=18) == -3
    assert call(positions=18) == -3 and call(freqs=20) == -3
    assert call(n_tokens=0, positions=None) == 0
    assert B.lca_launch_count() == before
    x = torch.zeros((3, 2, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        B.rope(x, None, torch.zeros(3, dtype=torch.int32), torch.zeros(32, dtype=torch.float64))      # not on a CUDA device
    with pytest.raises(ValueError):
        B.rope(None, None, None, None)


def test_rope_frequencies(B):
    f, factor = B.rope_frequencies(64, 10000.0, device="cpu")
    want = torch.tensor([10000.0 ** (-2 * i / 64) for i in range(32)], dtype=torch.float64)
    assert torch.allclose(f, want, rtol=1e-15, atol=0) and factor == 1.0
    f, factor = B.rope_frequencies(64, 10000.0, B.ROPE_LINEAR, 8.0, device="cpu")
    assert torch.allclose(f, want / 8, rtol=1e-15, atol=0) and factor == 1.0
    f, factor = B.rope_frequencies(64, 10000.0, B.ROPE_BASE, 8.0, device="cpu")
    assert f[0] == 1.0 and abs(float(f[31] * 8 / want[31]) - 1) < 1e-12 and factor == 1.0       # the slowest pair is 8 times slower
    f, factor = B.rope_frequencies(64, 10000.0, B.ROPE_RAMP, 32.0, 4096.0, device="cpu")
    turns = 4096 * want / (2 * math.pi)
    keep = ((turns - 1) / 31).clamp(0, 1)
    assert torch.allclose(f, want * keep + want / 32 * (1 - keep), rtol=1e-14, atol=0) and abs(factor - (0.1 * math.log(32) + 1)) < 1e-6
    assert float(f[0]) == 1.0 and abs(float(f[31] * 32 / want[31]) - 1) < 1e-12
    bad = [(4, 64, 1e4, 1.0), (-1, 64, 1e4, 1.0), (0, 63, 1e4, 1.0), (0, 0, 1e4, 1.0), (0, 64, 0.0, 1.0), (0, 64, float("inf"), 1.0), (1, 64, 1e4, 0.0),
           (1, 64, 1e4, float("nan")), (2, 2, 1e4, 2.0), (3, 64, 1e4, 2.0)]
    for kind, rot, base, scale in bad:
        with pytest.raises(B.LcaError):
            B.rope_frequencies(rot, base, kind, scale, device="cpu")
    with pytest.raises(B.LcaError):
        B.rope_frequencies(64, 1e4, B.ROPE_RAMP, 2.0, 4096.0, fast=1.0, slow=1.0, device="cpu")
    assert B.lca_rope_frequencies(0, 64, 1e4, 1.0, 0.0, 32.0, 1.0, None, C.c_float()) == -1
    assert B.lca_rope_frequencies(0, 64, 1e4, 1.0, 0.0, 32.0, 1.0, (C.c_double * 32)(), None) == -1


def test_verify_refusals(B):
    before = B.lca_launch_count()
    def call(**kw):
        a = B.LcaVerifyArgs(1, 2, 3, 100, 16, 16, 16, None, 16, 16, 16, 16, 16, 16)
        for k, v in kw.items():
            setattr(a, k, v)
        return B.lca_verify_drafts(a)
    assert B._lib.lca_verify_drafts(None, None) == -1
    for kw in (dict(dtype=2), dict(batch=0), dict(n_drafts=-1), dict(vocab=0), dict(target_probs=None), dict(draft_tokens=None), dict(u_accept=None),
               dict(u_sample=None), dict(accepted=None), dict(tokens_out=None), dict(n_tok=None), dict(n_tok_out=None)):
        assert call(**kw) == -1, kw
    assert call(target_probs=18) == -3 and call(draft_probs=18) == -3 and call(dtype=0, draft_probs=17) == -3
    for name in ("draft_tokens", "n_draft", "u_accept", "u_sample", "n_tok", "accepted", "tokens_out", "n_tok_out"):
        assert call(**{name: 18}) == -3, name
    assert call(vocab=0x7fffffff) == -2 and call(vocab=0x7fffffff - 4095) == -2
    assert B.lca_launch_count() == before
    with pytest.raises(ValueError):
        B.verify_drafts(torch.zeros((2, 4, 100)), None, torch.zeros((2, 3), dtype=torch.int32), torch.zeros((2, 3)), torch.zeros(2))


def test_descriptor_refuses_tensors_that_do_not_fit_together(B):
    u8 = lambda *s: torch.zeros(s, dtype=torch.uint8)  # noqa: E731
    good = [u8(4, 2, 16, 64), u8(4, 2, 16, 64), u8(4, 2, 16, 2), u8(4, 2, 16, 2), u8(4, 2, 16), u8(4, 2, 16), torch.zeros((2, 3), dtype=torch.int32)]
    c = B.paged4_cache(*good)
    assert (c.n_pages, c.page_size, c.table_width, c.layout) == (4, 16, 3, (2, 128, 128))
    assert (c.pages.n_pages, c.pages.page_size, c.pages.table_width) == (4, 16, 3)
    bad = {0: [None, u8(4, 2, 16), u8(4, 2, 16, 64).float(), u8(4, 2, 16, 128)[..., ::2]], 1: [None, u8(3, 2, 16, 64)], 2: [None, u8(4, 2, 16, 4)],
           3: [u8(4, 2, 16, 1)], 4: [None, u8(4, 2, 8)], 5: [u8(4, 1, 16)], 6: [torch.zeros((2, 3)), torch.zeros(3, dtype=torch.int32)]}
    for i, xs in bad.items():
        for x in xs:
            args = list(good)
            args[i] = x
            with pytest.raises(ValueError):
                B.paged4_cache(*args)


def test_helpers_refuse_tensors_that_are_not_on_the_current_device(B, p):
    c = B.new_paged4_cache(p, 8, 16, 4, "cpu")
    i = torch.zeros(64, dtype=torch.int32)
    before = B.lca_launch_count()
    rows = torch.zeros((4, 1, 512), dtype=torch.bfloat16), torch.zeros((4, 1, 64), dtype=torch.bfloat16)
    for call in (lambda: B.page_update(p, c, i, i, i, i, i, i, i, i, i), lambda: B.paged4_write(p, c, *rows, i[:4]), lambda: B.paged4_read(p, c, i[:4], *rows),
                 lambda: B.decode_attention_paged4(p, c, torch.zeros((2, 1, 16, 512)).bfloat16(), torch.zeros((2, 1, 16, 64)).bfloat16(), i, i),
                 lambda: B.decode_update_paged4(p, c, None, None, i, i, qbar=torch.zeros((2, 1, 576)))):
        with pytest.raises(ValueError):
            call()
    assert B.lca_launch_count() == before


def test_reference_format():
    r = np.random.RandomState(0)
    x = r.randn(3, 2, 128) * np.exp(r.randn(3, 2, 1) * 3)
    pool = R.Pool(2, 2, 16, 128, 128, False, 0)
    pool.write(x, 2 * x, [3, 17, 30])
    v = pool.sem()[[0, 1, 1], :, [3, 1, 14]]
    # half the widest step, 2, of a block whose largest is at least 3: a third of it
    block = np.abs(x).reshape(3, 2, 4, 32).max(-1).repeat(32, -1)
    assert np.all(np.abs(v - x) <= block / 3)
    assert np.array_equal(R.unpack(R.pack(np.arange(16).reshape(2, 8))), np.arange(16).reshape(2, 8))
    (codes, shifts), E = R.encode_row([np.concatenate([np.full(32, 6.0), np.full(32, 6.0 * 2.0 ** -20)])])[0][0], 0
    assert codes[0] == 7 and list(shifts) == [0, 14] and codes[40] == 0


def test_reference_verification_is_the_targets_distribution():
    # over a grid of random numbers the tokens come out with the target's probabilities
    target = np.array([[0.5, 0.3, 0.2], [0.1, 0.2, 0.7]])
    draft = np.array([[0.2, 0.6, 0.2]])
    n = 200
    u = (np.arange(n) + 0.5) / n
    count = np.zeros(3)
    for x in range(3):
        for a in u:
            for b in u[::10]:
                k, out = R.verify(target, draft, [x], [a], b, 1)
                count[out[0]] += draft[0, x]
    assert np.allclose(count / count.sum(), target[0], atol=0.01)
