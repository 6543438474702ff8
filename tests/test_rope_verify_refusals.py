"""Rotary positions and draft verification, host side: calls whose sizes or addresses no kernel may be given (no GPU needed)."""
import pytest
import torch

from tests.test_paged4 import B  # noqa: F401


def verify(B, **kw):
    a = B.LcaVerifyArgs(1, 2, 3, 100, 16, 16, 16, None, 16, 16, 16, 16, 16, 16)
    for k, v in kw.items():
        setattr(a, k, v)
    return B.lca_verify_drafts(a)


@pytest.mark.parametrize("n_drafts", [0x7fffffff, 0x7fffffff - 1, 0x7fffffff - 256, 0x7fffffff - 4095])
def test_more_drafts_than_a_step_of_a_block_can_be_added_to(B, n_drafts):
    # (the kernel counts drafts with 32 bits, 256 at a time)
    before = B.lca_launch_count()
    assert verify(B, n_drafts=n_drafts, vocab=1) == -2
    assert B.lca_launch_count() == before


def rope(B, **kw):
    a = B.LcaRopeArgs(0, 0, 0, 4, 2, 64, 64, 1.0, 8, 16, 16, 1 << 20, 256, 64, 2 << 20, 256, 64, 3 << 20, 128, 64, 4 << 20, 128, 64)
    for k, v in kw.items():
        setattr(a, k, v)
    return B.lca_rope(a)


def test_outputs_on_what_others_read_or_write(B):
    before = B.lca_launch_count()
    q, q_out, k, k_out = (i << 20 for i in (1, 2, 3, 4))
    for kw in (dict(q_out=k), dict(k_out=q), dict(k_out=q_out), dict(k=q, q_out=q), dict(k=q, k_out=q), dict(k=q, q_out=q, k_out=q)):
        assert rope(B, **kw) == -1, kw
    # in place, but element for element
    for kw in (dict(q_out=q, q_out_token_stride=512), dict(q_out=q, q_head_stride=192), dict(k_out=k, k_token_stride=576), dict(k_out=k, k_out_head_stride=80),
               dict(k=None, k_out=None, q_out=q, q_token_stride=768)):
        assert rope(B, **kw) == -1, kw
    assert B.lca_launch_count() == before


@pytest.fixture()
def on_host(B, monkeypatch):
    """The verify helper with its checks alone: tensors of the host stand for the device's, and the library is not called."""
    monkeypatch.setattr(B, "_device", lambda x, where: x.get_device())
    monkeypatch.setattr(B, "_raw_stream", lambda dev, stream: 0)
    monkeypatch.setattr(B._lib, "lca_verify_drafts", lambda *a: 0)
    i32, f32 = dict(dtype=torch.int32), dict(dtype=torch.float32)
    good = dict(target_probs=torch.zeros((2, 4, 9), **f32), draft_probs=torch.zeros((2, 3, 9), **f32), draft_tokens=torch.zeros((2, 3), **i32),
                u_accept=torch.zeros((2, 3), **f32), u_sample=torch.zeros(2, **f32))
    return lambda **kw: B.verify_drafts(**{**good, **kw})


def test_rows_of_another_length_are_not_taken_for_a_request_s(on_host):
    i32, f32 = dict(dtype=torch.int32), dict(dtype=torch.float32)
    on_host()
    on_host(draft_tokens=torch.zeros((5, 3), **i32), u_accept=torch.zeros((2 * 3,), **f32), out=torch.zeros((3, 4), **i32))      # more requests, no rows at all
    for bad in (dict(draft_tokens=torch.zeros((2, 4), **i32)), dict(u_accept=torch.zeros((2, 5), **f32)), dict(out=torch.zeros((2, 5), **i32)),
                dict(u_accept=torch.zeros((3, 2), **f32)), dict(draft_tokens=torch.zeros((7,), **i32)), dict(out=torch.zeros((4, 4, 1), **i32))):
        with pytest.raises(ValueError):
            on_host(**bad)


def test_counters_out_without_counters_in(on_host):
    n = torch.full((2,), 7, dtype=torch.int32)
    assert on_host()[2] is None and on_host(n_tok=n, n_tok_out=n)[2] is n
    with pytest.raises(ValueError):                                            # not left as it was, with no word
        on_host(n_tok_out=n)
