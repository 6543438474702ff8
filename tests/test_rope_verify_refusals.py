"""Rotary positions and draft verification, host side: calls whose sizes or addresses no kernel may be given (no GPU needed)."""
import pytest

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
