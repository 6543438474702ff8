"""Draft verification by clusters of every size: the CTAs of a request exchange their sums through one another's shared memory."""
import pytest
import torch

from tests.test_rope_verify_gpu import DEV, B, check_verify, make, no_timeout  # noqa: F401

pytestmark = pytest.mark.gpu

# CTAs of a request, one more for vocabularies just above 1024, 2048, 4096 and 8192 tokens (as long as the batch leaves room)
SIZES = [(1, 1024), (2, 1025), (4, 2049), (8, 4097), (16, 8193)]


@pytest.mark.parametrize("ctas,V", SIZES)
def test_the_shortest_way_to_the_exchange(B, ctas, V):
    # no draft to look at and hardly a token a warp: the sums are exchanged as early as they can be.  Launches one behind the other, so that CTAs
    # of a cluster start while others of the device are still busy; every one has to find the same token.
    target, _, tokens, ua, us = make(3, 0, V, ctas, torch.bfloat16)
    check_verify(B, target, None, tokens, ua, us)
    first = B.verify_drafts(target, None, tokens, ua, us)
    accepted, out = (torch.full((300,) + x.shape, -7, dtype=torch.int32, device=DEV) for x in first[:2])
    for i in range(300):
        B.verify_drafts(target, None, tokens, ua, us, accepted=accepted[i], out=out[i])
    torch.cuda.synchronize()
    assert torch.equal(accepted, first[0].expand_as(accepted)) and torch.equal(out, first[1].expand_as(out))


@pytest.mark.parametrize("nb,n,V", [(100, 3, 2049), (185, 1, 4000), (93, 2, 30011), (64, 4, 128000), (5, 3, 3001), (370, 1, 2600), (371, 1, 2600)])
def test_requests_for_every_number_of_ctas(B, nb, n, V):
    # four CTAs for up to 185 requests, two for up to 370, then one
    for dtype in (torch.float32, torch.bfloat16):
        target, q, tokens, ua, us = make(nb, n, V, nb + V, dtype)
        check_verify(B, target, q, tokens, ua, us, n_tok=torch.arange(50, 50 + nb, dtype=torch.int32, device=DEV))
        check_verify(B, target, None, tokens, ua, us)
