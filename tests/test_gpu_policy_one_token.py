"""Packed sequences of one token each: an advantage a sequence is one a token, unless a capture keeps the offsets from view."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_one_token_each(hl):
    g = torch.Generator(device="cuda").manual_seed(1)
    logp, old, adv = (torch.randn(50, generator=g, device="cuda") for _ in range(3))
    offsets = torch.arange(51, device="cuda")
    d = [torch.empty(50, device="cuda") for _ in range(3)]
    for out, said in zip(d, (None, False, True)):
        hl.hilore_policy_loss(hl.policy_loss_desc(logp, old, adv, offsets=offsets, dlogp=out, adv_per_token=said))
    assert torch.equal(d[0], d[1]) and torch.equal(d[0], d[2])
    offsets[7] = 6  # the seventh is empty, the eighth has two tokens
    with pytest.raises(ValueError, match="adv_per_token"):
        hl.policy_loss_desc(logp, old, adv, offsets=offsets)


def test_under_capture(hl):
    """Made inside a captured call the descriptor has to be told."""
    logp, old, adv = (torch.randn(50, device="cuda") for _ in range(3))
    offsets, out = torch.arange(51, device="cuda"), torch.zeros(50, device="cuda")
    want = torch.zeros(50, device="cuda")
    hl.hilore_policy_loss(hl.policy_loss_desc(logp, old, adv, offsets=offsets, dlogp=want, adv_per_token=True))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        with pytest.raises(ValueError, match="adv_per_token"):
            hl.policy_loss_desc(logp, old, adv, offsets=offsets, dlogp=out)
        desc = hl.policy_loss_desc(logp, old, adv, offsets=offsets, dlogp=out, adv_per_token=True)
        hl.hilore_policy_loss(desc)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
