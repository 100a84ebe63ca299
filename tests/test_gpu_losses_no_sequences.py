"""Tokens without a sequence: offsets of one element.  What lies behind it is no offset, and no output of a token is written."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


def offsets(first, behind):
    """One offset, a slice of a longer tensor."""
    return torch.tensor([first, behind, behind, behind], device="cuda")[:1]


# 24 tokens, below the one-workgroup sizes; 9001, above them
@pytest.mark.parametrize("n", [24, 9001])
@pytest.mark.parametrize("first", [0, 5])
@pytest.mark.parametrize("lists", [None, [], [-1], [0], [-1, 3]])
@pytest.mark.parametrize("norm", [0.0, 4.0])
def test_preference(hl, n, first, lists, norm):
    logp, d = torch.randn(n, device="cuda"), torch.full((n,), 9.0, device="cuda")
    stats = torch.full((6,), 2.0, device="cuda")
    pairs = {}
    if lists is not None:
        number = torch.tensor(lists, dtype=torch.int32, device="cuda")
        pairs = dict(chosen=number, rejected=number.clone(), pair_loss=torch.full((len(lists),), 2.0, device="cuda"))
    hl.hilore_preference_loss(hl.preference_loss_desc(logp, offsets=offsets(first, n - 2), dlogp=d, stats=stats, n_norm=norm, **pairs))
    assert bool((d == 9.0).all())
    # a number past the sequences (all are) makes its pair's loss and the statistics NaN; a negative one takes no part
    past = [v >= 0 for v in lists or []]
    assert torch.isnan(stats).tolist() == [any(past)] * 6 and (any(past) or not stats.any())
    if lists:
        assert [math.isnan(v) for v in pairs["pair_loss"].tolist()] == past


@pytest.mark.parametrize("n", [24, 9001])
@pytest.mark.parametrize("mean", ["tokens", "sequences"])
def test_policy(hl, n, mean):
    logp, adv = torch.randn(n, device="cuda"), torch.ones(n, device="cuda")
    out = {k: torch.full((n,), 9.0, device="cuda") for k in ("dlogp", "token_loss")}
    flags, stats = torch.full((n,), 9, dtype=torch.uint8, device="cuda"), torch.full((8,), 2.0, device="cuda")
    hl.hilore_policy_loss(hl.policy_loss_desc(logp, logp, adv, offsets=offsets(0, n - 2), mean=mean, flags=flags, stats=stats, **out))
    assert bool((flags == 9).all()) and all(bool((v == 9.0).all()) for v in out.values()) and not stats.any()


def test_policy_without_advantages(hl):
    logp, d, stats = torch.randn(24, device="cuda"), torch.full((24,), 9.0, device="cuda"), torch.full((8,), 2.0, device="cuda")
    hl.hilore_policy_loss(hl.policy_loss_desc(logp, logp, torch.empty(0, device="cuda"), offsets=offsets(3, 20), dlogp=d, stats=stats))
    assert bool((d == 9.0).all()) and not stats.any()
