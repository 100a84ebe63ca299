"""The KL terms of the policy loss: K3 near its zero, and terms of weight 0.

Tolerance of K3 = exp(-x) - 1 + x, relative to its value.  Below |x| = 1 a series of positive or falling terms: a Horner
scheme whose last steps round twice, x * x and the product once each, and 2^-27 cut off: under 6 steps of 2^-24.  From 1
on expm1 within 1 step of at most 2^-22 where the value is 0.9 (x = -1.0986), 2^-23 where it is 0.72 (x = -1), 2^-24 where it is
0.37 (x = 1), and the sum's rounding: under 2^-21.6.  So 2^-21 throughout.  A token's loss is beta * kl, rounded, times a
weight, rounded, rounded again: 3 steps of 2^-24 more, under 2^-20.  stats[2] adds the tokens, all of one sign, times the
weight in fp32 over at most 256 tokens (10 roundings, and one at the end): 2^-21 + 12 * 2^-24, under 2^-19.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


def k3(x):
    """exp(-x) - 1 + x of fp32 values in 64 bits: the series below 1/16, where the sum would cancel."""
    x = x.double()
    series = torch.zeros_like(x)
    for k in range(14, -1, -1):  # (-x)^k / (k + 2)!
        series = series * -x + 1.0 / math.factorial(k + 2)
    return torch.where(x.abs() < 0.0625, x * x * series, torch.expm1(-x) + x)


def run(hl, logp, ref, old, adv, beta, kl=3, entropy=None, weight=0.0):
    n = logp.numel()
    out = {k: torch.empty(n, device="cuda") for k in ("dlogp", "token_loss")}
    if entropy is not None:
        out["dentropy"] = torch.empty(n, device="cuda")
    out["stats"] = torch.empty(8, device="cuda")
    hl.hilore_policy_loss(hl.policy_loss_desc(logp.cuda(), old.cuda(), adv.cuda(), logp_ref=None if ref is None else ref.cuda(),
                                              entropy=None if entropy is None else entropy.cuda(), sequences=adv.numel(), kl=kl,
                                              beta=beta, entropy_weight=weight, **out))
    return {k: v.cpu() for k, v in out.items()}


# 1200 tokens by one workgroup, 6000 by launches
@pytest.mark.parametrize("n", [1200, 6000])
@pytest.mark.parametrize("size", [1e-6, 1e-5, 1e-4, 1e-3, 1e-2, 0.1, 0.9, 1.1, 4.0, 30.0])
def test_k3_relative_to_its_value(hl, n, size):
    g = torch.Generator().manual_seed(51)
    x = size * (0.5 + torch.rand(n, generator=g)) * torch.where(torch.rand(n, generator=g) < 0.5, -1.0, 1.0)
    # the difference to a reference of 0 is the value itself
    got = run(hl, x, torch.zeros(n), x, torch.zeros(3), 0.25)
    want = k3(x)
    assert ((got["token_loss"].double() - 0.25 * want / n).abs() <= 2.0 ** -20 * (0.25 * want / n)).all()
    assert abs(float(got["stats"][2]) - float(want.mean())) <= 2.0 ** -19 * float(want.mean())


def test_k3_of_equal_policies(hl):
    logp = -torch.rand(100, generator=torch.Generator().manual_seed(1))
    got = run(hl, logp, logp, logp, torch.zeros(1), 0.25)
    assert not got["token_loss"].any() and not got["dlogp"].any() and float(got["stats"][2]) == 0.0


# 1200 tokens by one workgroup, 6000 by launches
@pytest.mark.parametrize("n", [1200, 6000])
@pytest.mark.parametrize("kl", [1, 2, 3])
def test_terms_of_weight_0_add_nothing(hl, n, kl):
    """A KL and an entropy that are only watched: infinite ones stay in their statistics."""
    g = torch.Generator().manual_seed(52)
    old = -torch.rand(n, generator=g)
    logp, ref, adv = old + 0.1 * torch.randn(n, generator=g), old.clone(), torch.randn(3, generator=g)
    entropy = torch.rand(n, generator=g)
    logp[7] = ref[7] - 95.0       # exp(95) is past fp32
    ref[n // 2], ref[n - 1] = -math.inf, math.inf
    entropy[11] = math.inf
    got = run(hl, logp, ref, old, adv, 0.0, kl, entropy)
    want = run(hl, logp, None, old, adv, 0.0, 0)
    for k in ("dlogp", "token_loss"):
        assert torch.equal(got[k], want[k]) and bool(torch.isfinite(got[k]).all()), k
    assert not got["dentropy"].any()
    assert torch.equal(got["stats"][[0, 1, 4, 5, 6, 7]], want["stats"][[0, 1, 4, 5, 6, 7]])
    assert not math.isfinite(float(got["stats"][2])) and float(got["stats"][3]) == math.inf
