"""The 64-bit implementations that the operators are tested against, pinned by torch's autograd,
by differences and by closed forms."""
import math

import pytest
import torch

import actor_reference as R

torch.manual_seed(0)


@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("norm", [False, True])
def test_heads_backward_is_autograd(pairs, norm):
    x = torch.randn(5, 3, 32, dtype=torch.float64, requires_grad=True)
    w = torch.randn(32, dtype=torch.float64, requires_grad=True) if norm else None
    pos, freq = torch.tensor([0, 7, 100000, -1, 3]), (100.0 ** -torch.rand(8)).float()
    g = torch.randn(5, 3, 32, dtype=torch.float64)
    out = R.heads_forward(x, w, 1e-6, pos, freq, pairs, 1.5)
    out.backward(g)
    dx, dw, _, _ = R.heads_backward(x.detach(), None if w is None else w.detach(), 1e-6, pos, freq, pairs, g, 1.5)
    assert torch.allclose(dx, x.grad, rtol=1e-12, atol=1e-13)
    if norm:
        assert torch.allclose(dw, w.grad, rtol=1e-12, atol=1e-13)


def test_rotation_keeps_lengths_and_relative_angles():
    x, y = torch.randn(1, 1, 16, dtype=torch.float64), torch.randn(1, 1, 16, dtype=torch.float64)
    freq = torch.tensor([1.0, 0.5, 0.25, 0.01, 0.3, 0.2, 0.1, 0.05])

    def at(v, p):
        return R.heads_forward(v, None, 0.0, torch.tensor([p]), freq, False)

    assert torch.allclose(at(x, 91).norm(), x.norm())
    assert torch.allclose((at(x, 5) * at(y, 9)).sum(), (at(x, 1005) * at(y, 1009)).sum())  # the distance alone counts
    assert torch.equal(at(x, 0), x)


def test_logprobs_are_torchs():
    z = 3.0 * torch.randn(6, 50, dtype=torch.float64)
    z[2, 10:] = -math.inf
    t = torch.tensor([0, 49, 3, -1, 7, 7])
    z[5, 7] = 60.0
    o = R.token_logprobs(z, t, 0.7)
    want = torch.log_softmax(0.7 * z, 1)
    live = t >= 0
    # torch subtracts a log sum of up to 42 from a logit of as much: half a step of 42 is 2^-48
    assert torch.allclose(o["logp"][live], want.gather(1, t.clamp(min=0)[:, None])[:, 0][live], rtol=1e-12, atol=2.0 ** -46)
    assert torch.allclose(0.7 * o["row_max"][live] + o["log_sum"][live], torch.logsumexp(0.7 * z, 1)[live])
    p = want.exp()
    assert torch.allclose(o["entropy"][live], -(p * want.clamp(min=-1e9)).sum(1)[live])
    assert all(float(v[3]) == 0.0 for v in o.values())
    assert 0 < -float(o["logp"][5]) < 1e-15  # not rounded away


@pytest.mark.parametrize("bonus", [False, True])
def test_logprobs_backward_is_autograd(bonus):
    z = (2.0 * torch.randn(5, 30, dtype=torch.float64)).requires_grad_()
    t, scale = torch.tensor([1, 29, -1, 4, 5]), 1.3
    g, e = torch.randn(5, dtype=torch.float64), torch.randn(5, dtype=torch.float64)
    g[3] = 0.0
    e[3] = 0.0
    o = R.token_logprobs(z, t, scale)
    (o["logp"] * g + (o["entropy"] * e if bonus else 0.0)).sum().backward()
    with torch.no_grad():
        d = R.token_logprobs_bwd(z, t, scale, o["row_max"], o["log_sum"], o["entropy"], g, e if bonus else None)
    assert torch.allclose(d, z.grad, rtol=1e-11, atol=1e-14)


def tokens(n, seed):
    g = torch.Generator().manual_seed(seed)
    old = -torch.rand(n, generator=g) * 3
    return old, old + 0.2 * torch.randn(n, generator=g), old + 0.1 * torch.randn(n, generator=g), torch.rand(n, generator=g)


@pytest.mark.parametrize("ratio", ["token", "sequence"])
@pytest.mark.parametrize("kl", [0, 1, 2, 3])
@pytest.mark.parametrize("mean", ["tokens", "sequences"])
def test_policy_gradient_is_the_difference_quotient(ratio, kl, mean):
    old, new, ref, ent = tokens(12, 5)
    # steps of 2^-10 that fp32 holds exactly, far from the thresholds
    old, new, ref = ((v * 1024).round() / 1024 for v in (old, new, ref))
    mask, adv = torch.tensor([1, 1, 0, 1, 1, 1, 1, 0, 0, 0, 0, 1]), torch.tensor([1.5, -0.7, 0.0, 2.0])
    kw = dict(adv=adv, sequences=4, logp_ref=ref if kl else None, entropy=ent, mask=mask, clip_high=0.28, dual_clip=3.0,
              beta=0.5, entropy_weight=0.25, kl=kl, ratio=ratio, mean=mean)
    o = R.policy_loss(new, old, **kw)
    h = 2.0 ** -10
    for t in range(12):
        up, down = new.clone(), new.clone()
        up[t] += h
        down[t] -= h
        a, b = R.policy_loss(up, old, **kw), R.policy_loss(down, old, **kw)
        if a["flags"] != b["flags"]:
            continue
        assert (a["stats"][0] - b["stats"][0]) / (2 * h) == pytest.approx(o["dlogp"][t], rel=1e-4, abs=2e-6)
    assert sum(o["token_loss"]) == pytest.approx(o["stats"][0])
    assert o["stats"][6:] == [7, 4]


def test_policy_closed_forms():
    old = torch.full((4,), -1.0)
    new = old + torch.tensor([0.0, 0.5, -0.5, 2.0])
    o = R.policy_loss(new, old, torch.tensor([2.0]), 1)
    assert o["token_loss"] == pytest.approx([-0.5, -0.6, -0.5 * math.exp(-0.5), -0.6], rel=1e-6)
    assert o["flags"] == [1, 2, 1, 2] and o["dlogp"][1] == o["dlogp"][3] == 0.0
    o = R.policy_loss(new, old, torch.tensor([-2.0]), 1, dual_clip=3.0)
    assert o["token_loss"] == pytest.approx([0.5, 0.5 * math.exp(0.5), 0.4, 1.5], rel=1e-6)
    assert o["flags"] == [1, 1, 2, 2]
    assert R.policy_loss(new, old, torch.tensor([0.0]), 1)["stats"][0] == 0.0
    assert R.policy_loss(new, old, torch.tensor([1.0]), 1, mask=torch.zeros(4))["stats"] == [0.0] * 8


@pytest.mark.parametrize("loss,eps", [("logistic", 0.0), ("logistic", 0.2), ("hinge", 0.0), ("squared", 0.0)])
@pytest.mark.parametrize("length_mean", [False, True])
def test_preference_gradient_is_the_difference_quotient(loss, eps, length_mean):
    ref, new, _, _ = tokens(15, 9)
    ref, new = ((v * 1024).round() / 1024 for v in (ref, new))
    mask = torch.tensor([1] * 9 + [0, 1, 1, 0, 0, 0])
    kw = dict(sequences=5, logp_ref=ref, mask=mask, chosen=torch.tensor([0, 0, 2, -1, 3]), rejected=torch.tensor([1, 2, 1, 1, 4]),
              beta=0.5, label_smoothing=eps, margin=0.125, loss=loss, length_mean=length_mean)
    o = R.preference_loss(new, **kw)
    assert o["stats"][5] == 3.0 and o["pair_loss"][3:] == [0.0, 0.0]  # a negative number; an empty sequence
    h = 2.0 ** -10
    for t in range(15):
        up, down = new.clone(), new.clone()
        up[t] += h
        down[t] -= h
        a, b = (R.preference_loss(v, **kw)["stats"][0] for v in (up, down))
        assert (a - b) / (2 * h) == pytest.approx(o["dlogp"][t], rel=1e-5, abs=1e-8)


def test_preference_closed_forms():
    z = torch.zeros(4)
    assert R.preference_loss(z, 2, beta=0.3)["stats"][0] == pytest.approx(math.log(2.0))
    assert R.preference_loss(z, 2, beta=0.25, loss="hinge")["stats"][0] == 1.0
    assert R.preference_loss(z, 2, beta=0.25, loss="squared")["stats"][0] == 4.0
    assert R.preference_loss(z, 2, mask=z)["stats"] == [0.0] * 6
