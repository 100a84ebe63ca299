"""The example's update against 64-bit autograd of the same model.

The step's roundings: bf16 storage (half a step, 2^-8 of a value, 0.2 % of a tensor's norm each) of
the projection's rows, the turned heads, the mixed rows, the logits, their gradient and what is made of
it.  A gradient gathers at most eight of these, independent: under 0.6 % of its norm, and the logits' rounding
moves each probability by up to 2^-8 of a logit of a few units, 1 %, which every gradient sees.
Three times their sum is allowed.
"""
import importlib.util
import os

import pytest
import torch

import actor_reference as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example(hl):
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "policy_update.py")
    spec = importlib.util.spec_from_file_location("policy_update", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def reference(actor, example, loss):
    """Gradients of the loss by autograd in 64 bits on the host, from the same bf16 weights."""
    p = {k: v.cpu().double().requires_grad_() for k, v in actor.p16.items()}
    n, d, H, K = actor.tokens, actor.dim, actor.heads, actor.key_heads
    ids, targets, mask = actor.ids.cpu(), actor.targets.cpu(), actor.mask.cpu()
    qkv = p["embedding"][ids] @ p["w_qkv"].t()
    q, k, v = (x.reshape(n, h, d) for x, h in zip(qkv.split([H * d, K * d, K * d], 1), (H, K, K)))
    pos, freq = actor.positions.cpu(), actor.inv_freq.cpu()
    q, k = (R.heads_forward(x, w, 1e-6, pos, freq, False) for x, w in ((q, p["w_q"]), (k, p["w_k"])))
    ends, out = actor.offsets.tolist(), []
    for a, b in zip(ends, ends[1:]):
        s = torch.einsum("ihd,jhd->hij", q[a:b], k[a:b].repeat_interleave(H // K, 1)) * d ** -0.5
        s = s.masked_fill(torch.ones(b - a, b - a, dtype=torch.bool).triu(1), float("-inf"))
        out.append(torch.einsum("hij,jhd->ihd", s.softmax(-1), v[a:b].repeat_interleave(H // K, 1)).reshape(b - a, -1))
    logits = torch.cat(out) @ p["w_out"].t()
    lp = torch.log_softmax(logits, 1)
    logp = lp.gather(1, targets.clamp(min=0)[:, None])[:, 0]
    entropy = -(lp.exp() * lp).sum(1)
    valid = mask != 0
    ref, old = actor.t["logp_ref"].cpu().double(), actor.t["logp_old"].cpu().double()
    if loss == "policy":
        adv = torch.cat([actor.adv[i].cpu().double().expand(b - a) for i, (a, b) in enumerate(zip(ends, ends[1:]))])
        r = (logp - old).exp()
        policy = -torch.minimum(r * adv, r.clamp(1 - example.CLIP_LOW, 1 + example.CLIP_HIGH) * adv)
        x = logp - ref
        each = policy + example.KL_BETA * ((-x).exp() - 1 + x) - example.BONUS * entropy
        value = each[valid].mean()
    else:
        sums = torch.stack([(logp - ref)[a:b][valid[a:b]].sum() for a, b in zip(ends, ends[1:])])
        value = torch.nn.functional.softplus(-example.PREFERENCE_BETA * (sums[0::2] - sums[1::2])).mean()
    value.backward()
    return float(value.detach()), logp.detach(), {k: v.grad for k, v in p.items()}


@pytest.mark.parametrize("loss", ["policy", "preference"])
@pytest.mark.parametrize("lengths,vocab", [((5, 2), 50), ((40, 23, 64, 31), 1000), ((3, 130, 17, 9, 70, 33), 4001)])
def test_gradients(example, loss, lengths, vocab):
    actor = example.Actor(lengths, vocab, seed=vocab)
    g = torch.Generator(device="cuda").manual_seed(3)
    for k in ("w_q", "w_k"):
        actor.p16[k].add_(0.2 * torch.randn(actor.dim, generator=g, device="cuda"))
    actor.set_batch(torch.randint(0, vocab, (actor.tokens,), generator=g, device="cuda"))
    actor.adv.copy_(torch.randn(len(lengths), generator=g, device="cuda"))
    logp = actor.forward().clone()
    # ratios of about exp(+-0.1): inside the clip, where a probability's rounding moves no flag
    actor.t["logp_old"].copy_(logp + 0.05 * torch.randn(actor.tokens, generator=g, device="cuda").clamp(-2, 2))
    actor.t["logp_ref"].copy_(logp + 0.1 * torch.randn(actor.tokens, generator=g, device="cuda"))
    value = float(actor.loss(loss))
    actor.backward()
    want, ref_logp, grads = reference(actor, example, loss)
    live = (actor.mask != 0).cpu()
    assert (logp.cpu().double() - ref_logp)[live].abs().max() < 0.05
    assert abs(value - want) < 0.05 * max(1.0, abs(want))
    off = {k: float((actor.grad[k].cpu().double() - grads[k]).norm() / grads[k].norm()) for k in actor.NAMES}
    assert max(off.values()) < 0.05, off


@pytest.mark.parametrize("loss", ["policy", "preference"])
def test_runs(example, loss):
    losses = example.train(loss, steps=6)
    assert all(torch.isfinite(torch.tensor(losses)))
    assert losses == example.train(loss, steps=6)  # the same bits again
