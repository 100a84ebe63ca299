"""hilore_policy_loss and hilore_preference_loss against 64 bits.

Tolerances.  Log ratios and differences are fp32 differences in both.  exp and expm1 are
within 2 steps, and a token's value has at most 12 further fp32 roundings of terms whose sizes the
reference adds up: 2^-20 of that sum.  Sums over tokens are in 64 bits, rounded once: the
same 2^-20 of the sizes' sum and 2^-23 of the value.  A sequence's mean log ratio is an fp32 rounding of a 64-bit
mean on both sides; where the last bits of the two sums differ it can fall on the other side, one
step of at most 1: 2^-23 of a ratio, inside the 2^-20.  The preference loss is in 64 bits throughout but for the
token differences: outputs are off by their one rounding, 2^-24, and exp's and log1p's last bits.
"""
import math

import pytest
import torch

import actor_reference as R

pytestmark = pytest.mark.gpu


def batch(n, seed, sigma=0.3):
    g = torch.Generator().manual_seed(seed)
    old = -3.0 * torch.rand(n, generator=g)
    new = old + sigma * torch.randn(n, generator=g)
    ref = old + 0.2 * torch.randn(n, generator=g)
    return g, new, old, ref, 2.0 * torch.rand(n, generator=g)


def layout(kind, g):
    """(n, sequences, offsets, mask): rows of one length or packed, empty ones among them."""
    if kind == "rows":
        n, s, offsets = 33 * 7, 33, None
    elif kind == "one":
        n, s, offsets = 1, 1, None
    elif kind == "long":
        n, s, offsets = 3 * 5000, 3, None
    elif kind == "many":
        n, s, offsets = 2500 * 2, 2500, None
    else:  # packed; the first tokens and the last ones are in no sequence
        lengths = [0, 5, 1, 0, 0, 700, 64, 3, 257, 0, 1023, 2]
        offsets = torch.tensor([11] + [11 + sum(lengths[:i + 1]) for i in range(len(lengths))])
        n, s = int(offsets[-1]) + 300, len(lengths)
    mask = (torch.rand(n, generator=g) < 0.7).to(torch.uint8) * 3
    if kind == "rows":
        mask[7:21] = 0  # two sequences without a valid token
    return n, s, offsets, mask


def on(t):
    return None if t is None else t.cuda()


def inside(n, offsets):
    t = torch.zeros(n, dtype=torch.bool)
    t[slice(None) if offsets is None else slice(int(offsets[0]), int(offsets[-1]))] = True
    return t


def run_policy(hl, n, s, offsets, mask, new, old, adv, ref=None, ent=None, dent=True, **kw):
    out = {k: torch.full((n,), 9.0, device="cuda") for k in ("dlogp", "dentropy", "token_loss")}
    out["flags"] = torch.full((n,), 9, dtype=torch.uint8, device="cuda")
    out["stats"] = torch.empty(8, device="cuda")
    if ent is None:
        del out["dentropy"]
    hl.hilore_policy_loss(hl.policy_loss_desc(on(new), on(old), on(adv), logp_ref=on(ref), entropy=on(ent), mask=on(mask),
                                              offsets=on(offsets), sequences=s, **out, **kw))
    return {k: v.cpu() for k, v in out.items()}


def check_policy(got, want, n, offsets):
    live = inside(n, offsets)
    size = torch.tensor([0.0 if v is None else v for v in want["size"]], dtype=torch.float64)
    for k in got:
        if k == "stats":
            continue
        assert bool((got[k][~live] == 9).all()), k  # tokens of no sequence are left as they were
        w = torch.tensor([0.0 if v is None else v for v in want[k]], dtype=torch.float64)
        if k == "flags":
            assert torch.equal(got[k][live].long(), w[live].long())
        else:
            off = (got[k].double() - w).abs()[live]
            limit = (2.0 ** -20 * size + 2.0 ** -22 * w.abs() + 1e-38)[live]
            assert (off <= limit).all(), (k, float((off / limit).max()), int((off / limit).argmax()))
    total = float(size.sum())
    for i, (a, b) in enumerate(zip(got["stats"].tolist(), want["stats"])):
        assert abs(a - b) <= 2.0 ** -20 * (total if i < 4 else abs(b)) + 2.0 ** -23 * abs(b) + (2.0 ** -20 * max(1.0, abs(b)) if i == 3 else 0.0), (i, a, b)


@pytest.mark.parametrize("kind", ["rows", "one", "long", "many", "packed"])
@pytest.mark.parametrize("ratio,mean", [("token", "tokens"), ("token", "sequences"), ("sequence", "tokens"), ("sequence", "sequences")])
@pytest.mark.parametrize("kl,dual,bonus,norm", [(0, 0.0, 0.0, 0.0), (1, 3.0, 0.0, 0.0), (2, 0.0, 0.01, 777.0), (3, 1.5, 0.01, 0.0)])
def test_policy(hl, kind, ratio, mean, kl, dual, bonus, norm):
    g = torch.Generator().manual_seed(17)
    n, s, offsets, mask = layout(kind, g)
    _, new, old, ref, ent = batch(n, 18)
    adv = torch.randn(s, generator=g)
    adv[torch.rand(s, generator=g) < 0.2] = 0.0
    if kind == "rows":
        adv[0] = 0.0
    bad = mask == 0
    for t, v in ((new, math.nan), (old, math.inf), (ref, -math.inf), (ent, math.nan)):
        t[bad] = v  # masked places hold anything
    kw = dict(clip_low=0.2, clip_high=0.28, dual_clip=dual, beta=0.04 if kl else 0.0, entropy_weight=bonus, kl=kl, ratio=ratio,
              mean=mean, n_norm=norm)
    got = run_policy(hl, n, s, offsets, mask, new, old, adv, ref if kl else None, ent if bonus else None, **kw)
    want = R.policy_loss(new, old, adv, s, ref if kl else None, ent if bonus else None, mask, offsets, **kw)
    check_policy(got, want, n, offsets)


@pytest.mark.parametrize("kind", ["rows", "packed"])
def test_policy_advantage_of_each_token(hl, kind):
    g = torch.Generator().manual_seed(3)
    n, s, offsets, mask = layout(kind, g)
    _, new, old, ref, ent = batch(n, 4)
    adv = torch.randn(n, generator=g)
    got = run_policy(hl, n, s, offsets, mask, new, old, adv, kl=0, mean="sequences")
    check_policy(got, R.policy_loss(new, old, adv, s, None, None, mask, offsets, mean="sequences"), n, offsets)


@pytest.mark.parametrize("n", [600, 30000])
@pytest.mark.parametrize("ratio", ["token", "sequence"])
def test_policy_hides_no_nan(hl, n, ratio):
    """A valid token whose ratio is NaN, a bound or not, and an advantage that is."""
    s = 6
    _, new, old, _, _ = batch(n, 30)
    adv = torch.tensor([1.0, -1.0, 0.0, math.nan, 0.5, -0.5])
    length = n // s
    new[3], old[length + 5] = math.nan, -math.inf
    new[length + 5] = -math.inf
    new[2 * length + 1] = math.nan  # no advantage: no policy term
    mask = torch.ones(n, dtype=torch.uint8)
    mask[4 * length + 2], new[4 * length + 2] = 0, math.nan
    got = run_policy(hl, n, s, None, mask, new, old, adv, ratio=ratio)
    bad = torch.zeros(n, dtype=torch.bool)
    bad[3 * length:4 * length] = True
    bad[3] = bad[length + 5] = True
    if ratio == "sequence":
        bad[:2 * length] = True
    for k in ("dlogp", "token_loss"):
        assert torch.equal(torch.isnan(got[k].cpu()), bad), k
    assert math.isnan(float(got["stats"][0])) and math.isnan(float(got["stats"][1]))


def test_policy_is_the_update_coefficient(hl):
    """With the symmetric clip, K3 and the tokens' mean, dlogp is what hilore_grpo_coeffs gives."""
    P, G, T = 3, 8, 40
    g, new, old, ref, _ = batch(P * G * T, 6)
    mask = (torch.rand(P * G * T, generator=g) < 0.8).to(torch.uint8)
    rewards = torch.randint(0, 2, (P * G,), generator=g).float()
    rewards[8:16] = 1.0  # a group of equal rewards: no advantage
    adv, coeff = torch.empty(P * G, device="cuda"), torch.empty(P * G * T, device="cuda")
    flags = torch.empty(P * G * T, dtype=torch.uint8, device="cuda")
    hl.hilore_grpo_coeffs(rewards.cuda(), new.cuda(), old.cuda(), ref.cuda(), mask.cuda(), P, G, T, 0.2, 1e-6, 1e-3, 0.0, adv, None,
                          flags, coeff)
    got = run_policy(hl, P * G * T, P * G, None, mask, new, old, adv.cpu(), ref, beta=1e-3, kl=3)
    size = torch.tensor(R.policy_loss(new, old, adv.cpu(), P * G, ref, None, mask, beta=1e-3, kl=3)["size"])
    assert ((got["dlogp"] - coeff.cpu()).abs() <= 2.0 ** -19 * size + 1e-30).all()
    assert torch.equal(got["flags"], flags.cpu())


def test_policy_edges(hl):
    """No valid token, no token, no output but the gradient; infinite ratios where they do not count."""
    n = 24
    _, new, old, _, _ = batch(n, 8)
    got = run_policy(hl, n, 4, None, torch.zeros(n, dtype=torch.uint8), new, old, torch.ones(4))
    assert not got["stats"].any() and not got["dlogp"].any() and not got["flags"].any()
    e = torch.empty(0, device="cuda")
    stats = torch.full((8,), 3.0, device="cuda")
    hl.hilore_policy_loss(hl.policy_loss_desc(e, e, e, sequences=0, stats=stats))
    assert not stats.any()
    hl.hilore_policy_loss(hl.policy_loss_desc(e, e, torch.ones(2, device="cuda"), stats=stats.fill_(1.0),
                                              offsets=torch.zeros(3, dtype=torch.int64, device="cuda")))
    assert not stats.any()
    whole = run_policy(hl, n, 4, None, None, new, old, torch.ones(4))
    alone = torch.empty(n, device="cuda")
    hl.hilore_policy_loss(hl.policy_loss_desc(new.cuda(), old.cuda(), torch.ones(4, device="cuda"), sequences=4, dlogp=alone))
    assert torch.equal(alone.cpu(), whole["dlogp"])
    new[0], old[0] = 0.0, -1000.0  # ratio infinite
    got = run_policy(hl, n, 4, None, None, new, old, torch.tensor([1.0, -1.0, 0.0, 1.0]))
    assert math.isfinite(float(got["stats"][0])) and float(got["dlogp"][0]) == 0.0
    got = run_policy(hl, n, 4, None, None, new, old, torch.tensor([0.0, 1.0, 1.0, 1.0]))
    assert float(got["token_loss"][0]) == 0.0 and float(got["dlogp"][0]) == 0.0
    got = run_policy(hl, n, 4, None, None, new, old, torch.tensor([-1.0, 1.0, 1.0, 1.0]), dual_clip=2.0)
    assert float(got["token_loss"][0]) == pytest.approx(2.0 / n) and float(got["dlogp"][0]) == 0.0


@pytest.mark.parametrize("offsets", [[5, 3, 900, -7, 12], [-4, 10, 1 << 50, 20, 24], [24, 24, 24, 24, 24], [0, 1 << 62, -(1 << 62), 3, 30]])
def test_offsets_out_of_range_read_nothing(hl, offsets):
    """Offsets that break the contract: nothing outside the tensors is read or written."""
    n = 24
    _, new, old, _, _ = batch(n, 8)
    guard = torch.full((3 * n,), 4.0, device="cuda")
    out = guard[n:2 * n]
    hl.hilore_policy_loss(hl.policy_loss_desc(new.cuda(), old.cuda(), torch.ones(4, device="cuda"), dlogp=out,
                                              offsets=torch.tensor(offsets, device="cuda"), ratio="sequence"))
    hl.hilore_preference_loss(hl.preference_loss_desc(new.cuda(), dlogp=out, offsets=torch.tensor(offsets, device="cuda")))
    assert bool((guard[:n] == 4.0).all()) and bool((guard[2 * n:] == 4.0).all())


# ------------------------------------------------------------- preference --
def pair_lists(s, g):
    """Pairs of random sequences: the same one in many, against itself, negative numbers among them."""
    c, r = torch.randint(0, s, (3 * s + 1,), generator=g), torch.randint(0, s, (3 * s + 1,), generator=g)
    c[::9], r[4::13] = -1, -5
    c[-1] = r[-1] = s - 1
    return c.to(torch.int32), r.to(torch.int32)


def check_preference(hl, n, s, offsets, mask, new, ref, chosen, rejected, **kw):
    pairs = s // 2 if chosen is None else chosen.numel()
    out = dict(dlogp=torch.full((n,), 9.0, device="cuda"), rewards=torch.empty(s, device="cuda"),
               pair_loss=torch.empty(pairs, device="cuda"), stats=torch.empty(6, device="cuda"))
    hl.hilore_preference_loss(hl.preference_loss_desc(on(new), on(ref), on(mask), on(offsets), s, on(chosen), on(rejected), **out, **kw))
    want = R.preference_loss(new, s, ref, mask, offsets, chosen, rejected, **kw)
    live = inside(n, offsets)
    assert bool((out["dlogp"].cpu()[~live] == 9.0).all())
    # sums of the same numbers in another order differ by n 2^-53 of their sizes: 1e-12 here
    for k in ("dlogp", "rewards", "pair_loss", "stats"):
        got = out[k].cpu().double()
        w = torch.tensor([0.0 if v is None else v for v in want[k]], dtype=torch.float64)
        if k == "dlogp":
            got, w = got[live], w[live]
        assert ((got - w).abs() <= 2.0 ** -23 * w.abs() + 1e-9).all(), (k, float((got - w).abs().max()))


@pytest.mark.parametrize("kind", ["rows", "one", "long", "many", "packed"])
@pytest.mark.parametrize("lists", [False, True])
@pytest.mark.parametrize("loss,eps,margin,length_mean,norm", [
    ("logistic", 0.0, 0.0, False, 0.0), ("logistic", 0.1, 0.25, True, 0.0), ("hinge", 0.0, 0.0, False, 50.0),
    ("squared", 0.0, 0.0, True, 0.0)])
def test_preference(hl, kind, lists, loss, eps, margin, length_mean, norm):
    g = torch.Generator().manual_seed(27)
    n, s, offsets, mask = layout(kind, g)
    _, new, _, ref, _ = batch(n, 28, 0.1)
    new[mask == 0], ref[mask == 0] = math.nan, math.inf
    chosen, rejected = pair_lists(s, g) if lists else (None, None)
    check_preference(hl, n, s, offsets, mask, new, ref, chosen, rejected, beta=0.25, loss=loss, label_smoothing=eps, margin=margin,
                     length_mean=length_mean, n_norm=norm)


def test_preference_without_reference_and_mask(hl):
    g = torch.Generator().manual_seed(2)
    _, new, _, _, _ = batch(40 * 9, 29)
    check_preference(hl, 360, 40, None, None, new, None, None, None, beta=0.1)
    c, r = pair_lists(40, g)
    check_preference(hl, 360, 40, None, None, new, None, c, r, beta=2.0)


def test_preference_of_wide_margins(hl):
    """Differences of thousands: no overflow, the loss linear on one side and 0 on the other."""
    new = torch.zeros(4, 1000)
    new[0], new[3] = -5.0, -5.0
    stats, loss, d = torch.empty(6, device="cuda"), torch.empty(2, device="cuda"), torch.empty(4, 1000, device="cuda")
    hl.hilore_preference_loss(hl.preference_loss_desc(new.cuda(), beta=1.0, dlogp=d, pair_loss=loss, stats=stats))
    assert loss.tolist() == [5000.0, 0.0] and stats.tolist() == [2500.0, 0.5, 0.0, -2500.0, -2500.0, 2.0]
    assert bool((d[0] == -0.5).all()) and bool((d[1] == 0.5).all()) and not d[2:].any()


def test_preference_edges(hl):
    new = torch.randn(4, 10)
    stats, d = torch.full((6,), 2.0, device="cuda"), torch.ones(4, 10, device="cuda")
    hl.hilore_preference_loss(hl.preference_loss_desc(new.cuda(), mask=torch.zeros(4, 10, dtype=torch.bool, device="cuda"), dlogp=d, stats=stats))
    assert not stats.any() and not d.any()
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    hl.hilore_preference_loss(hl.preference_loss_desc(new.cuda(), chosen=none, rejected=none, dlogp=d.fill_(1.0), stats=stats.fill_(1.0)))
    assert not stats.any() and not d.any()
    e = torch.empty(0, device="cuda")
    hl.hilore_preference_loss(hl.preference_loss_desc(e, sequences=0, dlogp=e, stats=stats.fill_(1.0)))
    assert not stats.any()
    # a number past the sequences
    for norm in (0.0, 3.0):
        c, r = (torch.tensor(v, dtype=torch.int32, device="cuda") for v in ([0, 4], [1, 2]))
        loss = torch.empty(2, device="cuda")
        hl.hilore_preference_loss(hl.preference_loss_desc(new.cuda(), chosen=c, rejected=r, dlogp=d, stats=stats, pair_loss=loss, n_norm=norm))
        assert torch.isnan(loss).tolist() == [False, True] and torch.isnan(stats).all() and torch.isnan(d).all()


def test_the_same_bits_again(hl):
    g = torch.Generator().manual_seed(5)
    n, s, offsets, mask = layout("packed", g)
    _, new, old, ref, ent = batch(n, 6)
    adv = torch.randn(s, generator=g)
    runs = [run_policy(hl, n, s, offsets, mask, new, old, adv, ref, ent, kl=3, beta=0.1, entropy_weight=0.1, ratio="sequence") for _ in range(3)]
    assert all(torch.equal(runs[0][k], r[k]) for r in runs[1:] for k in r)
