"""Preference losses of infinite margins: a masked token's log-probability is -inf, and so is its sequence's sum."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


def run(hl, length, worse, **kw):
    """Two pairs of ordinary tokens; sequence `worse` of the first one has a token of log-probability -inf."""
    logp = torch.zeros(4, length)
    logp[2] = 0.25 / length
    logp[worse, length // 2] = -math.inf
    out = dict(dlogp=torch.empty(4, length, device="cuda"), rewards=torch.empty(4, device="cuda"),
               pair_loss=torch.empty(2, device="cuda"), stats=torch.empty(6, device="cuda"))
    hl.hilore_preference_loss(hl.preference_loss_desc(logp.cuda(), beta=0.5, **out, **kw))
    return {k: v.cpu().double() for k, v in out.items()}


# 4 x 10 tokens by one workgroup, 4 x 3000 by launches
@pytest.mark.parametrize("length", [10, 3000])
@pytest.mark.parametrize("lists", [False, True])
def test_logistic_of_an_infinite_margin(hl, length, lists):
    pairs = {}
    if lists:
        pairs = {k: torch.tensor(v, dtype=torch.int32, device="cuda") for k, v in (("chosen", [0, 2]), ("rejected", [1, 3]))}
    # the second pair: beta h = 0.125, sums in fp64 of fp32 tokens that are 0.25 / length within 2^-24; loss and slope
    # are within as much, and each output has one rounding: 2^-22 of the value
    loss, slope = math.log1p(math.exp(-0.125)), -0.5 / (1.0 + math.exp(0.125)) / 2.0
    for worse, first, first_slope in ((1, 0.0, 0.0), (0, math.inf, -0.25)):
        got = run(hl, length, worse, **pairs)
        assert float(got["pair_loss"][0]) == first and float(got["pair_loss"][1]) == pytest.approx(loss, rel=2.0 ** -22)
        assert float(got["rewards"][worse]) == -math.inf
        assert bool((got["dlogp"][0] == first_slope).all()) and bool((got["dlogp"][1] == -first_slope).all())
        assert torch.allclose(got["dlogp"][2], torch.full((length,), slope, dtype=torch.float64), rtol=2.0 ** -22, atol=0)
        assert float(got["stats"][0]) == (math.inf if first else pytest.approx(loss / 2.0, rel=2.0 ** -22))
        assert float(got["stats"][1]) == (0.5 if first else 1.0) and float(got["stats"][5]) == 2.0


@pytest.mark.parametrize("worse", [0, 1])
def test_smoothed_logistic_of_an_infinite_margin(hl, worse):
    """Both terms have a weight: the loss is infinite on either side."""
    assert float(run(hl, 10, worse, label_smoothing=0.1)["pair_loss"][0]) == math.inf


def test_a_margin_that_is_no_number_stays(hl):
    logp, ref = torch.zeros(2, 10), torch.zeros(2, 10)
    logp[1, 3] = ref[1, 3] = -math.inf
    loss, d = torch.empty(1, device="cuda"), torch.empty(2, 10, device="cuda")
    hl.hilore_preference_loss(hl.preference_loss_desc(logp.cuda(), ref.cuda(), pair_loss=loss, dlogp=d))
    assert math.isnan(float(loss)) and bool(torch.isnan(d).all())
