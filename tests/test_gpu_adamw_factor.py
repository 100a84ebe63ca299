"""hilore_adamw with a factor of the caller's in norm[1]: g = grad * norm[1] for every value that is
not NaN, and those above 1 among them (a trainer that scales its loss down scales gradients back up).

A power of two is exact, so the step has to be that of the gradients scaled beforehand, bit for bit.
"""
import pytest
import torch

from paper_2609_33570_amd import workloads as wl

pytestmark = pytest.mark.gpu


def state(eight):
    g, n = wl.rng(31, eight), 5000

    def rand(size, sigma):
        return torch.from_numpy(g.standard_normal(size).astype("float32") * sigma).cuda()

    t = dict(grad=rand(n, 1e-3), p=rand(n, 1.0))
    if eight:
        t["m"], t["v"] = (torch.from_numpy(g.integers(1, 100, n).astype("uint8")).cuda() for _ in range(2))
        t["m_scales"], t["v_scales"] = rand(-(-n // 256), 1e-4).abs(), rand(-(-n // 256), 1e-4).abs()
    else:
        t["m"], t["v"] = rand(n, 1e-3), rand(n, 1e-3).square()
    return t


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("factor", [0.0, 0.25, 1.0, 2.0, 1024.0, -2.0])
def test_factor(hl, factor, eight):
    scaled, given = state(eight), state(eight)
    start = given["p"].clone()
    scaled["grad"] *= factor
    norm = torch.tensor([1.0, factor], device="cuda")
    for t, n in ((scaled, None), (given, norm)):
        hl.hilore_adamw([hl.adamw_tensor(lr=1e-2, weight_decay=0.1, **t)], 0.9, 0.999, 1e-8, 2, norm=n, seed=5)
    for k, v in scaled.items():
        assert k == "grad" or torch.equal(v, given[k]), k
    assert not torch.equal(given["p"], start)


@pytest.mark.parametrize("eight", [False, True])
def test_nan_skips(hl, eight):
    t, before = state(eight), state(eight)
    norm = torch.tensor([1.0, float("nan")], device="cuda")
    hl.hilore_adamw([hl.adamw_tensor(lr=1e-2, **t)], 0.9, 0.999, 1e-8, 2, norm=norm)
    for k, v in t.items():
        assert torch.equal(v, before[k]), k
