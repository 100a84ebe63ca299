"""hilore_adamw and hilore_grad_norm over hundreds of tensors of every kind: each has to come out
bit for bit as in a call of its own, whatever travels with it in a launch.

The random bits of a tensor go by its number in the call, so the call of its own has as many
tensors without elements before it.
"""
import pytest
import torch

from paper_2609_33570_amd import workloads as wl

pytestmark = pytest.mark.gpu
STEP = dict(beta1=0.9, beta2=0.95, eps=1e-8, step=3, seed=1234)


def tensor(g, n, kind):
    """Tensors of one entry, by kind: parameter (f32, bf16, both), gradient type, state type."""
    param, grad16, eight = kind
    blocks = -(-n // 256)

    def rand(size, sigma):
        return torch.from_numpy(g.standard_normal(size).astype("float32") * sigma).cuda()

    t = dict(grad=rand(n, 1e-2).bfloat16() if grad16 else rand(n, 1e-2))
    if param != 1:
        t["p"] = rand(n, 1.0)
    if param != 0:
        t["p16"] = rand(n, 1.0).bfloat16()
    if eight:
        t["m"], t["v"] = (torch.from_numpy(g.integers(1, 100, n).astype("uint8")).cuda() for _ in range(2))
        t["m_scales"], t["v_scales"] = rand(blocks, 1e-4).abs(), rand(blocks, 1e-4).abs()
    else:
        t["m"], t["v"] = rand(n, 1e-3), rand(n, 1e-3).square()
    return t


def copy(t):
    return {k: v.clone() for k, v in t.items()}


def empty(kind):
    return tensor(wl.rng(0, 0), 0, kind)


KINDS = [(p, g16, e) for p in (0, 1, 2) for g16 in (False, True) for e in (False, True)]


@pytest.mark.parametrize("kinds", [KINDS, [k for k in KINDS if not k[2]], [(0, False, False)], [(1, True, True)]],
                         ids=["all", "f32_states", "plain", "bf16_8bit"])
def test_each_as_alone(hl, kinds):
    g = wl.rng(11, len(kinds))
    sizes = [0 if i % 29 == 5 else int(g.integers(1, 700)) if i % 7 else int(g.integers(4000, 9000)) for i in range(310)]
    sizes[0], sizes[-1] = 0, 0  # an empty one first and last
    lrs = [1e-3 * (1 + i % 23) for i in range(len(sizes))]
    start = [tensor(g, n, kinds[i % len(kinds)]) for i, n in enumerate(sizes)]
    norm = torch.tensor([3.0, 0.5], device="cuda")

    def desc(t, i):
        return hl.adamw_tensor(lr=lrs[i], weight_decay=0.01 * (i % 5), **t)

    together = [copy(t) for t in start]
    hl.hilore_adamw(hl.adamw_tensors([desc(t, i) for i, t in enumerate(together)]), norm=norm, **STEP)
    for i in range(len(sizes)):
        alone = copy(start[i])
        before = desc(empty(kinds[0]), 0)
        hl.hilore_adamw(hl.adamw_tensors([before] * i + [desc(alone, i)]), norm=norm, **STEP)
        for k, v in alone.items():
            assert torch.equal(v, together[i][k]), (i, sizes[i], k)
            if sizes[i] and k == "p":
                assert not torch.equal(v, start[i][k]), (i, k)


@pytest.mark.parametrize("count", [1, 287, 288, 289, 600])
def test_norm_of_many(hl, count):
    """Sums are fp64: the norm is within one rounding to fp32, 2^-24, and the root's, 2^-24."""
    g = wl.rng(12, count)
    sizes = [0 if i % 31 == 3 else int(g.integers(1, 3000)) if i % 40 else int(g.integers(30000, 50000)) for i in range(count)]
    tensors = [tensor(g, n, (0, i % 3 == 0, False)) for i, n in enumerate(sizes)]
    norm = torch.zeros(2, device="cuda")
    hl.hilore_grad_norm(hl.adamw_tensors([hl.adamw_tensor(**t) for t in tensors]), 0.25, norm)
    want = float(sum(t["grad"].double().square().sum() for t in tensors)) ** 0.5
    got = norm.double().cpu()
    assert abs(float(got[0]) - want) <= 2.0 ** -23 * want
    assert abs(float(got[1]) - min(1.0, 0.25 / (want + 1e-6))) <= 2.0 ** -22
