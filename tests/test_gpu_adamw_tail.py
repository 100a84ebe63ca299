"""hilore_adamw with 8-bit states: a value that is not finite stays in its own block of 256.

Without a norm a step is not skipped for a gradient that is not finite.  Its block is lost then,
and every other one, a tensor's last and partly filled block among them, has to come out bit
for bit as it does when that value is a finite one.  (A large one: blocks past 2^12 and those that
share their wave are scaled by other instructions, the same on both sides then.)
"""
import pytest
import torch

from paper_2609_33570_amd import workloads as wl

pytestmark = pytest.mark.gpu
NAN, INF = float("nan"), float("inf")


def state(n, param, grad16):
    g = wl.rng(n, 21)
    blocks = -(-n // 256)

    def rand(size, sigma):
        return torch.from_numpy(g.standard_normal(size).astype("float32") * sigma).cuda()

    t = dict(grad=rand(n, 1e-2).bfloat16() if grad16 else rand(n, 1e-2))
    if param != "bf16":
        t["p"] = rand(n, 1.0)
    if param != "f32":
        t["p16"] = rand(n, 1.0).bfloat16()
    t["m"], t["v"] = (torch.from_numpy(g.integers(1, 100, n).astype("uint8")).cuda() for _ in range(2))
    t["m_scales"], t["v_scales"] = rand(blocks, 1e-4).abs(), rand(blocks, 1e-4).abs()
    return t


@pytest.mark.parametrize("n", [257, 300, 511, 513, 4095, 4097, 4100, 8500, 70003])
@pytest.mark.parametrize("param,grad16", [("f32", False), ("bf16", True), ("master", False)])
@pytest.mark.parametrize("where", ["grad", "m_scales", "v_scales"])
@pytest.mark.parametrize("bad", [NAN, INF])
def test_other_blocks_are_untouched(hl, n, param, grad16, where, bad):
    outs = []
    for value in (1e6 if where == "grad" else 1e4, bad):
        t = state(n, param, grad16)
        t[where][0] = value
        arr = hl.adamw_tensors([hl.adamw_tensor(lr=1e-3, weight_decay=0.1, **t)])
        for step in (1, 2):  # the second step reads what the first one stored
            hl.hilore_adamw(arr, 0.9, 0.999, 1e-8, step, seed=step)
        torch.cuda.synchronize()
        outs.append(t)
    for k, v in outs[0].items():
        first = 1 if k.endswith("scales") else 256
        assert torch.equal(v[first:], outs[1][k][first:]), k
        assert torch.isfinite(v[first:].float()).all(), k
    assert not torch.isfinite(outs[1]["m_scales" if where != "v_scales" else "v_scales"][0])


def test_a_tensor_shorter_than_a_block(hl):
    """The lanes past the end of the only block."""
    for n in (1, 7, 8, 9, 255):
        t = state(n, "f32", False)
        t["grad"][n - 1] = NAN
        hl.hilore_adamw([hl.adamw_tensor(lr=1e-3, **t)], 0.9, 0.999, 1e-8, 1)
        assert torch.isnan(t["m_scales"][0]) and torch.isfinite(t["p"][:n - 1]).all() and torch.isnan(t["p"][n - 1])
