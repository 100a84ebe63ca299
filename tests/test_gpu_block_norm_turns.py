"""The block norms where a workgroup takes several turns of rows, with the last turn
part full: sums over rows then run over turns, rows side by side and workgroups.

The bounds are those of the backward's other tests, 1e-5 of the size of a sum's terms: a sum in
parts (turns, then rows side by side, then workgroups) has fewer roundings than one in order.
"""
import pytest
import torch

from test_gpu_block_norm import backward, inputs

pytestmark = pytest.mark.gpu

# rows past 256 or 512 workgroups of 8, 4, 2 and 1 rows side by side; two and four pieces a thread
SHAPES = [(9001, 128), (2600, 1000), (2049, 1800), (1100, 3584), (700, 4104), (600, 8200)]


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("gate", ["channel", "token"])
def test_several_turns(hl, orc, rows, cols, gate):
    backward(hl, orc, inputs(rows, cols, True, gate, seed=rows + cols), 0.37)


def test_l_units_over_turns(hl, orc):
    backward(hl, orc, inputs(2600, 1024, True, "channel", seed=5), 0.5, 1, 128)
    backward(hl, orc, inputs(600, 8448, True, "channel", seed=6), 0.5, 0, 64)


@pytest.mark.parametrize("rows,cols", [(5003, 1000), (3001, 4104), (1601, 8200)])
def test_forward_over_turns(hl, rows, cols):
    """Rows of one pattern, which come out alike whatever turn they fall into."""
    t = inputs(7, cols, True, "token", seed=cols)
    res, y, gate = (t[k].repeat(-(-rows // 7), 1)[:rows].cuda() for k in ("res", "y", "gate"))
    h, n = torch.empty_like(res), torch.empty_like(res)
    hl.hilore_block_norm(hl.block_norm_desc(res, y=y, w_post=t["w_post"].cuda(), gate=gate, w_pre=t["w_pre"].cuda(), h=h,
                                            n=n))
    assert torch.isfinite(n.float()).all() and n.float().abs().sum() > 0
    for out in (h, n):
        assert torch.equal(out, out[:7].repeat(-(-rows // 7), 1)[:rows])
