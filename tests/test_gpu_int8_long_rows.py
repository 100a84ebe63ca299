"""Rounding of rows longer than a workgroup holds in registers (32768 values), which are read twice:
bit for bit as the definition, alone and in front of a product."""
import numpy as np
import pytest
import torch

import layer_reference as ref
from gpu_util import filled
from paper_2609_33570_amd import workloads as wl
from test_gpu_int8 import linear_case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens,k", [(5, 32752), (5, 32768), (5, 32784), (3, 65552), (2, 131072), (1, 1 << 20), (1100, 32784)])
@pytest.mark.parametrize("factor", [False, True])
def test_rounding(hl, tokens, k, factor):
    g = wl.rng(k, 51)
    x = torch.from_numpy(g.standard_normal((tokens, k + 24), dtype=np.float32) *
                         np.exp(g.uniform(-20, 20, (tokens, 1))).astype(np.float32)).bfloat16()
    x[0, k - 1] = x[0].abs().max() * 2  # the largest value is the row's last one
    if tokens > 1:
        x[1] = 0
    f = torch.from_numpy(g.uniform(0.5, 2.0, k).astype(np.float32)) if factor else None
    codes, scales = filled((tokens, k), torch.int8, 77), filled(tokens, torch.float32, float("nan"))
    hl.hilore_quantize_tokens(x.cuda()[:, :k], codes, scales, factor=None if f is None else f.cuda())
    v = x[:, :k].float()
    want, s = ref.token_codes(v if f is None else v * f)
    assert torch.equal(codes.cpu().long(), want) and torch.equal(scales.cpu(), s)


def test_not_finite(hl):
    """In the second half of a long row."""
    k = 65552
    x = torch.ones(4, k, dtype=torch.bfloat16)
    x[1, 40000], x[2, k - 1] = float("nan"), float("-inf")
    codes, scales = filled((4, k), torch.int8, 77), filled(4, torch.float32, 7.0)
    hl.hilore_quantize_tokens(x.cuda(), codes, scales)
    assert torch.isnan(scales[1:3]).all() and not codes[1:3].any()
    assert (codes[[0, 3]] == 127).all() and torch.isfinite(scales[[0, 3]]).all()


@pytest.mark.parametrize("tokens,k,n", [(1, 32784, 136), (20, 65552, 72), (70, 32784, 264), (3, 131072, 8)])
@pytest.mark.parametrize("kw", [dict(pad=8), dict(pad=16, factor=True, w_scales=False)], ids=["forward", "gradient"])
def test_linear(hl, tokens, k, n, kw):
    linear_case(hl, tokens, k, n, seed=tokens + k, **kw)
