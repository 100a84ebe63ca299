"""The 64-bit references of the layer operators on the host: gradients against central
differences, the 8-bit rounding against its own properties."""
import numpy as np
import pytest
import torch

import layer_reference as ref


@pytest.mark.parametrize("post", [True, False])
@pytest.mark.parametrize("gate", [None, "channel", "token", "element"])
def test_norm_gradients_against_differences(post, gate):
    """Every gradient against (f(x + e) - f(x - e)) / 2e in 64 bits.  With e = 1e-5 the
    difference's own errors are about e^2 (curvature, values of order 1) and 2^-53 / e, both
    below 1e-9; 1e-7 of the largest gradient leaves room for sums of terms."""
    gen = torch.Generator().manual_seed(5)

    def draw(*shape):
        return torch.randn(shape, generator=gen, dtype=torch.float64)

    rows, cols, scale, eps = 3, 8, 0.7, 1e-6
    x = {"res": draw(rows, cols), "y": draw(rows, cols), "w_post": draw(cols) if post else None,
         "gate": {None: None, "channel": draw(cols), "token": draw(rows, 1),
                  "element": draw(rows, cols)}[gate], "w_pre": draw(cols)}
    dn, dh = draw(rows, cols), draw(rows, cols)

    def loss(x):
        h, _, enter = ref.norm_forward(x["res"], x["y"], x["w_post"], x["gate"], scale, x["w_pre"], eps)
        return float((enter(h)[0] * dn).sum() + (h * dh).sum())

    h, r_post, enter = ref.norm_forward(x["res"], x["y"], x["w_post"], x["gate"], scale, x["w_pre"], eps)
    got = ref.norm_backward(h, x["y"], x["w_post"], x["gate"], scale, x["w_pre"], r_post, enter(h)[1], dn, dh)
    for name, grad in (("res", "dres"), ("y", "dy"), ("w_post", "dw_post"), ("gate", "dgate"),
                       ("w_pre", "dw_pre")):
        if x[name] is None:
            continue
        want = torch.zeros_like(x[name])
        for i in range(want.numel()):
            side = []
            for e in (1e-5, -1e-5):
                t = x[name].clone()
                t.view(-1)[i] += e
                side.append(loss({**x, name: t}))
            want.view(-1)[i] = (side[0] - side[1]) / 2e-5
        assert (got[grad] - want).abs().max() <= 1e-7 * max(1.0, float(want.abs().max())), name


def test_code_grid_is_e4m3fn():
    codes = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(ref.GRID, codes)


def test_random_rounding_is_unbiased():
    """Mean of many roundings of one value.  The variance of one is at most spacing^2 / 4, so
    the mean of 2^16 has a standard deviation of at most spacing / 512; six of them."""
    n = 1 << 16
    x = np.full(n, 1.0)
    x[0::256] = 448.0 * 0.97  # the blocks' largest value
    for v in (0.013, 0.7, 1.03, 17.3, 200.1):
        x[1:] = np.where(np.arange(1, n) % 256 == 0, x[1:], v)
        word = ref.words(11, 3, n, 0)
        for u in (word & 0xFFFF, word >> 16):
            value, scale, k = ref.encode(x, u / 65536.0, False)
            keep = np.arange(n) % 256 != 0
            j = np.searchsorted(ref.GRID, v / scale[0])
            spacing = (ref.GRID[j] - ref.GRID[j - 1]) * scale[0]
            assert abs(value[keep].mean() - v) <= 6 * spacing / 512, v
