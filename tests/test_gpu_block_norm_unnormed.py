"""hilore_block_norm_bwd of a block output that has no norm: dy = scale * gate * D does not depend on
y, so values of y that are not finite (read for the gate's gradient) leave it and dres as they are,
bit for bit, and reach those of the gate's gradients that they belong to alone."""
import pytest
import torch

from paper_2609_33570_amd import workloads as wl

pytestmark = pytest.mark.gpu


def run(hl, rows, cols, gate, y, dn=True, code=None):
    g = wl.rng(rows + cols, 41)

    def values(*shape, sigma=1.0):
        return (torch.from_numpy(g.standard_normal(shape, dtype="float32")) * sigma).bfloat16().cuda()

    h, dn_t, dh, w = values(rows, cols), values(rows, cols, sigma=1e-2), values(rows, cols, sigma=1e-2), values(cols)
    gate_t = values(*{"channel": (cols,), "token": (rows, 1), "element": (rows, cols)}[gate])
    r = torch.rsqrt(h.float().square().mean(1) + 1e-6)
    out = {"dres": torch.empty_like(h), "dy": torch.empty_like(h),
           "dgate": torch.empty(gate_t.shape, dtype=torch.bfloat16 if gate == "element" else torch.float32, device="cuda")}
    saved = hl.unit_desc(x=y) if code is None else hl.unit_desc(codes=y)
    first = dict(h=hl.unit_desc(x=h), w_pre=w, rstd_pre=r, dn=dn_t) if dn else {}
    hl.hilore_block_norm_bwd(hl.block_norm_bwd_desc(y=saved, gate=gate_t, scale=0.5, dh=dh, **first, **out), code or 0, 0)
    torch.cuda.synchronize()
    return out


@pytest.mark.parametrize("rows,cols", [(3, 64), (5, 896), (2, 8192), (2, 8208)])
@pytest.mark.parametrize("gate", ["channel", "token", "element"])
@pytest.mark.parametrize("dn", [True, False])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_y_that_is_not_finite(hl, rows, cols, gate, dn, bad):
    y = torch.from_numpy(wl.rng(3, 42).standard_normal((rows, cols), dtype="float32")).bfloat16().cuda()
    want = run(hl, rows, cols, gate, y, dn)
    y[1, 17] = bad
    got = run(hl, rows, cols, gate, y, dn)
    assert torch.equal(got["dres"], want["dres"]) and torch.equal(got["dy"], want["dy"])
    changed = ~torch.isfinite(got["dgate"].float())
    place = {"channel": (17,), "token": (1, 0), "element": (1, 17)}[gate]
    assert changed[place] and changed.sum() == 1
    changed[place] = True
    assert torch.equal(got["dgate"][~changed], want["dgate"][~changed])


def test_a_nan_code(hl):
    """The plain cast's NaN code in a saved y."""
    codes = torch.full((2, 64), 0x38, dtype=torch.uint8, device="cuda")
    want = run(hl, 2, 64, "element", codes, code="e4m3fn_cast")
    codes[0, 5] = 0x7F
    got = run(hl, 2, 64, "element", codes, code="e4m3fn_cast")
    assert torch.equal(got["dres"], want["dres"]) and torch.equal(got["dy"], want["dy"])
    assert torch.isnan(got["dgate"][0, 5]) and torch.isnan(got["dgate"]).sum() == 1
