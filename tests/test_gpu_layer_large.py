"""Layer operators past 2^32 elements and bytes: the last rows and elements come out as the same
values do in a small call, bit for bit."""
import pytest
import torch

from paper_2609_33570_amd import workloads as wl

pytestmark = pytest.mark.gpu
ROWS, COLS = 262_150, 16_384  # 2^32 + 98304 elements


@pytest.fixture(autouse=True)
def room():
    if torch.cuda.mem_get_info()[0] < 80 << 30:
        pytest.skip("needs 80 GB of device memory")
    yield
    torch.cuda.empty_cache()


def rows_of(g, count=10):
    """`count` rows, and as many thousands of them as ROWS."""
    x = torch.from_numpy(g.standard_normal((count, COLS), dtype="float32")).bfloat16().cuda()
    return x, x.repeat(ROWS // count, 1)


def test_block_norm(hl):
    g = wl.rng(1, 1)
    w = torch.ones(COLS, dtype=torch.bfloat16, device="cuda") * 1.5
    small, big = rows_of(g)
    outs = []
    for x in (small, big):
        n = torch.empty_like(x)
        codes, scales = torch.empty(x.shape, dtype=torch.int8, device="cuda"), torch.empty(len(x), device="cuda")
        r = torch.empty(len(x), device="cuda")
        hl.hilore_block_norm(hl.block_norm_desc(x, w_pre=w, n=n, codes=codes, code_scales=scales, rstd_pre=r))
        outs.append((n, codes, scales, r))
    for a, b in zip(*outs):
        assert torch.equal(a, b[:10]) and torch.equal(a, b[-10:])


@pytest.mark.parametrize("l_unit", [False, True])
def test_block_norm_bwd(hl, l_unit):
    g = wl.rng(2, 1)
    w = torch.ones(COLS, dtype=torch.bfloat16, device="cuda") * 1.5
    small, big = rows_of(g)
    outs = []
    for x in (small, big):
        r = torch.ones(len(x), device="cuda")
        if l_unit:
            codes = torch.empty(x.shape, dtype=torch.uint8, device="cuda")
            scales = torch.empty((len(x), COLS // 256), device="cuda")
            unit = hl.unit_desc(x=x, codes=codes, scales=scales)
            hl.hilore_compress([unit], "int8", 256)
            h = hl.unit_desc(codes=codes, scales=scales)
        else:
            h = hl.unit_desc(x=x)
        dres = torch.empty_like(x)
        hl.hilore_block_norm_bwd(hl.block_norm_bwd_desc(h=h, w_pre=w, rstd_pre=r, dn=x, dres=dres), "int8", 256)
        torch.cuda.synchronize()
        outs.append(dres)
    assert torch.equal(outs[0], outs[1][:10]) and torch.equal(outs[0], outs[1][-10:])


def test_int8(hl):
    g = wl.rng(3, 1)
    k = 64
    w = torch.from_numpy(g.integers(-127, 128, (COLS, k), dtype="int8")).cuda()
    x = torch.from_numpy(g.standard_normal((10, k), dtype="float32")).bfloat16().cuda()
    outs = []
    for t in (x, x.repeat(ROWS // 10, 1)):
        out = torch.empty((len(t), COLS), dtype=torch.bfloat16, device="cuda")
        hl.hilore_int8_linear(hl.int8_desc(w=w, out=out, x=t))
        outs.append(out)
    assert torch.equal(outs[0], outs[1][:10]) and torch.equal(outs[0], outs[1][-10:])


def test_rounding(hl):
    g = wl.rng(4, 1)
    small, big = rows_of(g)
    outs = []
    for x in (small, big):
        codes, scales = torch.empty(x.shape, dtype=torch.int8, device="cuda"), torch.empty(len(x), device="cuda")
        hl.hilore_quantize_tokens(x, codes, scales)
        outs.append((codes, scales))
    for a, b in zip(*outs):
        assert torch.equal(a, b[:10]) and torch.equal(a, b[-10:])


def test_adamw(hl):
    n, tail = (1 << 31) + 4099, 4099
    big = {k: torch.full((n,), v, device="cuda") for k, v in (("p", 1.0), ("grad", 0.01), ("m", 0.002), ("v", 1e-5))}
    big["grad"][-tail:] = torch.linspace(-1, 1, tail, device="cuda")
    start = 1 << 31  # 16-byte aligned
    small = {k: v[start:].clone() for k, v in big.items()}
    norms = []
    for t in (big, small):
        norm = torch.zeros(2, device="cuda")
        arr = hl.adamw_tensors([hl.adamw_tensor(lr=1e-3, weight_decay=0.1, **t)])
        hl.hilore_grad_norm(arr, 1.0, norm)
        hl.hilore_adamw(arr, 0.9, 0.999, 1e-8, 2)
        norms.append(float(norm[0]))
    for k in ("p", "m", "v"):
        assert torch.equal(big[k][start:], small[k])
        assert (big[k][:1 << 20] == big[k][0]).all() and torch.equal(big[k][start - 5:start], big[k][:5])
    want = (float(torch.tensor(0.01).double()) ** 2 * start + norms[1] ** 2) ** 0.5
    assert abs(norms[0] - want) <= 2.0 ** -22 * want
