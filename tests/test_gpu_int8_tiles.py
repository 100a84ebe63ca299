"""GPU parity of the int8 products of many tokens: tiles of both sizes, several tiles for a
workgroup, tiles that end inside the operands, and k in parts that are added up.

Every product of at most 2^17 codes is exact in int32, so the 64-bit product of the same codes
is the oracle: with unit scales and fp32 output the only rounding is the one of the sum to
fp32.  With scales out is at most five fp32 roundings from the 64-bit value, 5 2^-24 of the
product's size and of what is added, and for bf16 one rounding more, 2^-8 across a tie.
"""
import pytest
import torch

from gpu_util import filled

pytestmark = pytest.mark.gpu
U = 2.0 ** -24

# few and many tiles, one to 17 parts of k, last tiles of 1 to 256 rows and 8 to 256 channels
SHAPES = [(65, 528, 264), (70, 131072, 8), (100, 18944, 1032), (130, 4112, 264), (257, 16, 8), (300, 3584, 520),
          (515, 65536, 264), (900, 18944, 3592), (1300, 64, 4104), (2049, 18944, 1032), (2100, 1040, 2056),
          (4400, 2064, 4104), (5200, 2064, 5128), (5400, 1040, 5128), (33, 18944, 3584), (64, 3584, 18944)]


def random_codes(seed, *shape):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(-127, 128, shape, generator=g, device="cuda", dtype=torch.int8)


def sums(a, w):
    return a.double() @ w.double().t().contiguous()


@pytest.mark.parametrize("tokens,k,n", SHAPES)
def test_sums(hl, tokens, k, n):
    a, w = random_codes(tokens, tokens, k), random_codes(n, n, k)
    ones = torch.ones(tokens, device="cuda")
    out = filled((tokens, n + 8), torch.float32, 7.0)
    hl.hilore_int8_matmul(hl.int8_desc(w=w, out=out[:, :n], a=a, a_scales=ones))
    assert torch.equal(out[:, :n], sums(a, w).float())
    assert (out[:, n:] == 7.0).all()


@pytest.mark.parametrize("tokens,k,n", [(130, 4112, 264), (700, 18944, 1032), (900, 18944, 3592), (1300, 64, 4104),
                                        (5200, 2064, 5128)])
@pytest.mark.parametrize("out_f32", [False, True])
@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("scaled", [False, True])
def test_outputs(hl, tokens, k, n, out_f32, accumulate, scaled):
    g = torch.Generator(device="cuda").manual_seed(k)
    a, w = random_codes(tokens, tokens, k), random_codes(n, n, k)
    sa = torch.rand(tokens, generator=g, device="cuda") * 1e-2 + 1e-4
    sw = torch.rand(n, generator=g, device="cuda") * 1e-2 + 1e-4 if scaled else None
    bias = torch.randn(n, generator=g, device="cuda").bfloat16() if scaled else None
    out0 = torch.randn(tokens, n + 8, generator=g, device="cuda").to(torch.float32 if out_f32 else torch.bfloat16)
    out = out0.clone()
    hl.hilore_int8_matmul(hl.int8_desc(w=w, out=out[:, :n], a=a, a_scales=sa, w_scales=sw, bias=bias,
                                       accumulate=accumulate))
    want = sums(a, w) * sa.double()[:, None]
    if scaled:
        want = want * sw.double()
    size = want.abs()
    if scaled:
        want, size = want + bias.double(), size + bias.double().abs()
    if accumulate:
        want, size = want + out0[:, :n].double(), size + out0[:, :n].double().abs()
    tol = 5 * U * size + (0.0 if out_f32 else 2.0 ** -8 * want.abs())
    assert ((out[:, :n].double() - want).abs() <= tol).all()
    assert torch.equal(out[:, n:], out0[:, n:])


def test_same_bits_each_time(hl):
    """Parts of k are added as integers: no order changes a result."""
    a, w = random_codes(1, 128, 18944), random_codes(2, 3584, 18944)
    sa = torch.rand(128, device="cuda")
    outs = [filled((128, 3584), torch.bfloat16, float("nan")) for _ in range(3)]
    for out in outs:
        hl.hilore_int8_matmul(hl.int8_desc(w=w, out=out, a=a, a_scales=sa))
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


@pytest.mark.parametrize("tokens", [70, 700])
def test_no_depth(hl, tokens):
    """k = 0: the bias alone."""
    n = 264
    bias = torch.randn(n, device="cuda").bfloat16()
    out = filled((tokens, n), torch.bfloat16, float("nan"))
    hl.hilore_int8_matmul(hl.int8_desc(w=torch.empty(n, 0, dtype=torch.int8, device="cuda"), out=out,
                                       a=torch.empty(tokens, 0, dtype=torch.int8, device="cuda"),
                                       a_scales=torch.ones(tokens, device="cuda"), bias=bias))
    assert torch.equal(out, bias.expand(tokens, n))


@pytest.mark.parametrize("tokens,k,n", [(4200, 4112, 4104), (4400, 2064, 4104), (1789, 4864, 18944), (6167, 1616, 9480)])
@pytest.mark.parametrize("out_f32,accumulate", [(False, False), (True, False), (False, True)])
def test_last_tiles_in_quarters(hl, tokens, k, n, out_f32, accumulate):
    """A last round of few large tiles goes as quarters, some of which lie past the operands."""
    a, w = random_codes(tokens, tokens, k), random_codes(n, n, k)
    g = torch.Generator(device="cuda").manual_seed(k)
    sa = torch.rand(tokens, generator=g, device="cuda") * 1e-2 + 1e-4
    sw = torch.rand(n, generator=g, device="cuda") * 1e-2 + 1e-4
    bias = torch.randn(n, generator=g, device="cuda").bfloat16()
    out0 = torch.randn(tokens + 3, n + 8, generator=g, device="cuda").to(torch.float32 if out_f32 else torch.bfloat16)
    out = out0.clone()
    hl.hilore_int8_matmul(hl.int8_desc(w=w, out=out[:tokens, :n], a=a, a_scales=sa, w_scales=sw, bias=bias,
                                       accumulate=accumulate))
    want = sums(a, w) * sa.double()[:, None] * sw.double()
    size = want.abs() + bias.double().abs()
    want = want + bias.double()
    if accumulate:
        want, size = want + out0[:tokens, :n].double(), size + out0[:tokens, :n].double().abs()
    tol = 5 * U * size + (0.0 if out_f32 else 2.0 ** -8 * want.abs())
    assert ((out[:tokens, :n].double() - want).abs() <= tol).all()
    assert torch.equal(out[:, n:], out0[:, n:]) and torch.equal(out[tokens:], out0[tokens:])
