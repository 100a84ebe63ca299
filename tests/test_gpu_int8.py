"""GPU parity of hilore_int8_linear, hilore_int8_matmul and hilore_quantize_tokens.

The rounding of tokens is a sequence of IEEE fp32 operations and has to match bit for bit.
Sums are exact: with unit scales and fp32 output every sum below 2^24 has to be the integer.
Otherwise out is at most five fp32 roundings from the 64-bit value: 5 2^-24 of the product's
size and of the bias, and for bf16 one rounding more, 2^-9 (2^-8 allowed across a tie).
"""
import numpy as np
import pytest
import torch

import layer_reference as ref
from gpu_util import filled
from paper_2609_33570_amd import workloads as wl

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def codes(g, *shape):
    return torch.from_numpy(g.integers(-127, 128, shape, dtype=np.int8))


def exact_sums(hl, tokens, k, n, seed, lo=-127):
    g = wl.rng(seed, 1)
    a, w = codes(g, tokens, k), codes(g, n, k)
    if k * 127 * 127 >= 1 << 24:  # keep the sums below 2^24: small values in one operand
        m = max(1, (1 << 24) // (k * 127) - 1)
        w = w % m if m < 127 else w
        w = w.to(torch.int8)
    out = filled((tokens, n + 8), torch.float32, 7.0)
    ones = torch.ones(tokens, device="cuda")
    at, wt = a.cuda(), w.cuda()
    hl.hilore_int8_matmul(hl.int8_desc(w=wt, out=out[:, :n], a=at, a_scales=ones))
    torch.cuda.synchronize()
    assert torch.equal(out[:, :n].cpu().double(), ref.int_product(a, w)), (tokens, k, n)
    assert (out[:, n:] == 7.0).all()


@pytest.mark.parametrize("tokens", [1, 2, 3, 8, 15, 16, 17, 31, 32, 33, 48, 63, 64, 65, 100, 127, 128, 129, 255, 256, 257, 300, 513, 701])
def test_token_counts(hl, tokens):
    for k, n in ((64, 64), (144, 72), (528, 264)):
        exact_sums(hl, tokens, k, n, seed=tokens)


@pytest.mark.parametrize("k", [16, 32, 48, 64, 80, 112, 128, 144, 240, 256, 272, 512, 528, 1024, 1040, 3584, 4112])
def test_depths(hl, k):
    for tokens, n in ((1, 8), (5, 136), (17, 520), (130, 264), (260, 512)):
        exact_sums(hl, tokens, k, n, seed=k)


@pytest.mark.parametrize("n", [8, 16, 24, 56, 64, 72, 120, 128, 136, 248, 256, 264, 504, 512, 520, 1032, 2056])
def test_widths(hl, n):
    for tokens, k in ((1, 16), (4, 272), (33, 512), (96, 128), (259, 528)):
        exact_sums(hl, tokens, k, n, seed=n)


@pytest.mark.parametrize("tokens,k,n", [(1, 18944, 3584), (64, 18944, 3584), (16, 3584, 18944), (1000, 3584, 4096),
                                        (2049, 896, 4864), (4100, 4096, 1024)])
def test_model_shapes(hl, tokens, k, n):
    """Sums as they come (rounded to fp32 once from int32): all outputs against the int64 sums."""
    g = torch.Generator(device="cuda").manual_seed(tokens)
    a, w = (torch.randint(-127, 128, s, generator=g, device="cuda", dtype=torch.int8) for s in ((tokens, k), (n, k)))
    out = filled((tokens, n), torch.float32, float("nan"))
    ones = torch.ones(tokens, device="cuda")
    hl.hilore_int8_matmul(hl.int8_desc(w=w, out=out, a=a, a_scales=ones))
    want = a.double() @ w.double().t().contiguous()
    assert torch.equal(out, want.float())


def test_extreme_sums(hl):
    """The largest magnitude that fits, 131072 * 127^2 < 2^31, both signs."""
    k = 131072
    a = torch.full((2, k), 127, dtype=torch.int8, device="cuda")
    a[1] = -127
    for tokens in (2, 40):
        x = a.repeat(tokens // 2, 1)
        w = torch.full((8, k), 127, dtype=torch.int8, device="cuda")
        out = filled((tokens, 8), torch.float32, 7.0)
        ones = torch.ones(tokens, device="cuda")
        hl.hilore_int8_matmul(hl.int8_desc(w=w, out=out, a=x, a_scales=ones))
        want = float(np.float32(k * 127 * 127))
        assert (out[0::2] == want).all() and (out[1::2] == -want).all()


def linear_case(hl, tokens, k, n, seed, factor=False, bias=False, w_scales=True, out_f32=False, accumulate=False, pad=0):
    g = wl.rng(seed, 2)
    x = torch.from_numpy(g.standard_normal((tokens, k + pad), dtype=np.float32))
    x[:, ::97] *= 40
    x = x.to(torch.bfloat16)
    w = codes(g, n, k)
    ws = torch.from_numpy(g.uniform(1e-4, 1e-2, n).astype(np.float32)) if w_scales else None
    f = torch.from_numpy(g.uniform(1e-4, 1e-2, k).astype(np.float32)) if factor else None
    b = torch.from_numpy(g.standard_normal(n, dtype=np.float32)).to(torch.bfloat16) if bias else None
    out0 = torch.from_numpy(g.standard_normal((tokens, n + pad), dtype=np.float32)).to(torch.float32 if out_f32 else torch.bfloat16)
    out = out0.cuda()
    xt, wt, wst, ft, bt = (None if t is None else t.cuda() for t in (x, w, ws, f, b))
    hl.hilore_int8_linear(hl.int8_desc(w=wt, out=out[:, :n], x=xt[:, :k], factor=ft, w_scales=wst, bias=bt, accumulate=accumulate))
    torch.cuda.synchronize()
    v = x[:, :k].float()
    if f is not None:
        v = v * f
    a, s = ref.token_codes(v)
    want = ref.int_product(a, w) * s.double()[:, None]
    if ws is not None:
        want = want * ws.double()
    size = want.abs()
    if b is not None:
        want, size = want + b.double(), size + b.double().abs()
    if accumulate:
        want, size = want + out0[:, :n].double(), size + out0[:, :n].double().abs()
    got = out[:, :n].cpu().double()
    tol = 5 * U * size + (0.0 if out_f32 else 2.0 ** -8 * want.abs())
    assert ((got - want).abs() <= tol).all()
    assert torch.equal(out[:, n:].cpu(), out0[:, n:])  # nothing between the rows is touched


@pytest.mark.parametrize("tokens,k,n", [(1, 64, 40), (1, 3584, 512), (3, 896, 128), (16, 272, 264), (20, 1040, 136),
                                        (70, 512, 248), (131, 896, 264), (300, 3584, 520), (600, 144, 1032)])
@pytest.mark.parametrize("kw", [dict(), dict(bias=True, pad=8), dict(factor=True, w_scales=False, pad=16),
                                dict(out_f32=True, bias=True), dict(accumulate=True), dict(accumulate=True, out_f32=True, pad=8)],
                         ids=["plain", "bias", "gradient", "f32", "added", "added_f32"])
def test_linear(hl, tokens, k, n, kw):
    linear_case(hl, tokens, k, n, seed=tokens + k + n, **kw)


@pytest.mark.parametrize("k", [16, 32, 240, 256, 2048, 2064, 8192, 18944])
@pytest.mark.parametrize("factor", [False, True])
def test_rounding_bit_for_bit(hl, k, factor):
    g = wl.rng(k, 3)
    tokens, pad = 37, 8
    x = torch.from_numpy(g.standard_normal((tokens, k + pad), dtype=np.float32) * np.exp(g.uniform(-30, 30, (tokens, 1))).astype(np.float32))
    x = x.to(torch.bfloat16)
    x[1] = 0
    x[2] = x[2] * 0 + 2.0 ** -70     # below the smallest scale
    x[3, :k] = torch.tensor([1.0, -1.0, 0.5, -0.5]).repeat(k // 4)  # ties: 63.5
    f = torch.from_numpy(g.uniform(0.5, 2.0, k).astype(np.float32)) if factor else None
    codes_t, scales = filled((tokens, k), torch.int8, 77), filled(tokens, torch.float32, float("nan"))
    hl.hilore_quantize_tokens(x.cuda()[:, :k], codes_t, scales, factor=None if f is None else f.cuda())
    v = x[:, :k].float()
    want, s = ref.token_codes(v if f is None else v * f)
    assert torch.equal(codes_t.cpu().long(), want) and torch.equal(scales.cpu(), s)


@pytest.mark.parametrize("tokens", [6, 70])
def test_nan_and_infinity_stay_in_their_token(hl, tokens):
    k, n = 256, 64
    g = wl.rng(8, 4)
    x = torch.from_numpy(g.standard_normal((tokens, k), dtype=np.float32)).to(torch.bfloat16)
    x[1, 3], x[2, 200], x[4, 0] = float("nan"), float("inf"), float("-inf")
    w = codes(g, n, k).cuda()
    out = filled((tokens, n), torch.bfloat16, 7.0)
    hl.hilore_int8_linear(hl.int8_desc(w=w, out=out, x=x.cuda()))
    out = out.cpu()
    assert torch.isnan(out[[1, 2, 4]]).all()
    rest = [i for i in range(tokens) if i not in (1, 2, 4)]
    assert torch.isfinite(out[rest].float()).all()


def test_empty(hl):
    """No tokens: nothing; no depth: bias or zeros."""
    w = torch.zeros((16, 0), dtype=torch.int8, device="cuda")
    bias = torch.arange(16, device="cuda").to(torch.bfloat16)
    for b in (bias, None):
        out = filled((3, 16), torch.bfloat16, 7.0)
        x = torch.zeros((3, 0), dtype=torch.bfloat16, device="cuda")
        hl.hilore_int8_linear(hl.int8_desc(w=w, out=out, x=x, bias=b))
        assert torch.equal(out, (bias if b is not None else torch.zeros_like(bias)).expand(3, 16))
    out = torch.zeros((0, 16), dtype=torch.bfloat16, device="cuda")
    x = torch.zeros((0, 32), dtype=torch.bfloat16, device="cuda")
    hl.hilore_int8_linear(hl.int8_desc(w=torch.zeros((16, 32), dtype=torch.int8, device="cuda"), out=out, x=x))


def test_gradient_of_the_input(hl):
    """dX = (dY * sw) W on the codes: against the transposed product in 64 bits, with the error of
    rounding a token to 127 steps: half a step per term, as independent errors uniform in it
    (step / sqrt(12)), six deviations; and by differences of the forward's own layer, which is
    linear in what its operand stands for."""
    tokens, k, n = 50, 512, 272
    g = wl.rng(12, 5)
    dy = torch.from_numpy(g.standard_normal((tokens, n), dtype=np.float32) * 1e-3).to(torch.bfloat16)
    w = codes(g, n, k)
    sw = torch.from_numpy(g.uniform(1e-4, 1e-2, n).astype(np.float32))
    dx = filled((tokens, k), torch.float32, float("nan"))
    hl.hilore_int8_linear(hl.int8_desc(w=w.t().contiguous().cuda(), out=dx, x=dy.cuda(), factor=sw.cuda()))
    v = dy.float() * sw
    want = v.double() @ w.double()
    step = v.abs().amax(1).double() / 127
    tol = 6 * step[:, None] / 12 ** 0.5 * w.double().square().sum(0).sqrt()
    got = dx.cpu().double()
    assert ((got - want).abs() <= tol).all()
    # f(x) = sum(dy * (x W^T sw)): its difference in one direction against dX along it
    e = torch.from_numpy(g.standard_normal((tokens, k), dtype=np.float32)).double()
    f = (dy.double() * ((e @ w.double().t()) * sw.double())).sum()
    assert abs(float((got * e).sum() - f)) <= float(tol.square().sum().sqrt())


def test_graph_and_stream(hl):
    for tokens in (1, 40, 300):
        k, n = 896, 520
        g = wl.rng(tokens, 6)
        x = torch.from_numpy(g.standard_normal((tokens, k), dtype=np.float32)).to(torch.bfloat16).cuda()
        w = codes(g, n, k).cuda()
        a, b = filled((tokens, n), torch.bfloat16, 0.0), filled((tokens, n), torch.bfloat16, 0.0)
        da, db = hl.int8_desc(w=w, out=a, x=x), hl.int8_desc(w=w, out=b, x=x)
        ws = torch.empty(hl.hilore_int8_workspace_bytes(da), dtype=torch.uint8, device="cuda")
        ws2 = torch.empty_like(ws)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            hl.hilore_int8_linear(da, workspace=ws)
        side = torch.cuda.Stream()
        for i in range(3):
            x.mul_(1.5)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            hl.hilore_int8_linear(db, workspace=ws2, stream=side.cuda_stream)
            side.synchronize()
            assert torch.equal(a, b), (tokens, i)
