"""GPU parity of hilore_adamw and hilore_grad_norm against the 64-bit reference.

Tolerances, with u = 2^-24 (one fp32 rounding).  The new m and v are two products and a
sum: 3 u of the terms' sizes.  The parameter is p d - q with d rounded from 64 bits and q
seven fp32 operations on m and v, one of them the hardware reciprocal (1 ulp = 2 u) and one a
square root: 2 u |p| + 12 u |q| and one more rounding, |q| the size of the terms that m is
formed from.  An 8-bit state is one of the two codes
around its value and the random bits say which; the fp32 value decides otherwise than the
64-bit one only where it lies within its own error, 2^-20 of itself at the most, of the
threshold, whose distance from the next is at least 1/16 of it: n 2^-16 of n codes, and one.
Parameters in bf16 are rounded likewise, with 2^-8 between neighbours: n 2^-12 and one, none
further from the value than that spacing and the fp32 error.
"""
import numpy as np
import pytest
import torch

import layer_reference as ref
from gpu_util import dev, host

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
B1, B2, EPS = 0.9, 0.999, 1e-8


def f8(x):
    return torch.from_numpy(x).to(torch.float8_e4m3fn)


def make(n, seed, param="f32", grad="f32", bits=32, tail=0, size=1e-3):
    """Host and device state of one tensor; `tail` sentinel elements follow every buffer."""
    g = np.random.default_rng(seed)

    def pad(x, value):
        return np.concatenate([x, np.full(tail, value, dtype=x.dtype)])

    t = {"n": n, "bits": bits, "lr": 1e-2 * (1 + seed % 3), "wd": 0.1 * (seed % 2), "tail": tail}
    p = g.standard_normal(n).astype(np.float32)
    t["p"] = torch.from_numpy(pad(p, 7.0)) if param != "bf16" else None
    t["p16"] = torch.from_numpy(pad(p, 7.0)).to(torch.bfloat16) if param != "f32" else None
    # a few gradients of exactly zero, sizes over six decades
    grad_v = (g.standard_normal(n) * size * 10.0 ** g.uniform(-3, 3, n)).astype(np.float32)
    grad_v[g.random(n) < 0.05] = 0.0
    t["grad"] = torch.from_numpy(pad(grad_v, 7.0)).to(torch.bfloat16 if grad == "bf16" else torch.float32)
    m = (g.standard_normal(n) * size).astype(np.float32)
    r = (np.abs(g.standard_normal(n)) * size).astype(np.float32)
    if bits == 32:
        t["m"], t["v"] = (torch.from_numpy(pad(x.astype(np.float32), 7.0)) for x in (m, r * r))
        t["m_scales"] = t["v_scales"] = None
    else:
        for name, x in (("m", m), ("v", r)):
            b = ref.pad_blocks(x)
            s = (np.abs(b).max(1) / 448.0).astype(np.float32) if n else np.zeros(0, np.float32)
            codes = f8((b / np.where(s > 0, s, 1.0)[:, None]).reshape(-1)[:n].astype(np.float32))
            t[name] = torch.cat([codes.view(torch.uint8), torch.full((tail,), 0x5A, dtype=torch.uint8)])
            t[name + "_scales"] = torch.cat([torch.from_numpy(s), torch.full((tail,), 7.0)])
    t["dev"] = {k: t[k].cuda() if t[k] is not None else None
                for k in ("p", "p16", "grad", "m", "v", "m_scales", "v_scales")}
    return t


def descriptor(hl, t):
    n, blocks = t["n"], -(-t["n"] // 256)
    cut = {k: None if v is None else v[:blocks if "scales" in k else n] for k, v in t["dev"].items()}
    return hl.adamw_tensor(lr=t["lr"], weight_decay=t["wd"], **cut)


def values(t, name, n):
    """State `name` in 64 bits (r for an 8-bit v)."""
    x = t[name][:n]
    if t["bits"] == 32:
        return x.double().numpy()
    v = x.view(torch.float8_e4m3fn).double().numpy()
    return v * np.repeat(t[name + "_scales"][:-(-n // 256)].double().numpy(), 256)[:n]


def check(t, index, step, seed, clip=1.0):
    """One step of this tensor: the device's state against the reference from the host's."""
    n, out = t["n"], {k: None if v is None else v.cpu() for k, v in t["dev"].items()}
    for k, v in t["dev"].items():  # nothing past the end is written
        if v is not None and t["tail"]:
            assert torch.equal(out[k][-t["tail"]:].float(), t[k][-t["tail"]:].float()), k
    if n == 0:
        return
    lr, wd = float(np.float32(t["lr"])), float(np.float32(t["wd"]))
    p0 = (t["p"] if t["p"] is not None else t["p16"])[:n].double().numpy()
    g0, m0, v0 = t["grad"][:n].double().numpy(), values(t, "m", n), values(t, "v", n)
    if t["bits"] == 8:
        v0 = v0 ** 2
    p, m, v, q = ref.adamw(p0, g0, m0, v0, lr, wd, B1, B2, EPS, step, clip)
    g1 = g0 * clip
    if t["bits"] == 32:
        assert (np.abs(out["m"][:n].double().numpy() - m) <= 4 * U * (np.abs(m0) + np.abs(g1)) + 1e-45).all()
        assert (np.abs(out["v"][:n].double().numpy() - v) <= 6 * U * (v0 + g1 ** 2) + 1e-45).all()
    else:
        word = ref.words(seed, index, n, 0)
        for name, x, u in (("m", m, word & 0xFFFF), ("v", np.sqrt(v), word >> 16)):
            want, scale, k = ref.encode(x, u / 65536.0, name == "v")
            s = out[name + "_scales"][:-(-n // 256)].double().numpy()
            assert (np.abs(s - scale) <= 8 * U * scale).all(), name
            code = out[name][:n].view(torch.uint8).numpy()
            got = (code & 0x7F).astype(np.int64)
            assert (got <= 126).all() and (np.abs(got - k) <= 1).all(), name
            assert (got != k).sum() <= 1 + n * 2.0 ** -16, (name, (got != k).sum())
            assert ((code & 0x80 != 0) <= (x < 0)).all() and ((got == 0) | ((code & 0x80 != 0) == (x < 0))).all()
    if t["p"] is not None:
        got = out["p"][:n]
        assert (np.abs(got.double().numpy() - p) <= 4 * U * np.abs(p0) + 16 * U * q).all()
        if t["p16"] is not None:  # the nearest bf16 of the stored parameter
            assert torch.equal(out["p16"][:n], got.to(torch.bfloat16))
    else:
        word = (ref.words(seed, index, n, 0x3C6EF372) & 0xFFFF) / 65536.0
        quantum = np.exp2(np.frexp(p)[1].astype(np.float64) - 8.0)
        want = np.sign(p) * np.floor(np.abs(p) / quantum + word) * quantum
        got = out["p16"][:n].double().numpy()
        assert (np.abs(got - p) <= 1.001 * quantum + 4 * U * np.abs(p0) + 16 * U * q).all()
        assert (got != want).sum() <= 1 + n * 2.0 ** -12


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("grad", ["f32", "bf16"])
@pytest.mark.parametrize("param", ["f32", "bf16", "master"])
def test_kinds_and_lengths(hl, param, grad, bits):
    """Every kind of tensor at lengths around the lane's, the block's and the chunk's ends, in
    one call of two launches, sentinels behind every buffer."""
    lengths = [0, 1, 2, 3, 4, 5, 63, 255, 256, 257, 259, 511, 513, 1023, 4095, 4096, 4097, 4100, 8191, 16385, 40001]
    lengths = lengths + lengths[::-1] + [7] * 5
    assert len(lengths) > 44
    ts = [make(n, 100 + i, param, grad, bits, tail=9) for i, n in enumerate(lengths)]
    hl.hilore_adamw([descriptor(hl, t) for t in ts], B1, B2, EPS, 3, seed=17)
    torch.cuda.synchronize()
    for i, t in enumerate(ts):
        check(t, i, 3, 17)


def test_mixed_kinds_in_one_call_and_first_step(hl):
    kinds = [(p, g, b) for p in ("f32", "bf16", "master") for g in ("f32", "bf16") for b in (8, 32)]
    ts = [make(700 + 37 * i, 300 + i, *k, tail=3) for i, k in enumerate(kinds)]
    hl.hilore_adamw(hl.adamw_tensors([descriptor(hl, t) for t in ts]), B1, B2, EPS, 1, seed=0)
    torch.cuda.synchronize()
    for i, t in enumerate(ts):
        check(t, i, 1, 0)


def test_scales_of_many_tensors_in_one_array(hl):
    """8-bit scales start at any 4-byte boundary."""
    ts = [make(n, 350 + n, "f32", "f32", 8) for n in (255, 256, 300, 1000)]
    for name in ("m_scales", "v_scales"):
        joined, at = torch.cat([t[name] for t in ts]).cuda(), 0
        for t in ts:
            t["dev"][name] = joined[at:at + t[name].numel()]
            at += t[name].numel()
    hl.hilore_adamw([descriptor(hl, t) for t in ts], B1, B2, EPS, 2, seed=1)
    torch.cuda.synchronize()
    for i, t in enumerate(ts):
        check(t, i, 2, 1)


def test_large_tensor_random_words(hl):
    t = make(3_000_001, 400, "bf16", "bf16", 8)
    hl.hilore_adamw([descriptor(hl, t)], B1, B2, EPS, 1000, seed=0xFFFFFFF0)
    torch.cuda.synchronize()
    check(t, 0, 1000, 0xFFFFFFF0)


@pytest.mark.parametrize("count,size", [(1, 1), (1, 16384), (3, 16385), (150, 777), (2, 1_500_000)])
@pytest.mark.parametrize("grad", ["f32", "bf16"])
def test_norm(hl, count, size, grad):
    """fp64 sums: the result is the reference's to a rounding of the fp32 output (and 2^-40)."""
    ts = [make(size, 500 + i, "f32", grad, 32, tail=4) for i in range(count)]
    grads = [t["grad"][:size].float().numpy() for t in ts]
    norm = torch.full((2,), float("nan"), device="cuda")
    for max_norm in (0.5, 1e9, float("inf")):
        hl.hilore_grad_norm([descriptor(hl, t) for t in ts], max_norm, norm)
        want = ref.grad_norm(grads, max_norm)
        got = host(norm).astype(np.float64)
        assert abs(got[0] - want[0]) <= 2 * U * want[0] and abs(got[1] - want[1]) <= 2 * U, (got, want)


def test_norm_extremes(hl):
    """Squares beyond fp32's range either way; nothing at all; zero gradients; mixed types."""
    norm = torch.zeros(2, device="cuda")
    for v in (1e30, 1e-30):
        g = torch.full((1000,), v, device="cuda")
        hl.hilore_grad_norm([hl.adamw_tensor(grad=g, m=g, v=g, p=g)], 1.0, norm)
        assert abs(float(norm[0]) / (float(np.float32(v)) * 1000 ** 0.5) - 1) <= 2 * U
    hl.hilore_grad_norm([], 1.0, norm)
    assert norm.tolist() == [0.0, 1.0]
    z, b = torch.zeros(3, device="cuda"), torch.ones(9, device="cuda", dtype=torch.bfloat16)
    f = torch.zeros(9, device="cuda")
    hl.hilore_grad_norm([hl.adamw_tensor(grad=z, m=z, v=z, p=z), hl.adamw_tensor(grad=b, m=f, v=f, p=f)], 6.0, norm)
    assert norm.tolist() == [3.0, 1.0]


def test_clipped_step(hl):
    ts = [make(5000 + i, 600 + i, "f32", "f32", 8 if i % 2 else 32) for i in range(4)]
    arr = hl.adamw_tensors([descriptor(hl, t) for t in ts])
    norm = torch.zeros(2, device="cuda")
    hl.hilore_grad_norm(arr, 0.25, norm)
    hl.hilore_adamw(arr, B1, B2, EPS, 7, norm=norm, seed=5)
    clip = float(norm[1])
    assert clip < 0.5
    for i, t in enumerate(ts):
        check(t, i, 7, 5, clip)


@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_step_with_a_bad_gradient_is_skipped(hl, bad):
    ts = [make(3000, 700 + i, k, "f32", b) for i, (k, b) in enumerate([("f32", 32), ("master", 8), ("bf16", 8)])]
    ts[1]["dev"]["grad"][1234] = bad
    arr = hl.adamw_tensors([descriptor(hl, t) for t in ts])
    norm = torch.zeros(2, device="cuda")
    hl.hilore_grad_norm(arr, 1.0, norm)
    assert not torch.isfinite(norm[0]) and torch.isnan(norm[1])
    hl.hilore_adamw(arr, B1, B2, EPS, 2, norm=norm)
    torch.cuda.synchronize()
    for t in ts:
        for k in ("p", "p16", "m", "v", "m_scales", "v_scales"):
            if t[k] is not None:
                assert torch.equal(t["dev"][k].cpu().float(), t[k].float()), k


def test_small_changes_add_up_in_eight_bits(hl):
    """Without gradient r falls by sqrt(beta2) a step, far below a code's spacing: 400 steps
    have to leave 0.999^200 of it in the mean.  One rounding's variance is at most a quarter of
    the squared spacing, r/8 at most, so 400 of them leave a relative deviation of at most
    sqrt(400) / 16 = 1.25 per element and 0.005 in the mean of 2^16; five of these.  The blocks'
    largest values keep r's scale in place."""
    n = 1 << 16
    t = make(n, 800, "f32", "f32", 8)
    t["dev"]["grad"].zero_()
    r0 = torch.full((n,), 112.0)
    t["dev"]["v"].copy_(r0.to(torch.float8_e4m3fn).view(torch.uint8))
    t["dev"]["v_scales"].fill_(1e-4)
    arr = [descriptor(hl, t)]
    arr = hl.adamw_tensors(arr)
    for step in range(1, 401):
        hl.hilore_adamw(arr, B1, B2, EPS, step, seed=step)
    out = {**t, **{k: None if v is None else v.cpu() for k, v in t["dev"].items()}}
    r = values(out, "v", n)
    assert (r > 0).all()
    assert abs(r.mean() / 112e-4 / 0.999 ** 200 - 1) <= 0.025
    assert np.isfinite(host(t["dev"]["p"])).all()


def test_moment_never_vanishes(hl):
    """r a millionth of its block's largest value stays above zero in code."""
    n = 256
    t = make(n, 801, "f32", "f32", 8)
    g = torch.full((n,), 1e-9)
    g[0] = 10.0
    t["dev"]["grad"].copy_(g)
    t["dev"]["v"].zero_(), t["dev"]["v_scales"].zero_(), t["dev"]["m"].zero_(), t["dev"]["m_scales"].zero_()
    hl.hilore_adamw([descriptor(hl, t)], B1, B2, EPS, 1, seed=9)
    assert (t["dev"]["v"].cpu().view(torch.uint8) >= 1).all()


def test_zero_blocks(hl):
    """A block of zeros has scale 0 and codes 0, and its parameters only decay."""
    t = make(600, 802, "f32", "f32", 8)
    for k in ("grad", "m", "v", "m_scales", "v_scales"):
        t["dev"][k].zero_()
        t[k] = t["dev"][k].cpu()
    t["wd"] = 0.5
    hl.hilore_adamw([descriptor(hl, t)], B1, B2, EPS, 1)
    assert not t["dev"]["v_scales"].any() and not t["dev"]["v"].any() and not t["dev"]["m"].any()
    check(t, 0, 1, 0)


def test_graph_and_other_stream(hl):
    """Norm and step captured in a graph: three replays between eager work equal three eager
    steps on another stream bit for bit (the captured step count and seed stay)."""
    def fresh():
        ts = [make(3000 + 11 * i, 900 + i, "master", "f32", 8 if i % 2 else 32) for i in range(3)]
        return ts, hl.adamw_tensors([descriptor(hl, t) for t in ts]), torch.zeros(2, device="cuda")

    def once(arr, norm, ws, stream=None):
        hl.hilore_grad_norm(arr, 1.0, norm, workspace=ws, stream=stream)
        hl.hilore_adamw(arr, B1, B2, EPS, 4, norm=norm, seed=3, stream=stream)

    (a, arr_a, norm_a), (b, arr_b, norm_b) = fresh(), fresh()
    ws_a, ws_b = (torch.empty(hl.hilore_grad_norm_workspace_bytes(arr_a), dtype=torch.uint8, device="cuda") for _ in range(2))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        once(arr_a, norm_a, ws_a)
    side = torch.cuda.Stream()
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        once(arr_b, norm_b, ws_b, stream=side.cuda_stream)
        side.synchronize()
        for x, y in zip(a, b):
            for k, v in x["dev"].items():
                assert v is None or torch.equal(v.view(torch.uint8), y["dev"][k].view(torch.uint8)), k
        assert torch.equal(norm_a, norm_b)
    with pytest.raises(ValueError, match="explicit workspace"):
        hl.hilore_grad_norm(arr_b, 1.0, norm_b, stream=side.cuda_stream)


def test_lengths_past_32_bit_offsets(hl):
    """A tensor whose byte offsets pass 2^32: its ends against a small tensor's arithmetic."""
    n = (1 << 30) + 4099
    g = torch.empty(n, dtype=torch.bfloat16, device="cuda").fill_(1e-3)
    p = torch.zeros(n, device="cuda")
    m, v = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    norm = torch.zeros(2, device="cuda")
    arr = hl.adamw_tensors([hl.adamw_tensor(grad=g, m=m, v=v, p=p, lr=0.5)])
    hl.hilore_grad_norm(arr, float("inf"), norm)
    hl.hilore_adamw(arr, B1, B2, EPS, 1, norm=norm)
    gv = float(g[0])
    assert abs(float(norm[0]) / (gv * n ** 0.5) - 1) <= 2 * U
    want = ref.adamw(np.zeros(1), np.array([gv]), np.zeros(1), np.zeros(1), 0.5, 0.0, B1, B2, EPS, 1)
    for t, w in ((p, want[0]), (m, want[1]), (v, want[2])):
        assert abs(float(t[0]) - w[0]) <= 16 * U * abs(w[0])
        assert torch.equal(t.min(), t.max())
