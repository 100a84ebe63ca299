"""GPU parity of hilore_block_norm and hilore_block_norm_bwd against the 64-bit reference.

Tolerances.  A bf16 output is rounded once (2^-9 of itself; 2^-8 allowed, as one more fp32
error can move it across a tie) from an fp32 value whose own error is a few roundings of the
terms it is formed from: 1e-5 of their sizes.  n is checked against the norm of the h that the
call wrote, which is its definition.  Row factors are fp32 sums of squares, without
cancellation: the sum's error is below cols 2^-24 of it in the worst order and about
sqrt(cols) 2^-24 in fact, half of it in the root: 1e-5.  Sums over rows (dw, a channel's dgate)
and over columns (a token's) may cancel: 1e-5 of the sum of the terms' magnitudes.
"""
import numpy as np
import pytest
import torch

import layer_reference as ref
from gpu_util import dev, filled, host
from paper_2609_33570_amd import workloads as wl

pytestmark = pytest.mark.gpu
REL = 1e-5


def values(g, *shape, sigma=1.0, mean=0.0):
    x = torch.from_numpy(g.standard_normal(shape, dtype=np.float32)) * sigma + mean
    return x.to(torch.bfloat16)


def padded(x, pad, value=float("nan")):
    """x on the device with `pad` sentinel elements after every row, as a view."""
    if x is None:
        return None
    full = torch.full((x.shape[0], x.shape[1] + pad), value, dtype=x.dtype)
    full[:, :x.shape[1]] = x
    return full.cuda()[:, :x.shape[1]]


def cuda(x):
    return None if x is None else x.cuda()


def f64(x):
    return None if x is None else x.double().cpu()


def inputs(rows, cols, post, gate, seed, y=True):
    g = wl.rng(seed, 7)
    t = {"res": values(g, rows, cols, sigma=2.0), "y": values(g, rows, cols) if y else None,
         "w_post": values(g, cols, sigma=0.1, mean=1.0) if post else None, "w_pre": values(g, cols, sigma=0.1, mean=1.0),
         "gate": {"none": None, "channel": values(g, cols), "token": values(g, rows, 1),
                  "element": values(g, rows, cols)}[gate],
         "dn": values(g, rows, cols, sigma=1e-2), "dh": values(g, rows, cols, sigma=1e-2)}
    heavy = g.choice(cols, max(1, cols // 50), replace=False)
    t["res"][:, heavy] *= 30
    return t


def near(got, want, size, what):
    """bf16 output against its value and the size of its terms."""
    bad = (got.double().cpu() - want).abs() > 2.0 ** -8 * want.abs() + REL * size
    assert not bad.any(), (what, int(bad.sum()), bad.nonzero()[:3].tolist())


def close(got, want, size, what):
    bad = (got.double().cpu().reshape(want.shape) - want).abs() > REL * size + 1e-30
    assert not bad.any(), (what, int(bad.sum()), bad.nonzero()[:3].tolist())


SHAPES = [(1, 8), (3, 16), (7, 64), (2, 504), (5, 512), (9, 520), (4, 896), (3, 2048), (2, 3584), (3, 4096), (2, 4104),
          (2, 8192), (1, 8200), (2, 16384), (301, 128)]


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("post,gate", [(True, "channel"), (True, "none"), (False, "token"), (True, "element"), (False, "none")])
def test_forward(hl, rows, cols, post, gate):
    t = inputs(rows, cols, post, gate, seed=rows * 31 + cols)
    scale, eps = 0.37, 1e-5
    h, n = filled((rows, cols), torch.bfloat16, float("nan")), filled((rows, cols), torch.bfloat16, float("nan"))
    r_post, r_pre = filled(rows, torch.float32, float("nan")), filled(rows, torch.float32, float("nan"))
    codes = filled((rows, cols), torch.int8, 77) if cols % 16 == 0 else None
    cs = filled(rows, torch.float32, float("nan")) if codes is not None else None
    res, y = padded(t["res"], 24), padded(t["y"], 8)
    w_post, gate_t, w_pre = cuda(t["w_post"]), cuda(t["gate"]), cuda(t["w_pre"])
    hl.hilore_block_norm(hl.block_norm_desc(res, y=y, w_post=w_post, gate=gate_t, scale=scale, w_pre=w_pre, eps=eps, h=h,
                                            n=n, codes=codes, code_scales=cs, rstd_post=r_post if post else None,
                                            rstd_pre=r_pre))
    torch.cuda.synchronize()
    scale32, eps32 = float(np.float32(scale)), float(np.float32(eps))
    want, want_post, enter = ref.norm_forward(f64(t["res"]), f64(t["y"]), f64(t["w_post"]), f64(t["gate"]), scale32,
                                              f64(t["w_pre"]), eps32)
    near(h, want, f64(t["res"]).abs() + (want - f64(t["res"])).abs(), "h")
    if post:
        close(r_post, want_post, want_post, "rstd_post")
    want_n, want_pre = enter(f64(h))
    close(r_pre, want_pre, want_pre, "rstd_pre")
    near(n, want_n, want_n.abs(), "n")
    if codes is not None:
        amax = want_n.abs().amax(1)
        close(cs, amax / 127, amax / 127, "code_scales")
        exact = want_n / (amax[:, None] / 127)
        # RNE of a value known to a few 1e-6 of itself
        assert ((codes.double().cpu() - exact).abs() <= 0.5 + 127 * REL).all()


def test_first_norm_last_sum_and_in_place(hl):
    """Without a block output (nothing is written but n), without a next norm, and h over res."""
    t = inputs(6, 896, True, "channel", seed=1)
    res, y, w_post, gate, w_pre = (cuda(t[k]) for k in ("res", "y", "w_post", "gate", "w_pre"))
    n = filled((6, 896), torch.bfloat16, float("nan"))
    hl.hilore_block_norm(hl.block_norm_desc(res, w_pre=w_pre, n=n))
    want = ref.norm_forward(f64(t["res"]), None, None, None, 1.0, f64(t["w_pre"]), float(np.float32(1e-6)))[2](f64(t["res"]))[0]
    near(n, want, want.abs(), "n")
    h, n2 = torch.empty_like(res), torch.empty_like(res)
    args = dict(y=y, w_post=w_post, gate=gate, scale=0.5)
    hl.hilore_block_norm(hl.block_norm_desc(res, h=h, **args))
    hl.hilore_block_norm(hl.block_norm_desc(res, h=res, w_pre=w_pre, n=n2, **args))
    assert torch.equal(h, res)
    # a recompute from the kept h gives the same bits
    hl.hilore_block_norm(hl.block_norm_desc(h, w_pre=w_pre, n=n))
    assert torch.equal(n, n2)


def test_rows_that_are_zero_huge_or_nan(hl):
    """Zero rows stay zero through eps, a NaN stays in its row, codes of both are defined."""
    rows, cols = 5, 256
    x = values(wl.rng(3, 1), rows, cols)
    x[1] = 0
    x[2, 17] = float("nan")
    x[3, 5] = float("inf")
    w = torch.ones(cols, dtype=torch.bfloat16)
    res, w_pre = x.cuda(), w.cuda()
    n, codes = torch.empty_like(res), filled((rows, cols), torch.int8, 77)
    cs, r = filled(rows, torch.float32, 7.0), filled(rows, torch.float32, 7.0)
    hl.hilore_block_norm(hl.block_norm_desc(res, w_pre=w_pre, n=n, codes=codes, code_scales=cs, rstd_pre=r, eps=1e-6))
    n, codes, cs = n.cpu(), codes.cpu(), cs.cpu()
    assert not n[1].any() and not codes[1].any() and cs[1] == 0
    assert torch.isnan(n[2]).all() and torch.isnan(cs[2]) and not codes[2].any()
    assert torch.isnan(cs[3]) and not codes[3].any()
    assert torch.isfinite(n[[0, 1, 4]].float()).all() and torch.isfinite(cs[[0, 1, 4]]).all()


def test_many_rows(hl):
    """More rows than any grid has workgroups at once, all of them one pattern."""
    rows, cols = 200_003, 64
    t = inputs(7, cols, True, "token", seed=4)
    big = {k: t[k].repeat(-(-rows // 7), 1)[:rows].cuda() for k in ("res", "y", "gate")}
    w_post, w_pre = t["w_post"].cuda(), t["w_pre"].cuda()
    h, n = torch.empty_like(big["res"]), torch.empty_like(big["res"])
    hl.hilore_block_norm(hl.block_norm_desc(big["res"], y=big["y"], w_post=w_post, gate=big["gate"], w_pre=w_pre, h=h, n=n))
    for out in (h, n):
        assert torch.equal(out, out[:7].repeat(-(-rows // 7), 1)[:rows])


# ---------------------------------------------------------------- backward --
def backward(hl, orc, t, scale, code=None, block=0, weights=True, dn=True, dh=True, accumulate=False, inplace=False,
             units=("h", "y")):
    """Runs the call on what the forward would have saved; returns outputs and the reference."""
    rows, cols = t["res"].shape
    h = t["res"]
    y = t["y"]
    saved, keep = {}, []
    for name, x in (("h", h), ("y", y)):
        if x is None:
            saved[name] = (None, None)
        elif code is not None and name in units:
            bits = host(x)
            c, s = orc.quantize(bits, code, block)
            xhat = torch.from_numpy(orc.dequantize(c, s, code, block).view(np.int16)).view(torch.bfloat16)
            ct, st = dev(c), dev(s) if s is not None else None
            keep += [ct, st]
            saved[name] = (hl.unit_desc(codes=ct, scales=st, rows=rows, cols=cols), xhat)
        else:
            xt = padded(x, 16)
            keep.append(xt)
            saved[name] = (hl.unit_desc(x=xt, cols=cols, ld=cols + 16), x)
    # the factors of the forward, from the values before the codec
    r_pre = (f64(h).square().mean(1) + 1e-6).rsqrt().float()
    r_post = (f64(y).square().mean(1) + 1e-6).rsqrt().float() if t["w_post"] is not None else None
    out = {"dres": filled((rows, cols), torch.bfloat16, float("nan")), "dy": filled((rows, cols), torch.bfloat16, float("nan"))}
    start = 0.5 if accumulate else float("nan")
    if weights:
        if dn:
            out["dw_pre"] = filled(cols, torch.float32, start)
        if t["w_post"] is not None:
            out["dw_post"] = filled(cols, torch.float32, start)
    kind = None if t["gate"] is None else tuple(t["gate"].shape)
    if kind is not None and y is not None and (weights or kind != (cols,)):
        out["dgate"] = filled(kind, torch.bfloat16 if kind == (rows, cols) and cols > 1 else torch.float32,
                              start if kind == (cols,) else float("nan"))
    dn_t, dh_t = padded(t["dn"], 8) if dn else None, cuda(t["dh"]) if dh else None
    if inplace:
        out["dres"] = dh_t
    args = {k: cuda(t[k]) for k in ("w_post", "gate")}
    args["w_pre"], rp, rq = (cuda(t["w_pre"]), cuda(r_pre), cuda(r_post)) if dn else (None, None, cuda(r_post))
    desc = hl.block_norm_bwd_desc(h=saved["h"][0] if dn else None, y=saved["y"][0], scale=scale, rstd_pre=rp, rstd_post=rq,
                                  dn=dn_t, dh=dh_t, **args, **out)
    hl.hilore_block_norm_bwd(desc, 0 if code is None else code, block, accumulate=accumulate)
    torch.cuda.synchronize()
    want = ref.norm_backward(f64(saved["h"][1]) if dn else None, f64(saved["y"][1]) if y is not None else None,
                             f64(t["w_post"]), f64(t["gate"]), float(np.float32(scale)), f64(t["w_pre"]) if dn else None,
                             f64(r_post), f64(r_pre), f64(t["dn"]) if dn else None, f64(t["dh"]) if dh else None)
    # sizes of the terms, for the tolerances
    size = {}
    hh = f64(saved["h"][1]).abs() * f64(r_pre)[:, None] if dn else None
    zero = torch.zeros(rows, cols, dtype=torch.float64)
    d = f64(t["dh"]).abs() if dh else zero
    if dn:
        tt = f64(t["dn"]).abs() * f64(t["w_pre"]).abs()
        d = d + f64(r_pre)[:, None] * (tt + hh * (tt * hh).mean(1, keepdim=True))
        size["dw_pre"] = (f64(t["dn"]).abs() * hh).sum(0)
    size["dres"] = d
    dz = abs(scale) * d
    if y is not None:
        yh = f64(saved["y"][1]).abs() * (1.0 if r_post is None else f64(r_post)[:, None])
        z = yh if t["w_post"] is None else yh * f64(t["w_post"]).abs()
        if t["gate"] is not None:
            size["dgate"] = (dz * z).sum_to_size(t["gate"].shape)
    if t["gate"] is not None:
        dz = dz * f64(t["gate"]).abs()
    if t["w_post"] is not None:
        size["dw_post"] = (dz * yh).sum(0)
        tt = dz * f64(t["w_post"]).abs()
        dz = f64(r_post)[:, None] * (tt + yh * (tt * yh).mean(1, keepdim=True))
    size["dy"] = dz
    for k, got in out.items():
        w = want[k]
        if got.dtype == torch.bfloat16:
            near(got, w, size[k], k)
        else:
            if accumulate and k != "dgate" or accumulate and kind == (cols,):
                w, size[k] = w + 0.5, size[k] + 0.5
            close(got, w, size[k], k)
    return out


@pytest.mark.parametrize("rows,cols", SHAPES + [(1500, 64), (700, 896)])
@pytest.mark.parametrize("post,gate", [(True, "channel"), (True, "none"), (False, "token"), (True, "element"),
                                       (True, "token"), (False, "channel"), (False, "none")])
def test_backward(hl, orc, rows, cols, post, gate):
    y = post or gate != "none"
    backward(hl, orc, inputs(rows, cols, post, gate, seed=rows * 17 + cols, y=y), 0.37)


@pytest.mark.parametrize("code,block", [(0, 32), (0, 256), (1, 64), (1, 128), (2, 0)])
@pytest.mark.parametrize("units", [("h", "y"), ("h",), ("y",)])
@pytest.mark.parametrize("cols", [256, 3584])
def test_backward_of_l_units(hl, orc, code, block, units, cols):
    backward(hl, orc, inputs(9, cols, True, "channel", seed=cols + block), 0.5, code, block, units=units)


def test_backward_parts(hl, orc):
    """Frozen weights; no gradient past the block; none through its norm; dres over dh; added sums."""
    t = inputs(33, 896, True, "channel", seed=9)
    backward(hl, orc, t, 0.5, weights=False)
    backward(hl, orc, t, 0.5, dh=False)
    backward(hl, orc, t, 0.5, dn=False)
    backward(hl, orc, t, 1.0, accumulate=True)
    backward(hl, orc, t, 1.0, inplace=True)
    backward(hl, orc, inputs(33, 896, False, "none", seed=10, y=False), 1.0, 1, 128, weights=False)
    backward(hl, orc, inputs(40, 896, True, "token", seed=11), 1.0, accumulate=True)


def test_backward_repeats_bit_for_bit(hl, orc):
    t = inputs(900, 896, True, "channel", seed=12)
    a, b = backward(hl, orc, t, 0.5), backward(hl, orc, t, 0.5)
    for k in a:
        assert torch.equal(a[k], b[k]), k


def test_backward_of_no_rows(hl):
    """No tokens: the sums over them are zero, or what was there."""
    cols = 64
    x = torch.zeros((0, cols), dtype=torch.bfloat16, device="cuda")
    w = torch.ones(cols, dtype=torch.bfloat16, device="cuda")
    r = torch.zeros(0, device="cuda")
    dw = filled(cols, torch.float32, 3.0)
    desc = hl.block_norm_bwd_desc(h=hl.unit_desc(x=x), w_pre=w, rstd_pre=r, dn=x, dw_pre=dw)
    hl.hilore_block_norm_bwd(desc, accumulate=True)
    assert (dw == 3.0).all()
    hl.hilore_block_norm_bwd(desc)
    assert (dw == 0.0).all()


def test_graph_of_forward_and_backward(hl):
    """Captured with a workspace, replayed three times with fresh inputs and eager work between."""
    rows, cols = 300, 896
    t = inputs(rows, cols, True, "channel", seed=20)
    res, y, w_post, gate, w_pre, dn, dh = (cuda(t[k]) for k in ("res", "y", "w_post", "gate", "w_pre", "dn", "dh"))

    def buffers():
        b = {k: torch.empty_like(res) for k in ("h", "n", "dres", "dy")}
        b.update({k: torch.empty(rows, device="cuda") for k in ("rstd_post", "rstd_pre")})
        b.update({k: torch.empty(cols, device="cuda") for k in ("dw_post", "dw_pre", "dgate")})
        return b

    def descs(b):
        f = hl.block_norm_desc(res, y=y, w_post=w_post, gate=gate, scale=0.5, w_pre=w_pre, h=b["h"], n=b["n"],
                               rstd_post=b["rstd_post"], rstd_pre=b["rstd_pre"])
        g = hl.block_norm_bwd_desc(h=hl.unit_desc(x=b["h"]), y=hl.unit_desc(x=y), w_post=w_post, gate=gate, scale=0.5,
                                   w_pre=w_pre, rstd_post=b["rstd_post"], rstd_pre=b["rstd_pre"], dn=dn, dh=dh,
                                   dres=b["dres"], dy=b["dy"], dw_post=b["dw_post"], dw_pre=b["dw_pre"], dgate=b["dgate"])
        return f, g

    a, b = buffers(), buffers()
    (fa, ga), (fb, gb) = descs(a), descs(b)
    ws = torch.empty(hl.hilore_block_norm_bwd_workspace_bytes(ga), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hl.hilore_block_norm(fa)
        hl.hilore_block_norm_bwd(ga, workspace=ws)
    for i in range(3):
        y.copy_(values(wl.rng(30 + i, 1), rows, cols))
        graph.replay()
        torch.cuda.synchronize()
        hl.hilore_block_norm(fb)
        hl.hilore_block_norm_bwd(gb)
        for k in a:
            assert torch.equal(a[k], b[k]), (i, k)
