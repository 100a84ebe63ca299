"""Argument checks of the layer operators' entry points and of their binding, on the host:
every invalid call is refused before the device is touched."""
import ctypes

import pytest
import torch

from paper_2609_33570_amd import hilore as E
from test_abi import FAKE, lib  # noqa: F401

OK, ARG, ALIGN, UNSUP, WORK = (E.HILORE_OK, E.HILORE_ERR_INVALID_ARG, E.HILORE_ERR_ALIGNMENT,
                               E.HILORE_ERR_UNSUPPORTED, E.HILORE_ERR_WORKSPACE)
NAN, INF = float("nan"), float("inf")


def make(cls, base, kw):
    d = cls()
    for k, v in {**base, **kw}.items():
        setattr(d, k, v)
    return d


def norm(lib, **kw):
    base = dict(res=FAKE, y=FAKE, w_post=FAKE, gate=FAKE, w_pre=FAKE, h=FAKE, n=FAKE, rows=4,
                cols=64, ld_res=64, ld_y=64, scale=1.0, eps=1e-6, gate_kind=E.GATE_CHANNEL)
    return lib.hilore_block_norm(ctypes.byref(make(E.hilore_block_norm_desc, base, kw)), None)


@pytest.mark.parametrize("want,kw", [
    (ARG, dict(rows=-1)), (ARG, dict(cols=-8)), (UNSUP, dict(cols=60)), (UNSUP, dict(cols=16392)),
    (UNSUP, dict(rows=1 << 31)), (ARG, dict(gate_kind=4)), (ARG, dict(gate_kind=-1)),
    (ARG, dict(gate_kind=0)), (ARG, dict(gate=None)), (ARG, dict(scale=NAN)), (ARG, dict(scale=INF)),
    (ARG, dict(eps=-1.0)), (ARG, dict(eps=NAN)), (ARG, dict(eps=INF)), (ARG, dict(y=None)),
    (ARG, dict(w_pre=None)), (ARG, dict(w_pre=None, n=None, rstd_pre=FAKE)),
    (ARG, dict(w_post=None, rstd_post=FAKE)), (ARG, dict(codes=FAKE)), (ARG, dict(code_scales=FAKE)),
    (ARG, dict(h=None, n=None)), (UNSUP, dict(codes=FAKE, code_scales=FAKE, cols=72, ld_res=72, ld_y=72)),
    (ARG, dict(res=None)), (ARG, dict(ld_res=56)), (ARG, dict(ld_y=56)), (ALIGN, dict(ld_res=68)),
    (ALIGN, dict(ld_y=68)), (ARG, dict(ld_res=72)), (ALIGN, dict(n=FAKE + 8)), (ALIGN, dict(w_pre=FAKE + 2)),
    (OK, dict(rows=0)), (OK, dict(cols=0)),
])
def test_block_norm(lib, want, kw):  # noqa: F811
    # h is res here: in place only where res is dense
    assert norm(lib, **kw) == want


def test_null_descriptors(lib):  # noqa: F811
    assert lib.hilore_block_norm(None, None) == ARG
    assert lib.hilore_block_norm_bwd(None, 0, 0, 0, None, 0, None) == ARG
    assert lib.hilore_int8_linear(None, None, 0, None) == ARG
    assert lib.hilore_int8_matmul(None, None, 0, None) == ARG
    assert lib.hilore_block_norm_bwd_workspace_bytes(None) == 0
    assert lib.hilore_int8_workspace_bytes(None, 1) == 0
    assert lib.hilore_grad_norm_workspace_bytes(None, 1) == 0


def saved(**kw):
    return make(E.hilore_unit_desc, dict(x=FAKE, rows=4, cols=256, ld=256), kw)


def norm_bwd(lib, code=0, block=128, ws=FAKE, ws_bytes=1 << 30, **kw):
    base = dict(h=saved(), y=saved(), w_post=FAKE, gate=FAKE, w_pre=FAKE, rstd_post=FAKE, rstd_pre=FAKE,
                dn=FAKE, dh=FAKE, dres=FAKE, dy=FAKE, dw_post=FAKE, dw_pre=FAKE, dgate=FAKE, rows=4,
                cols=256, ld_dn=256, scale=1.0, gate_kind=E.GATE_CHANNEL)
    d = make(E.hilore_block_norm_bwd_desc, base, kw)
    return lib.hilore_block_norm_bwd(ctypes.byref(d), code, block, 0, ws, ws_bytes, None)


LUNIT = dict(x=None, codes=FAKE, scales=FAKE)


@pytest.mark.parametrize("want,kw", [
    (ARG, dict(rows=-1)), (UNSUP, dict(cols=252)), (ARG, dict(gate_kind=7)), (ARG, dict(gate=None)),
    (ARG, dict(scale=NAN)), (ARG, dict(dn=None)), (ARG, dict(w_post=None)),
    (ARG, dict(gate=None, gate_kind=0)), (ARG, dict(dn=None, dh=None, w_pre=None, rstd_pre=None, dw_pre=None)),
    (ARG, dict(w_pre=None)), (ARG, dict(rstd_pre=None)), (ARG, dict(h=E.hilore_unit_desc())),
    (ARG, dict(ld_dn=248)), (ALIGN, dict(ld_dn=260)), (ARG, dict(rstd_post=None)),
    (ARG, dict(y=E.hilore_unit_desc())), (ARG, dict(y=saved(rows=5))), (ARG, dict(h=saved(cols=512, ld=512))),
    (ARG, dict(h=saved(ld=128))), (ALIGN, dict(h=saved(ld=260))), (ALIGN, dict(y=saved(x=FAKE + 4))),
    (ARG, dict(h=saved(x=None, codes=FAKE))), (ALIGN, dict(h=saved(**{**LUNIT, "codes": FAKE + 8}))),
    (ARG, dict(h=saved(**LUNIT), code=5)), (UNSUP, dict(h=saved(**LUNIT), block=48)),
    (ARG, dict(h=saved(**LUNIT), code=2, block=128)), (ALIGN, dict(dgate=FAKE + 4)),
    (UNSUP, dict(h=saved(cols=64, ld=64, **LUNIT), y=saved(cols=64, ld=64), cols=64, ld_dn=64)),
    (ARG, dict(ws=None)), (WORK, dict(ws_bytes=100)), (ALIGN, dict(ws=FAKE + 8)), (OK, dict(cols=0)),
])
def test_block_norm_bwd(lib, want, kw):  # noqa: F811
    assert norm_bwd(lib, **kw) == want


def product(lib, quantize, ws=FAKE, ws_bytes=1 << 30, **kw):
    base = dict(x=FAKE, a=FAKE, a_scales=FAKE, w=FAKE, w_scales=FAKE, out=FAKE, tokens=4, k=64, n=32, ldx=64, ldo=32)
    d = make(E.hilore_int8_desc, base, kw)
    return (lib.hilore_int8_linear if quantize else lib.hilore_int8_matmul)(ctypes.byref(d), ws, ws_bytes, None)


@pytest.mark.parametrize("quantize", [True, False])
def test_int8(lib, quantize):  # noqa: F811
    def f(**kw):
        return product(lib, quantize, **kw)

    for k in ("tokens", "k", "n"):
        assert f(**{k: -16}) == ARG
    assert f(k=72) == UNSUP and f(n=36) == UNSUP and f(k=131088, ldx=131088) == UNSUP
    assert f(n=1 << 26, ldo=1 << 26) == UNSUP and f(tokens=1 << 31) == UNSUP
    assert f(out=None) == ARG and f(ldo=24) == ARG and f(ldo=36) == ALIGN and f(w=None) == ARG
    assert f(out=FAKE + 2) == ALIGN and f(w=FAKE + 8) == ALIGN and f(w_scales=FAKE + 4) == ALIGN
    assert f(bias=FAKE + 2) == ALIGN
    if quantize:
        assert f(x=None) == ARG and f(ldx=56) == ARG and f(ldx=68) == ALIGN and f(factor=FAKE + 4) == ALIGN
        assert f(ws=None, ws_bytes=0) == ARG and f(ws_bytes=64) == WORK and f(ws=FAKE + 4) == ALIGN
    else:
        assert f(a=None) == ARG and f(a_scales=None) == ARG and f(a=FAKE + 4) == ALIGN
    assert f(tokens=0) == OK and f(n=0) == OK


def test_quantize_tokens(lib):  # noqa: F811
    def f(x=FAKE, factor=None, tokens=4, k=64, ldx=64, codes=FAKE, scales=FAKE):
        return lib.hilore_quantize_tokens(x, factor, tokens, k, ldx, codes, scales, None)

    assert f(tokens=-1) == ARG and f(k=-16) == ARG and f(k=72, ldx=72) == UNSUP
    assert f(tokens=1 << 31) == UNSUP
    assert f(x=None) == ARG and f(codes=None) == ARG and f(scales=None) == ARG and f(ldx=56) == ARG
    assert f(ldx=68) == ALIGN and f(x=FAKE + 8) == ALIGN and f(factor=FAKE + 4) == ALIGN
    assert f(tokens=0) == OK


def tensor(**kw):
    return make(E.hilore_adamw_tensor, dict(p=FAKE, grad=FAKE, m=FAKE, v=FAKE, n=1000, lr=1e-3), kw)


def adamw(lib, tensors, beta1=0.9, beta2=0.999, eps=1e-8, step=1, norm=None):
    arr = E.adamw_tensors(tensors)
    return lib.hilore_adamw(arr, len(arr), beta1, beta2, eps, step, norm, 0, None)


def test_adamw(lib):  # noqa: F811
    for kw in (dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0), dict(beta2=NAN), dict(eps=0.0), dict(eps=-1.0),
               dict(eps=1e-40), dict(eps=INF), dict(step=0)):
        assert adamw(lib, [tensor()], **kw) == ARG, kw
    assert adamw(lib, [tensor()], norm=FAKE + 2) == ALIGN
    for kw in (dict(p=None), dict(m=None), dict(v=None), dict(grad=None), dict(n=-1), dict(lr=NAN),
               dict(weight_decay=INF), dict(m_scales=FAKE), dict(v_scales=FAKE)):
        assert adamw(lib, [tensor(n=0), tensor(**kw)]) == ARG, kw
    for k in ("p", "p16", "grad", "m", "v"):
        assert adamw(lib, [tensor(**{k: FAKE + 8})]) == ALIGN, k
    assert adamw(lib, [tensor(m_scales=FAKE, v_scales=FAKE + 2)]) == ALIGN
    assert adamw(lib, [tensor(n=1 << 32)]) == UNSUP
    assert adamw(lib, []) == OK and adamw(lib, [tensor(n=0)]) == OK
    assert lib.hilore_adamw(None, 1, 0.9, 0.999, 1e-8, 1, None, 0, None) == ARG
    assert lib.hilore_adamw(None, -1, 0.9, 0.999, 1e-8, 1, None, 0, None) == ARG


def test_grad_norm(lib):  # noqa: F811
    arr = E.adamw_tensors([tensor(n=100000), tensor(n=0), tensor(n=3)])

    def f(max_norm=1.0, norm=FAKE, ws=FAKE, ws_bytes=1 << 20, n=3, arr=arr):
        return lib.hilore_grad_norm(arr, n, max_norm, norm, ws, ws_bytes, None)

    assert f(max_norm=0.0) == ARG and f(max_norm=NAN) == ARG and f(norm=None) == ARG and f(norm=FAKE + 2) == ALIGN
    assert f(ws=None) == ARG and f(ws=FAKE + 8) == ALIGN and f(ws_bytes=8) == WORK
    assert f(arr=None) == ARG and f(n=-1) == ARG
    assert f(arr=E.adamw_tensors([tensor(grad=None)]), n=1) == ARG
    assert f(arr=E.adamw_tensors([tensor(n=(1 << 32) - 1)] * 257), n=257) == UNSUP


def test_binding_refuses():
    """Shapes and types are checked before a pointer is taken (host tensors are refused after)."""
    x = torch.zeros(4, 64, dtype=torch.bfloat16)
    f = torch.zeros(4, 64)
    w = torch.zeros(64, dtype=torch.bfloat16)
    with pytest.raises(TypeError, match="res must be bfloat16"):
        E.block_norm_desc(f, h=x)
    with pytest.raises(ValueError, match="h must have shape"):
        E.block_norm_desc(x, h=torch.zeros(4, 32, dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="gate must be"):
        E._gate_kind(torch.zeros(4), 4, 64)
    with pytest.raises(ValueError, match="device tensors"):
        E.block_norm_desc(x, w_pre=w, n=x)
    with pytest.raises(ValueError, match="dgate without a gate"):
        E.block_norm_bwd_desc(dh=x, dgate=f)
    with pytest.raises(TypeError, match="w must be int8"):
        E.int8_desc(w=x, out=x, x=x)
    with pytest.raises(ValueError, match="out must have shape"):
        E.int8_desc(w=torch.zeros(8, 64, dtype=torch.int8), out=x, x=x)
    with pytest.raises(ValueError, match="needs x or a"):
        E.int8_desc(w=torch.zeros(64, 64, dtype=torch.int8), out=x)
    with pytest.raises(ValueError, match="p has 64 elements"):
        E.adamw_tensor(grad=f, m=f, v=f, p=torch.zeros(64))
    with pytest.raises(TypeError, match="m must be float8_e4m3fn or uint8"):
        E.adamw_tensor(grad=f, m=f, v=f, p=f, m_scales=torch.zeros(1), v_scales=torch.zeros(1))
    with pytest.raises(ValueError, match="m_scales needs 1"):
        c = torch.zeros(4, 64, dtype=torch.uint8)
        E.adamw_tensor(grad=f, m=c, v=c, p=f, m_scales=torch.zeros(2), v_scales=torch.zeros(1))
    with pytest.raises(ValueError, match="2 elements"):
        E.hilore_grad_norm(E.adamw_tensors([]), 1.0, torch.zeros(3))


def test_int8_output_size(lib):  # noqa: F811
    """More outputs than any memory holds: refused, and no workspace asked for."""
    for quantize in (True, False):
        assert product(lib, quantize, tokens=1 << 30, n=2048, ldo=2048) == UNSUP
        d = make(E.hilore_int8_desc, dict(tokens=1 << 30, n=2048, k=64), {})
        assert lib.hilore_int8_workspace_bytes(ctypes.byref(d), int(quantize)) == 0


@pytest.mark.parametrize("field", ["p", "p16", "grad", "m", "v", "m_scales", "v_scales"])
def test_adamw_addresses(lib, field):  # noqa: F811
    """Addresses travel as 48 bits: others are refused, wherever they stand."""
    kw = dict(p=FAKE, p16=FAKE, m_scales=FAKE, v_scales=FAKE) | {field: 1 << 48}
    assert adamw(lib, [tensor(), tensor(**kw)]) == UNSUP
