"""Argument checks of the entry points for heads, log-probabilities and losses and of their
binding, on the host: every invalid call is refused before the device is touched."""
import ctypes

import pytest
import torch

from paper_2609_33570_amd import hilore as E
from test_abi import FAKE, lib  # noqa: F401
from test_abi_layer import make, saved
from test_binding_keeps import Device

OK, ARG, ALIGN, UNSUP, WORK = (E.HILORE_OK, E.HILORE_ERR_INVALID_ARG, E.HILORE_ERR_ALIGNMENT,
                               E.HILORE_ERR_UNSUPPORTED, E.HILORE_ERR_WORKSPACE)
NAN, INF = float("nan"), float("inf")
BIG = 1 << 31


# ------------------------------------------------------------------- heads --
def heads(lib, **kw):  # noqa: F811
    base = dict(q=FAKE, k=FAKE, w_q=FAKE, w_k=FAKE, positions=FAKE, inv_freq=FAKE, q_out=FAKE + 4096, k_out=FAKE + 4096,
                tokens=4, ld_q=256, ld_k=128, q_token_stride=256, q_head_stride=64, k_token_stride=128, k_head_stride=64,
                heads_q=4, heads_k=2, dim=64, rotated=64, eps=1e-6, rope_scale=1.0, rotation=0)
    return lib.hilore_qk_norm_rope(ctypes.byref(make(E.hilore_qk_norm_rope_desc, base, kw)), None)


@pytest.mark.parametrize("want,kw", [
    (ARG, dict(tokens=-1)), (ARG, dict(heads_q=-1)), (ARG, dict(heads_k=-1)), (ARG, dict(dim=-16)), (ARG, dict(rotated=-16)),
    (ARG, dict(rotation=2)), (ARG, dict(rotation=-1)), (ARG, dict(eps=-1.0)), (ARG, dict(eps=NAN)), (ARG, dict(eps=INF)),
    (ARG, dict(rope_scale=INF)), (ARG, dict(rotated=80)), (UNSUP, dict(dim=72)), (UNSUP, dict(dim=528)),
    (UNSUP, dict(rotated=24)), (UNSUP, dict(tokens=BIG)), (UNSUP, dict(heads_q=65536, heads_k=1)),
    (ARG, dict(q=None)), (ARG, dict(q_out=None)), (ARG, dict(k=None)), (ARG, dict(k_out=None)), (ARG, dict(inv_freq=None)),
    (ARG, dict(ld_q=248)), (ARG, dict(ld_k=120)), (ALIGN, dict(ld_q=260)), (ALIGN, dict(ld_k=132)),
    (ARG, dict(q_token_stride=0)), (ARG, dict(q_head_stride=0)), (ARG, dict(q_token_stride=-256)),
    (ARG, dict(q_token_stride=248)),   # the tokens' heads would overlap
    (ARG, dict(q_token_stride=64, q_head_stride=248)),
    (ARG, dict(tokens=BIG - 1, q_token_stride=1 << 40, q_head_stride=1 << 40)),  # their product is past 64 bits
    (ARG, dict(q_token_stride=1 << 41)), (ARG, dict(ld_q=1 << 41)), (ALIGN, dict(q_token_stride=260)), (ALIGN, dict(k_head_stride=68, k_token_stride=136)),
    (ARG, dict(q_out=FAKE, ld_q=320)),  # in place only with the rows' strides
    (ARG, dict(k_out=FAKE, k_token_stride=64, k_head_stride=256)),
    (ALIGN, dict(q=FAKE + 8)), (ALIGN, dict(k_out=FAKE + 8)), (ALIGN, dict(w_q=FAKE + 2)), (ALIGN, dict(positions=FAKE + 4)),
    (ALIGN, dict(inv_freq=FAKE + 2)), (OK, dict(tokens=0)), (OK, dict(heads_q=0, heads_k=0)), (OK, dict(tokens=0, q=None)),
    (OK, dict(dim=0, rotated=0)),
])
def test_heads(lib, want, kw):  # noqa: F811
    assert heads(lib, **kw) == want


def heads_bwd(lib, code=0, block=64, ws=FAKE, ws_bytes=1 << 30, **kw):  # noqa: F811
    base = dict(q=saved(), k=saved(cols=128, ld=128), w_q=FAKE, w_k=FAKE, positions=FAKE, inv_freq=FAKE, dq=FAKE, dk=FAKE,
                dq_in=FAKE + 4096, dk_in=FAKE + 4096, dw_q=FAKE, dw_k=FAKE, tokens=4, q_token_stride=256, q_head_stride=64,
                k_token_stride=128, k_head_stride=64, ld_dq=256, ld_dk=128, heads_q=4, heads_k=2, dim=64, rotated=64,
                eps=1e-6, rope_scale=1.0, rotation=0)
    d = make(E.hilore_qk_norm_rope_bwd_desc, base, kw)
    return lib.hilore_qk_norm_rope_bwd(ctypes.byref(d), code, block, 0, ws, ws_bytes, None)


LUNIT = dict(x=None, codes=FAKE, scales=FAKE)


@pytest.mark.parametrize("want,kw", [
    (ARG, dict(tokens=-1)), (UNSUP, dict(dim=72)), (ARG, dict(dq=None)), (ARG, dict(dk=None)), (ARG, dict(w_q=None)),
    (ARG, dict(w_k=None)), (ARG, dict(heads_k=0)), (ARG, dict(q=E.hilore_unit_desc())), (ARG, dict(q=saved(rows=5))),
    (ARG, dict(k=saved())), (ARG, dict(q=saved(ld=128))), (ALIGN, dict(q=saved(ld=260))), (ALIGN, dict(q=saved(x=FAKE + 4))),
    (ARG, dict(q=saved(x=None, codes=FAKE))), (ALIGN, dict(q=saved(**{**LUNIT, "codes": FAKE + 8}))),
    (ARG, dict(q=saved(**LUNIT), code=5)), (UNSUP, dict(q=saved(**LUNIT), block=48)),
    (UNSUP, dict(q=saved(cols=448, **LUNIT), heads_q=7, ld_dq=448, block=256)), (ARG, dict(q=saved(**LUNIT), code=2)),
    (ARG, dict(ld_dq=248)), (ALIGN, dict(ld_dq=260)), (ARG, dict(q_token_stride=-8)), (ALIGN, dict(q_head_stride=4)),
    (ARG, dict(dq_in=FAKE, ld_dq=320)), (ARG, dict(inv_freq=None)), (ALIGN, dict(dw_q=FAKE + 4)), (ALIGN, dict(dq=FAKE + 2)),
    (ALIGN, dict(positions=FAKE + 4)), (ARG, dict(ws=None)), (ALIGN, dict(ws=FAKE + 4)), (WORK, dict(ws_bytes=64)),
    (OK, dict(heads_q=0, heads_k=0, dw_q=None, dw_k=None)), (OK, dict(tokens=0, dw_q=None, dw_k=None, dq=None, dk=None)),
])
def test_heads_bwd(lib, want, kw):  # noqa: F811
    assert heads_bwd(lib, **kw) == want


# ---------------------------------------------------------------- logprobs --
def logprobs(lib, ws=FAKE, ws_bytes=1 << 40, **kw):  # noqa: F811
    base = dict(logits=FAKE, targets=FAKE, logp=FAKE, entropy=FAKE, row_max=FAKE, log_sum=FAKE, rows=4, vocab=100000,
                ld=100000, scale=1.0, logits_f32=0)
    return lib.hilore_token_logprobs(ctypes.byref(make(E.hilore_token_logprobs_desc, base, kw)), ws, ws_bytes, None)


LOGITS = [
    (ARG, dict(rows=-1)), (ARG, dict(vocab=-1)), (ARG, dict(vocab=0)), (UNSUP, dict(rows=BIG)),
    (UNSUP, dict(vocab=1 << 28, ld=1 << 28)), (ARG, dict(scale=0.0)), (ARG, dict(scale=-1.0)), (ARG, dict(scale=NAN)),
    (ARG, dict(scale=INF)), (ARG, dict(scale=1e-40)), (ARG, dict(logits=None)), (ARG, dict(targets=None)),
    (ARG, dict(ld=99999)), (ALIGN, dict(logits=FAKE + 1)), (ALIGN, dict(logits=FAKE + 2, logits_f32=1)),
    (ALIGN, dict(targets=FAKE + 4)), (OK, dict(rows=0)), (OK, dict(rows=0, vocab=0, logits=None)),
]


@pytest.mark.parametrize("want,kw", LOGITS + [
    (ALIGN, dict(logp=FAKE + 2)), (ALIGN, dict(entropy=FAKE + 2)), (ALIGN, dict(row_max=FAKE + 2)),
    (ALIGN, dict(log_sum=FAKE + 2)), (ARG, dict(ws=None)), (ALIGN, dict(ws=FAKE + 8)), (WORK, dict(ws_bytes=16)),
])
def test_logprobs(lib, want, kw):  # noqa: F811
    assert logprobs(lib, **kw) == want


@pytest.mark.parametrize("want,kw", LOGITS + [
    (ARG, dict(row_max=None)), (ARG, dict(log_sum=None)), (ARG, dict(dlogp=None)), (ARG, dict(dlogits=None)),
    (ARG, dict(entropy=None)), (ARG, dict(ld_out=99999)), (ARG, dict(dlogits=FAKE, ld_out=100008)),
    (ALIGN, dict(dlogits=FAKE + 1)), (ALIGN, dict(dlogp=FAKE + 1)), (ALIGN, dict(dentropy=FAKE + 1)),
])
def test_logprobs_bwd(lib, want, kw):  # noqa: F811
    base = dict(logits=FAKE, targets=FAKE, row_max=FAKE, log_sum=FAKE, entropy=FAKE, dlogp=FAKE, dentropy=FAKE, dlogits=FAKE,
                rows=4, vocab=100000, ld=100000, ld_out=100000, scale=1.0, logits_f32=0)
    assert lib.hilore_token_logprobs_bwd(ctypes.byref(make(E.hilore_token_logprobs_bwd_desc, base, kw)), None) == want


# ------------------------------------------------------------------ losses --
SEQUENCES = [
    (ARG, dict(n_tokens=-1)), (ARG, dict(sequences=-1)), (ARG, dict(n_norm=NAN)), (ARG, dict(n_norm=INF)),
    (UNSUP, dict(n_tokens=BIG, offsets=FAKE)), (UNSUP, dict(sequences=BIG, offsets=FAKE)), (ARG, dict(n_tokens=33)),
    (ARG, dict(sequences=0)), (ARG, dict(logp=None)), (ALIGN, dict(offsets=FAKE + 4)), (ALIGN, dict(logp=FAKE + 2)),
    (ALIGN, dict(dlogp=FAKE + 1)), (ALIGN, dict(stats=FAKE + 2)), (ARG, dict(ws=None)), (ALIGN, dict(ws=FAKE + 4)),
    (WORK, dict(ws_bytes=256)),
]


@pytest.mark.parametrize("want,kw", SEQUENCES + [
    (ARG, dict(clip_low=0.0)), (ARG, dict(clip_low=1.0)), (ARG, dict(clip_low=NAN)), (ARG, dict(clip_high=0.0)),
    (ARG, dict(clip_high=INF)), (ARG, dict(dual_clip=-1.0)), (ARG, dict(dual_clip=1.0)), (ARG, dict(dual_clip=NAN)),
    (ARG, dict(beta=NAN)), (ARG, dict(entropy_weight=INF)), (ARG, dict(ratio=2)), (ARG, dict(kl=4)), (ARG, dict(kl=-1)),
    (ARG, dict(mean=2)), (UNSUP, dict(ratio=1, adv_per_token=1)), (ARG, dict(logp_old=None)), (ARG, dict(adv=None)),
    (ARG, dict(logp_ref=None)), (ARG, dict(kl=0)), (ARG, dict(entropy=None)), (ARG, dict(entropy=None, entropy_weight=0.0)),
    (ALIGN, dict(adv=FAKE + 2)), (ALIGN, dict(dentropy=FAKE + 2)), (ALIGN, dict(token_loss=FAKE + 2)),
])
def test_policy(lib, want, kw):  # noqa: F811
    kw = dict(kw)
    ws, ws_bytes = kw.pop("ws", FAKE), kw.pop("ws_bytes", 1 << 40)
    base = dict(logp=FAKE, logp_old=FAKE, logp_ref=FAKE, entropy=FAKE, adv=FAKE, mask=FAKE + 1, dlogp=FAKE, dentropy=FAKE,
                token_loss=FAKE, flags=FAKE + 3, stats=FAKE, n_tokens=32, sequences=4, clip_low=0.2, clip_high=0.2, beta=0.1,
                entropy_weight=0.1, kl=3)
    d = make(E.hilore_policy_loss_desc, base, kw)
    assert lib.hilore_policy_loss(ctypes.byref(d), ws, ws_bytes, None) == want


@pytest.mark.parametrize("want,kw", SEQUENCES + [
    (ARG, dict(beta=0.0)), (ARG, dict(beta=-1.0)), (ARG, dict(beta=INF)), (ARG, dict(margin=NAN)), (ARG, dict(loss=3)),
    (ARG, dict(loss=-1)), (ARG, dict(label_smoothing=0.6)), (ARG, dict(label_smoothing=-0.1)), (ARG, dict(label_smoothing=NAN)),
    (ARG, dict(label_smoothing=0.1, loss=1)), (ARG, dict(chosen=FAKE)), (ARG, dict(rejected=FAKE)), (ARG, dict(pairs=3)),
    (ARG, dict(pairs=-1)), (UNSUP, dict(pairs=BIG, chosen=FAKE, rejected=FAKE)),
    (UNSUP, dict(pairs=1 << 20, chosen=FAKE, rejected=FAKE, sequences=1 << 17, n_tokens=1 << 17)),
    (ALIGN, dict(chosen=FAKE + 2, rejected=FAKE)), (ALIGN, dict(rewards=FAKE + 2)), (ALIGN, dict(pair_loss=FAKE + 2)),
    (ALIGN, dict(logp_ref=FAKE + 2)),
])
def test_preference(lib, want, kw):  # noqa: F811
    kw = dict(kw)
    ws, ws_bytes = kw.pop("ws", FAKE), kw.pop("ws_bytes", 1 << 40)
    base = dict(logp=FAKE, logp_ref=FAKE, mask=FAKE + 1, dlogp=FAKE, rewards=FAKE, pair_loss=FAKE, stats=FAKE, n_tokens=32,
                sequences=4, pairs=2, beta=0.1)
    d = make(E.hilore_preference_loss_desc, base, kw)
    assert lib.hilore_preference_loss(ctypes.byref(d), ws, ws_bytes, None) == want


@pytest.mark.parametrize("scale,want", [(2.0 ** -126, OK), (2.0 ** 127, OK), (1.01 * 2.0 ** 127, ARG), (3.4e38, ARG), (2.0 ** -127, ARG)])
def test_logprobs_scales(lib, scale, want):  # noqa: F811
    for name, ws in (("token_logprobs", (None, 0)), ("token_logprobs_bwd", ())):
        d = getattr(E, f"hilore_{name}_desc")()
        d.vocab, d.ld, d.scale = 8, 8, scale
        assert getattr(lib, f"hilore_{name}")(ctypes.byref(d), *ws, None) == want


@pytest.mark.parametrize("block", [-1, 0, 3, 1 << 30, (1 << 30) + 1, (1 << 31) - 1])
def test_heads_bwd_without_codes_takes_any_block(lib, block):  # noqa: F811
    assert heads_bwd(lib, block=block, tokens=0, dw_q=None, dw_k=None) == OK


def test_null_descriptors(lib):  # noqa: F811
    assert lib.hilore_qk_norm_rope(None, None) == ARG
    assert lib.hilore_qk_norm_rope_bwd(None, 0, 0, 0, None, 0, None) == ARG
    assert lib.hilore_token_logprobs(None, None, 0, None) == ARG
    assert lib.hilore_token_logprobs_bwd(None, None) == ARG
    assert lib.hilore_policy_loss(None, None, 0, None) == ARG
    assert lib.hilore_preference_loss(None, None, 0, None) == ARG
    for f in ("qk_norm_rope_bwd", "token_logprobs", "policy_loss", "preference_loss"):
        assert getattr(lib, f"hilore_{f}_workspace_bytes")(None) == 0


# ----------------------------------------------------------------- binding --
def f(*shape):
    return Device(*shape, dtype=torch.float32)


def i(*shape):
    return Device(*shape, dtype=torch.int64)


def b(*shape):
    return Device(*shape)


class View(Device):
    def __init__(self, t):
        self.t = t


@pytest.mark.parametrize("error,make_desc", [
    (TypeError, lambda: E.qk_norm_rope_desc(q=f(3, 64), q_out=b(3, 2, 32))),
    (ValueError, lambda: E.qk_norm_rope_desc(q=b(3, 96), q_out=b(3, 2, 32))),
    (ValueError, lambda: E.qk_norm_rope_desc(q=b(3, 64), q_out=b(3, 64))),
    (ValueError, lambda: E.qk_norm_rope_desc(q=b(3, 64), q_out=b(3, 2, 32), k=b(3, 32))),
    (ValueError, lambda: E.qk_norm_rope_desc(q=b(3, 64), q_out=b(3, 2, 32), k=b(4, 32), k_out=b(4, 1, 32))),
    (ValueError, lambda: E.qk_norm_rope_desc(q=b(3, 64), q_out=b(3, 2, 32), w_q=b(64))),
    (TypeError, lambda: E.qk_norm_rope_desc(q=b(3, 64), q_out=b(3, 2, 32), positions=Device(3, dtype=torch.int32))),
    (ValueError, lambda: E.qk_norm_rope_desc(q=b(3, 64), q_out=b(3, 2, 32), positions=i(4))),
    (ValueError, lambda: E.qk_norm_rope_desc(q=b(3, 64), q_out=b(3, 2, 32), rotation="other")),
    (ValueError, lambda: E.qk_norm_rope_desc(q=b(3, 64), q_out=View(torch.zeros(3, 32, 2, dtype=torch.bfloat16).transpose(1, 2)))),
    (ValueError, lambda: E.qk_norm_rope_desc(q=View(torch.zeros(2, 3, 32, dtype=torch.bfloat16).transpose(0, 1)), q_out=b(3, 2, 32))),
    (ValueError, lambda: E.qk_norm_rope_bwd_desc(dq=None)),
    (ValueError, lambda: E.qk_norm_rope_bwd_desc(dq=b(3, 2, 32), dw_q=f(64))),
    (ValueError, lambda: E.qk_norm_rope_bwd_desc(dq=b(3, 2, 32), dk_in=b(3, 32))),
    (ValueError, lambda: E.token_logprobs_desc(f(3, 9), i(4))),
    (TypeError, lambda: E.token_logprobs_desc(Device(3, 9, dtype=torch.float16), i(3))),
    (TypeError, lambda: E.token_logprobs_desc(f(3, 9), Device(3, dtype=torch.int32))),
    (ValueError, lambda: E.token_logprobs_desc(f(3, 9), i(3), logp=f(3, 1))),
    (ValueError, lambda: E.token_logprobs_desc(View(torch.zeros(9, 3).t()), i(3))),
    (TypeError, lambda: E.token_logprobs_bwd_desc(f(3, 9), i(3), f(3), f(3), f(3), b(3, 9))),
    (ValueError, lambda: E.policy_loss_desc(f(12), f(11), f(3), sequences=3)),
    (ValueError, lambda: E.policy_loss_desc(f(12), f(12), f(4), sequences=3)),
    (ValueError, lambda: E.policy_loss_desc(f(12), f(12), f(3))),
    (ValueError, lambda: E.policy_loss_desc(f(12), f(12), f(3), offsets=i(4), sequences=2)),
    (ValueError, lambda: E.policy_loss_desc(f(3, 4), f(3, 4), f(3), stats=f(6))),
    (TypeError, lambda: E.policy_loss_desc(f(3, 4), f(3, 4), f(3), mask=f(12))),
    (ValueError, lambda: E.policy_loss_desc(f(3, 4), f(3, 4), f(3), ratio="word")),
    (ValueError, lambda: E.preference_loss_desc(f(4, 4), chosen=Device(2, dtype=torch.int32))),
    (ValueError, lambda: E.preference_loss_desc(f(4, 4), pair_loss=f(3))),
    (ValueError, lambda: E.preference_loss_desc(f(4, 4), loss="other")),
    (TypeError, lambda: E.preference_loss_desc(f(4, 4), chosen=i(2), rejected=i(2))),
])
def test_binding_refuses(error, make_desc):
    with pytest.raises(error):
        make_desc()


def test_host_tensors_are_refused():
    with pytest.raises(ValueError, match="device tensors"):
        E.token_logprobs_desc(torch.zeros(3, 9), torch.zeros(3, dtype=torch.int64))


def test_strides_of_descriptors():
    rows = View(torch.zeros(5, 5 * 32 + 16, dtype=torch.bfloat16)[:, :64])
    heads_first = View(torch.zeros(2, 5, 32, dtype=torch.bfloat16).transpose(0, 1))
    d = E.qk_norm_rope_desc(q=rows, q_out=heads_first, inv_freq=f(8))
    assert (d.tokens, d.heads_q, d.heads_k, d.dim, d.rotated) == (5, 2, 0, 32, 16)
    assert (d.ld_q, d.q_token_stride, d.q_head_stride) == (176, 32, 160)
    one = E.qk_norm_rope_desc(q=b(1, 64), q_out=b(1, 2, 32))
    assert (one.ld_q, one.q_token_stride, one.q_head_stride) == (64, 64, 32)
    t = E.token_logprobs_desc(View(torch.zeros(4, 11)[:, :7]), i(4))
    assert (t.rows, t.vocab, t.ld, t.logits_f32) == (4, 7, 11, 1)
    p = E.policy_loss_desc(f(3, 4), f(3, 4), f(12))
    assert (p.n_tokens, p.sequences, p.adv_per_token) == (12, 3, 1)
    assert E.preference_loss_desc(f(12), offsets=i(6)).pairs == 2


class OnDevice(Device):
    """A host tensor that says it is on device `n`."""

    def __init__(self, n, *shape, dtype=torch.float32):
        super().__init__(*shape, dtype=dtype)
        self.device = torch.device("cuda", n)


def test_another_device_is_refused(monkeypatch):
    with pytest.raises(ValueError, match="several devices"):
        E.token_logprobs_desc(OnDevice(0, 3, 9), OnDevice(1, 3, dtype=torch.int64))
    desc = E.token_logprobs_desc(OnDevice(1, 3, 9), OnDevice(1, 3, dtype=torch.int64))
    monkeypatch.setattr(E, "_device_now", lambda: 0)
    with pytest.raises(ValueError, match="device 1"):
        E.hilore_token_logprobs(desc)


def test_descriptors_keep_their_tensors():
    import gc
    import weakref

    t = {"q": b(4, 64), "q_out": b(4, 2, 32), "w": b(32), "codes": Device(4, 64, dtype=torch.uint8), "scales": f(4, 2)}
    refs = {k: weakref.ref(v) for k, v in t.items()}
    d = [E.qk_norm_rope_desc(q=t["q"], q_out=t["q_out"], w_q=t["w"]),
         E.qk_norm_rope_bwd_desc(dq=t["q_out"], q=E.unit_desc(codes=t["codes"], scales=t["scales"]), w_q=t["w"])]
    del t
    gc.collect()
    assert all(r() is not None for r in refs.values())
    del d
    gc.collect()
    assert all(r() is None for r in refs.values())
