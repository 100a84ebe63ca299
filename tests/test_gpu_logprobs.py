"""hilore_token_logprobs and its backward against 64 bits.

Tolerances.  A term of S is exp2 of d = c (z - m) with three roundings (c, the difference, the
product): off by 3 |d| 2^-24 ln 2 and half a step of its own; the mean of |d| under the softmax is at most
log2(vocab) <= 18, so S is off by 2^-18.5 for that, and by its summation: 64 terms a lane and batch
factors, 6 steps over lanes, as many joins as segments and waves, under 130 roundings, 2^-17 at worst.  So
S is off by less than 2^-16 of its other terms, logp by (1 - p) of that and 2^-21 of itself (products and
logarithm).  The entropy is formed from S and the mean of d, which has the same relative error:
2^-16 (2 + log vocab).  Backward starts from the stored row_max and log_sum; l = scale (z - m) - log S
is off by 2^-22 (|l| + |log S| + 1), p relatively by that, and bf16 outputs are rounded once, 2^-8.
"""
import math

import pytest
import torch

import actor_reference as R

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
LOWEST = {BF16: torch.finfo(BF16).min, F32: torch.finfo(F32).min}


def logits(rows, vocab, dtype, seed, pad=0):
    """[rows, vocab] in rows `pad` apart, peaked ones among them, and targets of all kinds."""
    g = torch.Generator().manual_seed(seed)
    z = torch.randn(rows, vocab + pad, generator=g) * (0.5 + 4.0 * torch.rand(rows, 1, generator=g))
    t = torch.randint(0, vocab, (rows,), generator=g)
    for r in range(0, rows, 3):
        z[r, int(t[r])] += 20.0 * float(torch.rand(1, generator=g))
    t[4::7] = -1
    t[5::11] = -(1 << 40)
    return z.to(dtype)[:, :vocab], t


def device(z):
    """The same strides on the device."""
    buf = torch.zeros(z.shape[0], z.stride(0) if z.shape[0] > 1 else z.shape[1], dtype=z.dtype, device="cuda")
    view = buf[:, :z.shape[1]]
    view.copy_(z)
    return view


def forward(hl, z, t, scale, entropy=True, workspace=None):
    out = {k: torch.full((z.shape[0],), 5.0, device="cuda") for k in ("logp", "entropy", "row_max", "log_sum")}
    if not entropy:
        del out["entropy"]
    hl.hilore_token_logprobs(hl.token_logprobs_desc(z, t, scale=scale, **out), workspace=workspace)
    return out


def check_forward(out, z, t, scale):
    want = R.token_logprobs(z.double(), t, scale)
    got = {k: v.cpu().double() for k, v in out.items()}
    assert torch.equal(got["row_max"], want["row_max"])
    vocab = z.shape[1]
    rest = -torch.expm1(want["logp"])
    for k, limit in (("logp", 2.0 ** -16 * rest + 2.0 ** -21 * want["logp"].abs()),
                     ("log_sum", 2.0 ** -16 * (1.0 - torch.exp(-want["log_sum"])) + 2.0 ** -22),
                     ("entropy", torch.full_like(rest, 2.0 ** -16 * (2.0 + math.log(vocab))))):
        if k in got:
            off = (got[k] - want[k]).abs()
            assert (off <= limit).all(), (k, float((off - limit).max()), int((off - limit).argmax()))
    return want


SIZES = [  # rows, vocab, pad: one token, odd vocabularies, one segment and several, split rows and whole ones
    (1, 1, 0), (3, 2, 0), (1, 131072, 0), (2, 50021, 0), (5, 50021, 3), (7, 7, 1), (64, 1000, 0), (13, 16384, 0), (13, 16385, 0),
    (9, 16383, 9), (11, 32768 + 5, 0), (1030, 1003, 0), (1100, 20001, 0), (1024, 257, 2), (30, 8191, 0), (4, 262144, 0),
]


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("rows,vocab,pad", SIZES)
@pytest.mark.parametrize("scale,entropy", [(1.0, True), (1.25, False), (0.6, True)])
def test_forward(hl, rows, vocab, pad, dtype, scale, entropy):
    z, t = logits(rows, vocab, dtype, rows + vocab, pad)
    out = forward(hl, device(z), t.cuda(), float(torch.tensor(scale)), entropy)
    check_forward(out, z, t, float(torch.tensor(scale, dtype=F32)))


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("rows,vocab,pad", SIZES)
@pytest.mark.parametrize("scale,bonus", [(1.0, False), (1.25, True)])
def test_backward(hl, rows, vocab, pad, dtype, scale, bonus):
    z, t = logits(rows, vocab, dtype, rows + vocab, pad)
    zd, td = device(z), t.cuda()
    o = forward(hl, zd, td, scale)
    g = torch.Generator().manual_seed(5)
    dlogp, dent = torch.randn(rows, generator=g), 0.1 * torch.randn(rows, generator=g)
    dlogp[1::4] = 0.0
    dent[1::8] = 0.0
    dlogp[4::7] = float("nan")  # rows without a token: whatever stands there
    # dense, and with rows that begin elsewhere than the logits'
    for extra in (0, 5):
        buf = torch.full((rows, vocab + extra), 3.0, dtype=dtype, device="cuda")
        hl.hilore_token_logprobs_bwd(hl.token_logprobs_bwd_desc(
            zd, td, o["row_max"], o["log_sum"], dlogp.cuda(), buf[:, :vocab], entropy=o["entropy"],
            dentropy=dent.cuda() if bonus else None, scale=scale))
        m, s, e = (o[k].cpu().double() for k in ("row_max", "log_sum", "entropy"))
        zz = z.double()
        want = R.token_logprobs_bwd(zz, t, scale, m, s, e, torch.nan_to_num(dlogp).double(), dent.double() if bonus else None)
        l = scale * (zz - m[:, None]) - s[:, None]
        h = dent.abs().double()[:, None] * (l.abs().clamp(max=200.0) + e.abs()[:, None] + 1.0) if bonus else 0.0
        size = scale * l.exp() * (torch.nan_to_num(dlogp).abs().double()[:, None] + h)
        # the chosen token's: g (1 - p) with a relative 2^-21 of its own
        off = (buf[:, :vocab].cpu().double() - want).abs()
        half = 2.0 ** -8 if dtype == BF16 else 2.0 ** -21
        limit = half * want.abs() + 2.0 ** -22 * size * (4.0 + l.abs().clamp(max=200.0) + s.abs()[:, None]) + 1e-37
        live = t >= 0
        assert (off[live] <= limit[live]).all(), (extra, float((off - limit)[live].max()))
        assert not buf[:, :vocab][~live.cuda()].any()
        assert bool((buf[:, vocab:] == 3.0).all())


def test_backward_in_place(hl):
    z, t = logits(40, 5003, BF16, 2, 6)
    zd, td = device(z), t.cuda()
    o = forward(hl, zd, td, 1.0)
    g = torch.randn(40).cuda()
    args = (td, o["row_max"], o["log_sum"], g)
    out = torch.empty(40, 5003, dtype=BF16, device="cuda")
    hl.hilore_token_logprobs_bwd(hl.token_logprobs_bwd_desc(zd, *args, out))
    hl.hilore_token_logprobs_bwd(hl.token_logprobs_bwd_desc(zd, *args, zd))
    assert torch.equal(out, zd)


def test_forward_and_backward_agree_with_differences(hl):
    """The forward kernel's logp at two points around z moves as the backward kernel says."""
    g = torch.Generator().manual_seed(3)
    z, t = torch.randn(6, 997, generator=g), torch.randint(0, 997, (6,), generator=g)
    step, h = torch.randn(6, 997, generator=g), 2.0 ** -6
    td, scale = t.cuda(), 1.5
    o = forward(hl, z.cuda(), td, scale)
    d, ones = torch.empty(6, 997, device="cuda"), torch.ones(6, device="cuda")
    hl.hilore_token_logprobs_bwd(hl.token_logprobs_bwd_desc(z.cuda(), td, o["row_max"], o["log_sum"], ones, d, entropy=o["entropy"],
                                                            dentropy=ones, scale=scale))
    up, down = (forward(hl, (z + s * h * step).cuda(), td, scale) for s in (1, -1))
    quotient = ((up["logp"] + up["entropy"]) - (down["logp"] + down["entropy"])).cpu().double() / (2 * h)
    along = (d.cpu().double() * step.double()).sum(1)
    # third derivatives over 6 times h^2 with steps of size 1 under weights that sum to 1 (about 10 at
    # scale 1.5), and 2^-16 (2 + log 997) of each value over 2 h
    assert ((quotient - along).abs() <= 10 * h * h + 4 * 2.0 ** -16 * 9 / (2 * h)).all(), (quotient - along).abs().max()


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("vocab", [40, 40000])
@pytest.mark.parametrize("scale", [1.0, 2.0])
def test_masked_columns(hl, dtype, vocab, scale):
    """-inf and the type's lowest value in masked places, rows that a mask leaves one column or none,
    infinities and NaN."""
    g = torch.Generator().manual_seed(4)
    z = torch.randn(12, vocab, generator=g)
    t = torch.full((12,), 7)
    z[0, 10:] = -math.inf
    z[1, 10:] = LOWEST[dtype]
    z[2] = -math.inf
    z[2, 7] = -3.0                   # one column left, the chosen one
    z[3] = LOWEST[dtype]
    z[3, 7] = 2.0
    z[4] = -math.inf
    z[4, 9] = 1.0                    # one left, another one
    z[5] = LOWEST[dtype]             # all the same
    z[6] = -math.inf                 # none
    z[7, 5] = math.inf
    z[8, 5] = math.nan
    z[9, 7] = math.nan
    z[10, 7] = -math.inf             # the chosen one is masked
    z[11, :] = 0.0
    z = z.to(dtype)
    o = forward(hl, z.cuda(), t.cuda(), scale)
    good = [0, 1, 2, 3, 5, 11]
    check_forward({k: v[good] for k, v in o.items()}, z[good], t[good], scale)
    assert float(o["logp"][2]) == 0.0 and float(o["entropy"][2]) == 0.0
    assert float(o["logp"][5]) == pytest.approx(-math.log(vocab), rel=1e-5)
    for r in (4, 10):
        assert float(o["logp"][r]) == -math.inf
        assert math.isfinite(float(o["entropy"][r])) and math.isfinite(float(o["log_sum"][r]))
    for r in (6, 7, 8, 9):
        assert math.isnan(float(o["logp"][r])) and math.isnan(float(o["entropy"][r])), r
    assert float(o["row_max"][6]) == -math.inf
    d, one = torch.empty(12, vocab, dtype=dtype, device="cuda"), torch.ones(12, device="cuda")
    hl.hilore_token_logprobs_bwd(hl.token_logprobs_bwd_desc(z.cuda(), t.cuda(), o["row_max"], o["log_sum"], one, d, entropy=o["entropy"],
                                                            dentropy=one, scale=scale))
    d = d.cpu().double()
    for r in (0, 1, 2, 3, 4, 5, 10, 11):
        assert torch.isfinite(d[r]).all(), r
    assert not d[0, 10:].any() and not d[1, 10:].any() and not d[2].any() and not d[3].any()
    assert float(d[4, 7]) == scale and float(d[10, 7]) == scale  # p = 0: the whole gradient
    for r in (6, 7, 8, 9):
        assert torch.isnan(d[r]).any(), r
    # rows without a gradient are not read
    none = torch.zeros(12, device="cuda")
    d = torch.ones(12, vocab, dtype=dtype, device="cuda")
    hl.hilore_token_logprobs_bwd(hl.token_logprobs_bwd_desc(z.cuda(), t.cuda(), o["row_max"], o["log_sum"], none, d))
    assert not d.any()


def test_targets_out_of_range(hl):
    z = torch.randn(3, 1000)
    t = torch.tensor([1000, 5, 1 << 60])
    o = forward(hl, z.cuda(), t.cuda(), 1.0)
    assert torch.isnan(o["logp"]).tolist() == [True, False, True]
    assert (o["log_sum"].cpu() - (torch.logsumexp(z, 1) - z.amax(1))).abs().max() < 1e-4
    d = torch.zeros(3, 1000, device="cuda")
    g = torch.tensor([0.0, 0.0, 1.0], device="cuda")
    hl.hilore_token_logprobs_bwd(hl.token_logprobs_bwd_desc(z.cuda(), t.cuda(), o["row_max"], o["log_sum"], g, d))
    assert torch.isnan(d[0]).all() and not d[1].any() and torch.isnan(d[2]).all()


def test_confident_tokens_keep_their_precision(hl):
    """logp of a token that is nearly sure: far below fp32's step at 1."""
    z = torch.full((3, 50000), -20.0)
    z[0, 3], z[1, 3], z[2, 3] = 0.0, 5.0, 15.0
    o = forward(hl, z.cuda(), torch.tensor([3, 3, 3]).cuda(), 1.0)
    want = -torch.log1p(49999.0 * torch.exp(torch.tensor([-20.0, -25.0, -35.0], dtype=torch.float64)))
    assert ((o["logp"].cpu().double() - want) / want).abs().max() < 2.0 ** -16
    d, g = torch.empty(3, 50000, device="cuda"), torch.ones(3, device="cuda")
    hl.hilore_token_logprobs_bwd(hl.token_logprobs_bwd_desc(z.cuda(), torch.tensor([3, 3, 3]).cuda(), o["row_max"], o["log_sum"], g, d))
    assert ((d[:, 3].cpu().double() + torch.expm1(want)) / want).abs().max() < 2.0 ** -15


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("vocab", [40003, 100003])
def test_a_rows_bits_do_not_depend_on_the_others(hl, dtype, vocab):
    """Split over workgroups or not, and wherever the row begins."""
    z, t = logits(1200, vocab, dtype, 9)
    zd, t = z.cuda(), t.abs().clamp(max=vocab - 1).cuda()
    whole = forward(hl, zd, t, 1.0)
    for a, b in ((0, 1), (3, 4), (1199, 1200), (5, 700), (7, 519), (7, 520)):
        some = forward(hl, zd[a:b], t[a:b], 1.0)
        assert all(torch.equal(some[k], whole[k][a:b]) for k in whole), (a, b)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("vocab", [16387, 32773, 65531, 65544, 100003, 262143])
def test_counts_of_rows_about_the_chip(hl, dtype, vocab):
    """One workgroup a row, larger ones, and a row split over several: right, and the same bits."""
    z, t = logits(260, vocab, dtype, 10)
    zd, td = z.cuda(), t.cuda()
    whole = forward(hl, zd.repeat(2, 1)[:515], td.repeat(2)[:515], 1.0)
    for rows in (1, 30, 128, 129, 200, 256, 257):
        some = forward(hl, zd[:rows], td[:rows], 1.0)
        assert all(torch.equal(some[k], whole[k][:rows]) for k in whole), rows
    few = forward(hl, zd[:60], td[:60], 1.0)
    check_forward(few, z[:60], t[:60], 1.0)


def test_shifted_slices(hl):
    """Targets and logits one row apart, as a causal model has them: addresses between 16-byte steps."""
    z, _ = logits(30, 4001, BF16, 12)
    ids = torch.randint(0, 4001, (30,))
    zd, idd = z.cuda(), ids.cuda()
    o = forward(hl, zd[:-1], idd[1:], 1.0)
    check_forward(o, z[:-1], ids[1:], 1.0)
    o = forward(hl, zd[1:], idd[:-1], 1.0)
    check_forward(o, z[1:], ids[:-1], 1.0)


@pytest.mark.parametrize("scale", [2.0 ** -126, 2.0 ** 127])
def test_ends_of_the_scales(hl, scale):
    """The distribution is uniform, or the largest logit's alone."""
    z, t = torch.tensor([[1.0, 2.0, 3.0]] * 2, device="cuda"), torch.tensor([2, 1], device="cuda")
    o, d = forward(hl, z, t, scale), torch.full((2, 3), 5.0, device="cuda")
    one = torch.ones(2, device="cuda")
    hl.hilore_token_logprobs_bwd(hl.token_logprobs_bwd_desc(z, t, o["row_max"], o["log_sum"], one, d, entropy=o["entropy"], dentropy=one, scale=scale))
    if scale > 1.0:
        assert o["logp"].tolist() == [0.0, -scale] and o["entropy"].tolist() == [0.0, 0.0]
        assert d.tolist() == [[0.0, 0.0, 0.0], [0.0, scale, -scale]]
    else:
        assert torch.allclose(o["logp"], -torch.log(3 * one), rtol=2.0 ** -21) and torch.allclose(o["entropy"], torch.log(3 * one), rtol=2.0 ** -21)
        assert (d.abs() <= scale).all()


def test_no_rows(hl):
    z = torch.empty(0, 100, dtype=BF16, device="cuda")
    t, e = torch.empty(0, dtype=torch.int64, device="cuda"), torch.empty(0, device="cuda")
    hl.hilore_token_logprobs(hl.token_logprobs_desc(z, t, logp=e))
    hl.hilore_token_logprobs_bwd(hl.token_logprobs_bwd_desc(z, t, e, e, e, z))


def test_past_32_bits(hl):
    """Rows behind 2^32 elements."""
    rows, vocab = 33000, 131072
    z = torch.zeros(rows, vocab, dtype=BF16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    some = [0, 16384, 32767, 32768, 32999]
    for r in some:
        z[r] = torch.randn(vocab, generator=g, device="cuda")
    t = torch.full((rows,), -1, device="cuda")
    t[some] = torch.tensor([5, 131071, 77, 1, 100000], device="cuda")
    o = forward(hl, z, t, 1.0)
    check_forward({k: v[some] for k, v in o.items()}, z[some].cpu(), t[some].cpu(), 1.0)
    d = torch.ones_like(z)
    hl.hilore_token_logprobs_bwd(hl.token_logprobs_bwd_desc(z, t, o["row_max"], o["log_sum"], torch.ones(rows, device="cuda"), d))
    small = torch.empty(len(some), vocab, dtype=BF16, device="cuda")
    hl.hilore_token_logprobs_bwd(hl.token_logprobs_bwd_desc(z[some], t[some], o["row_max"][some], o["log_sum"][some],
                                                            torch.ones(len(some), device="cuda"), small))
    assert torch.equal(d[some], small)
    d[some] = 0.0
    assert not d.any()
