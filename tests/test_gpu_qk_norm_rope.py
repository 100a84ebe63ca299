"""hilore_qk_norm_rope and its backward against 64 bits.

Tolerances.  Outputs are rounded once to bf16: half a step, 2^-8 of the value.  Before that the
fp32 arithmetic: the mean's sum takes at most 16 + 5 roundings, the factors and the rotation
about 10 more and the angle is right within 2^-25 of a turn (2e-7 of the rotated pair), so less than 40 steps
of 2^-24 relative to the head's largest value: 2^-18 of it.  Backward forms each column from terms
of the size heads_backward returns, with two such sums: 2^-17 of that.  A weight's gradient is
a sum of n terms in fp32, in the worst order n roundings: n 2^-24 of the terms' sizes, and 2^-18
for the terms themselves.
"""
import pytest
import torch

import actor_reference as R
from layer_reference import bf16

pytestmark = pytest.mark.gpu

SENTINEL = 7.0


def gen(seed):
    return torch.Generator().manual_seed(seed)


def randn(g, *shape, sigma=1.0):
    return (sigma * torch.randn(*shape, generator=g)).to(torch.bfloat16)


def freqs(rotated):
    half = rotated // 2
    return (10000.0 ** (-torch.arange(half, dtype=torch.float64) / max(half, 1))).float()


def strided(tokens, heads, dim, layout, pad=0):
    """(buffer full of sentinels, view [tokens, heads, dim]) on the device."""
    if layout == "heads":
        buf = torch.full((heads, tokens + pad, dim + pad), SENTINEL, dtype=torch.bfloat16, device="cuda")
        return buf, buf.transpose(0, 1)[:tokens, :, :dim]
    buf = torch.full((tokens, heads, dim + pad), SENTINEL, dtype=torch.bfloat16, device="cuda")
    return buf, buf[:, :, :dim]


def close(got, want, size, steps, what):
    got = got.double().cpu()
    limit = 2.0 ** -8 * want.abs() + steps * size + 1e-38
    bad = ~((got - want).abs() <= limit)
    assert not bad.any(), (what, int(bad.sum()), float(((got - want).abs() / limit)[bad].max()), bad.nonzero()[0].tolist())


SHAPES = [  # tokens, heads_q, heads_k, dim, rotated, pairs, norm, layout, pad
    (1, 28, 4, 128, 128, False, True, "tokens", 0), (1, 1, 0, 16, 16, False, True, "tokens", 0),
    (5, 14, 2, 64, 64, True, True, "heads", 8), (67, 3, 3, 80, 80, False, True, "tokens", 16),
    (33, 5, 1, 96, 32, True, True, "heads", 0), (130, 28, 4, 128, 128, False, True, "heads", 8),
    (9, 7, 1, 192, 192, False, True, "tokens", 8), (6, 16, 8, 256, 64, False, True, "heads", 0),
    (3, 2, 1, 512, 512, True, True, "tokens", 0), (17, 4, 2, 128, 0, False, True, "tokens", 0),
    (40, 33, 9, 32, 16, False, True, "heads", 8), (257, 6, 2, 64, 64, False, False, "tokens", 8),
    (2, 65, 0, 48, 48, True, False, "heads", 0), (700, 1, 1, 16, 16, True, True, "tokens", 0),
]


def inputs(shape, seed, positions="mixed"):
    tokens, hq, hk, dim, rotated, pairs, norm, layout, pad = shape
    g = gen(seed)
    rows = randn(g, tokens, (hq + 2 * hk) * dim + 24)
    if positions == "far":
        pos = torch.randint(0, 1 << 40, (tokens,), generator=g)
    else:
        pos = torch.randint(0, 5000, (tokens,), generator=g)
        pos[torch.rand(tokens, generator=g) < 0.2] = -1
        if tokens > 2:
            pos[0], pos[1], pos[2] = 0, 2 ** 31 - 1, -(2 ** 62)
    # what stands at padding is not to be seen
    rows[pos < 0] = float("nan")
    w = [(1.0 + randn(g, dim, sigma=0.2)) if norm else None for _ in range(2)]
    return g, rows, pos, w


def parts(rows, hq, hk, dim):
    return rows[:, :hq * dim], rows[:, hq * dim:(hq + hk) * dim]


def on(t):
    return None if t is None else t.cuda()


@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("positions", ["mixed", "far"])
def test_forward(hl, shape, positions):
    tokens, hq, hk, dim, rotated, pairs, norm, layout, pad = shape
    _, rows, pos, w = inputs(shape, 11, positions)
    freq, drows = freqs(rotated), rows.cuda()
    bufs, outs = zip(*(strided(tokens, h, dim, layout, pad) for h in (hq, max(hk, 1))))
    kept = [b.clone() for b in bufs]
    q, k = parts(drows, hq, hk, dim)
    hl.hilore_qk_norm_rope(hl.qk_norm_rope_desc(
        q=q, q_out=outs[0], k=k if hk else None, k_out=outs[1] if hk else None, inv_freq=on(freq) if rotated else None,
        positions=on(pos), w_q=on(w[0]), w_k=on(w[1]), rope_scale=1.25, rotation="pairs" if pairs else "halves"))
    torch.cuda.synchronize()
    for x, wi, out, buf, old, h in zip(parts(rows, hq, hk, dim), w, outs, bufs, kept, (hq, hk)):
        if h == 0:
            continue
        x = torch.where(pos[:, None] < 0, 0.0, x.double()).reshape(tokens, h, dim)
        want = R.heads_forward(x, None if wi is None else wi.double(), 1e-6, pos, freq, pairs, 1.25)
        close(out, want, want.abs().amax(-1, keepdim=True), 2.0 ** -18, shape)
        out.fill_(0.0)
        old.as_strided(out.shape, out.stride(), out.storage_offset()).fill_(0.0)
        assert torch.equal(buf, old)  # between the heads nothing is written


def test_without_positions_and_weights_of_one_side(hl):
    g = gen(3)
    x, w = randn(g, 37, 4 * 64), randn(g, 64)
    out = [torch.empty(37, 2, 64, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    d = x.cuda()
    hl.hilore_qk_norm_rope(hl.qk_norm_rope_desc(q=d[:, :128], k=d[:, 128:], q_out=out[0], k_out=out[1], inv_freq=freqs(64).cuda(),
                                                w_k=w.cuda()))
    pos = torch.arange(37)
    for i, wi in enumerate((None, w.double())):
        want = R.heads_forward(x.double()[:, 128 * i:128 * i + 128].reshape(37, 2, 64), wi, 1e-6, pos, freqs(64), False)
        close(out[i], want, want.abs().amax(-1, keepdim=True), 2.0 ** -18, i)


@pytest.mark.parametrize("tokens", [1, 50])
def test_in_place(hl, tokens):
    """The projection's rows turned where they stand; the values between are left as they were."""
    rows = randn(gen(4), tokens, 5 * 64).cuda()
    q, k, pos, freq, w = rows[:, :128], rows[:, 128:192], torch.arange(tokens).cuda() + 9, freqs(64).cuda(), randn(gen(5), 64).cuda()
    out = [torch.empty(tokens, h, 64, dtype=torch.bfloat16, device="cuda") for h in (2, 1)]
    hl.hilore_qk_norm_rope(hl.qk_norm_rope_desc(q=q, k=k, q_out=out[0], k_out=out[1], inv_freq=freq, positions=pos, w_q=w, w_k=w))
    there = rows.clone()
    hl.hilore_qk_norm_rope(hl.qk_norm_rope_desc(q=there[:, :128], k=there[:, 128:192],
                                                q_out=there[:, :128].unflatten(1, (2, 64)), k_out=there[:, 128:192].unflatten(1, (1, 64)),
                                                inv_freq=freq, positions=pos, w_q=w, w_k=w))
    assert torch.equal(there[:, :128], out[0].flatten(1)) and torch.equal(there[:, 128:192], out[1].flatten(1))
    assert torch.equal(there[:, 192:], rows[:, 192:])


def test_a_tokens_bits_do_not_depend_on_the_others(hl):
    rows, pos, freq, w = randn(gen(6), 5000, 6 * 128).cuda(), torch.arange(5000).cuda(), freqs(128).cuda(), randn(gen(7), 128).cuda()

    def run(a, b):
        q, k = torch.empty(b - a, 4, 128, dtype=torch.bfloat16, device="cuda"), torch.empty(b - a, 2, 128, dtype=torch.bfloat16, device="cuda")
        hl.hilore_qk_norm_rope(hl.qk_norm_rope_desc(q=rows[a:b, :512], k=rows[a:b, 512:], q_out=q, k_out=k, inv_freq=freq,
                                                    positions=pos[a:b], w_q=w, w_k=w))
        return q, k

    whole = run(0, 5000)
    for a, b in ((0, 1), (4999, 5000), (77, 400)):
        assert all(torch.equal(p, o[a:b]) for p, o in zip(run(a, b), whole))


# --------------------------------------------------------------- backward --
def unit_of(hl, x, code, block):
    """(descriptor, saved value in 64 bits) of bf16 rows as a unit."""
    if code is None:
        d = x.cuda()
        return hl.unit_desc(x=d), x.double()
    d = torch.nan_to_num(x).cuda()
    rows, cols = d.shape
    codes = torch.empty(rows, cols, dtype=torch.uint8, device="cuda")
    scales = torch.empty(rows, cols // block, device="cuda") if block else None
    xhat = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
    u = hl.unit_desc(x=d, codes=codes, scales=scales, xhat=xhat)
    hl.hilore_compress([u], code, block)
    hl.hilore_decompress([u], code, block)
    return hl.unit_desc(codes=codes, scales=scales), xhat.cpu().double()


CODES = [(None, None, 0), ("int8", "int8", 32), ("e4m3fn", None, 64), (None, "e4m3fn", 32), ("e4m3fn_cast", "e4m3fn_cast", 0),
         (None, "int8", 32), ("e4m3fn_cast", None, 0)]


def saved_as(shape):
    """The codes that the saved rows of a shape can have: blocks that divide them, none where none is read."""
    _, hq, hk, dim, _, _, norm, _, _ = shape
    return [c for c in CODES if (norm or c[:2] == (None, None)) and not (c[2] and (hq * dim % c[2] or hk * dim % c[2]))]


@pytest.mark.parametrize("shape,code_q,code_k,block", [(s, *c) for s in SHAPES for c in saved_as(s)], ids=str)
def test_backward(hl, shape, code_q, code_k, block):
    tokens, hq, hk, dim, rotated, pairs, norm, layout, pad = shape
    g, rows, pos, w = inputs(shape, 23)
    freq = freqs(rotated)
    saved = [x.clone() for x in parts(rows[:, :(hq + hk) * dim], hq, hk, dim)]
    units, values = zip(*(unit_of(hl, x, c, block) if norm and x.shape[1] else (None, x.double()) for x, c in zip(saved, (code_q, code_k))))
    grads = []
    for h in (hq, max(hk, 1)):
        _, view = strided(tokens, h, dim, layout, pad)
        view.copy_(randn(g, tokens, h, dim, sigma=0.01))
        view[pos.cuda() < 0] = float("nan")
        grads.append(view)
    drows = torch.full((tokens, (hq + 2 * hk) * dim + 8), SENTINEL, dtype=torch.bfloat16, device="cuda")
    dq_in, dk_in = parts(drows, hq, hk, dim)
    dw = [torch.full((dim,), 0.5, device="cuda") if norm else None for _ in range(2)]
    before = torch.full((dim,), 0.5, dtype=torch.float64)
    kw = dict(dq=grads[0], dk=grads[1] if hk else None, dq_in=dq_in, dk_in=dk_in if hk else None, q=units[0], k=units[1] if hk else None,
              inv_freq=on(freq) if rotated else None, positions=on(pos), w_q=on(w[0]), w_k=on(w[1]) if hk else None, dw_q=dw[0],
              dw_k=dw[1] if hk else None, rope_scale=0.75, rotation="pairs" if pairs else "halves")
    desc = hl.qk_norm_rope_bwd_desc(**kw)
    code = code_q or code_k or 0
    hl.hilore_qk_norm_rope_bwd(desc, code, block, accumulate=True)
    torch.cuda.synchronize()
    for i, (h, out) in enumerate(((hq, dq_in), (hk, dk_in))):
        if h == 0:
            continue
        gi = torch.where((pos < 0)[:, None, None], 0.0, grads[i].cpu().double())
        dx, dws, size, sizes = R.heads_backward(values[i].reshape(tokens, h, dim), None if w[i] is None else w[i].double(), 1e-6, pos,
                                                freq, pairs, gi, 0.75)
        close(out.unflatten(1, (h, dim)), dx, size, 2.0 ** -17, (shape, i))
        if norm:
            off = (dw[i].cpu().double() - before - dws).abs()
            assert (off <= (tokens * h * 2.0 ** -24 + 2.0 ** -18) * sizes + 2.0 ** -24).all(), (shape, i, float((off / (sizes + 1e-30)).max()))
    assert bool((drows[:, (hq + hk) * dim:] == SENTINEL).all())
    # the same call: the same bits; without accumulation the sums alone
    first, firsts = drows.clone(), [None if t is None else t.clone() for t in dw]
    for t in dw:
        if t is not None:
            t.fill_(0.5)
    hl.hilore_qk_norm_rope_bwd(desc, code, block, accumulate=True)
    assert torch.equal(first.view(torch.int16), drows.view(torch.int16))
    assert all(a is None or torch.equal(a, b) for a, b in zip(firsts, dw))


def test_backward_by_differences(hl):
    """A step along one input moves the output along the gradient (forward kernel against backward kernel)."""
    g = gen(31)
    x, w, go = torch.randn(4, 2, 64, generator=g), (1.0 + 0.2 * torch.randn(64, generator=g)).to(torch.bfloat16), randn(g, 4, 2, 64)
    x = x.to(torch.bfloat16)
    freq, pos = freqs(64), torch.tensor([3, 900, 0, 77])
    dx = torch.empty(4, 128, dtype=torch.bfloat16, device="cuda")
    xd, wd, god, fd, pd = (t.cuda() for t in (x.flatten(1), w, go, freq, pos))
    hl.hilore_qk_norm_rope_bwd(hl.qk_norm_rope_bwd_desc(dq=god, dq_in=dx, q=hl.unit_desc(x=xd), inv_freq=fd, positions=pd, w_q=wd))
    h = 2.0 ** -5
    step = torch.randn(4, 2, 64, generator=g).double()

    def value(v):
        return (R.heads_forward(v, w.double(), 1e-6, pos, freq, False) * go.double()).sum()

    quotient = (value(x.double() + h * h * step) - value(x.double() - h * h * step)) / (2 * h * h)
    along = (dx.cpu().double().reshape(4, 2, 64) * step).sum()
    # 512 products, each within 2^-8 of a gradient; the quotient's own error is (h^2)^2 of third derivatives
    assert abs(float(quotient - along)) <= 2.0 ** -8 * float((dx.cpu().double().reshape(4, 2, 64) * step).abs().sum()) + 1e-3


def test_one_gradient_for_all_tokens_and_heads(hl):
    g = gen(8)
    x, w, one = randn(g, 21, 3 * 64), randn(g, 64), randn(g, 64)
    args = dict(q=hl.unit_desc(x=x.cuda()), inv_freq=freqs(64).cuda(), positions=torch.arange(21).cuda(), w_q=w.cuda())
    outs = []
    for grad in (one.cuda().expand(21, 3, 64), one.cuda().expand(21, 3, 64).contiguous()):
        dx, dw = torch.empty(21, 192, dtype=torch.bfloat16, device="cuda"), torch.empty(64, device="cuda")
        hl.hilore_qk_norm_rope_bwd(hl.qk_norm_rope_bwd_desc(dq=grad, dq_in=dx, dw_q=dw, **args))
        outs.append((dx, dw))
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])


def test_only_what_is_wanted(hl):
    """Weights' gradients alone, inputs' alone, and a call without tokens, which clears the sums."""
    g = gen(9)
    x, w, go = randn(g, 300, 2 * 64).cuda(), randn(g, 64).cuda(), randn(g, 300, 2, 64).cuda()
    base = dict(dq=go, q=hl.unit_desc(x=x), inv_freq=freqs(64).cuda(), w_q=w)
    dx, dw, only_dx, only_dw = (torch.empty(300, 128, dtype=torch.bfloat16, device="cuda"), torch.empty(64, device="cuda"),
                                torch.empty(300, 128, dtype=torch.bfloat16, device="cuda"), torch.empty(64, device="cuda"))
    hl.hilore_qk_norm_rope_bwd(hl.qk_norm_rope_bwd_desc(dq_in=dx, dw_q=dw, **base))
    hl.hilore_qk_norm_rope_bwd(hl.qk_norm_rope_bwd_desc(dq_in=only_dx, **base))
    hl.hilore_qk_norm_rope_bwd(hl.qk_norm_rope_bwd_desc(dw_q=only_dw, **base))
    assert torch.equal(dx, only_dx) and torch.equal(dw, only_dw)
    in_place = go.clone()
    hl.hilore_qk_norm_rope_bwd(hl.qk_norm_rope_bwd_desc(**dict(base, dq=in_place, dq_in=in_place.flatten(1))))
    assert torch.equal(in_place.flatten(1), dx)
    none = hl.qk_norm_rope_bwd_desc(dq=go[:0], q=hl.unit_desc(x=x[:0]), inv_freq=freqs(64).cuda(), w_q=w, dw_q=dw)
    hl.hilore_qk_norm_rope_bwd(none, accumulate=True)
    assert torch.equal(dw, only_dw)
    hl.hilore_qk_norm_rope_bwd(none)
    assert not dw.any()


def test_zero_rows_and_large_values(hl):
    """A row of zeros gives zeros (eps under the root), values whose squares overflow give what fp32 gives: 0."""
    x = torch.zeros(2, 64, dtype=torch.bfloat16)
    x[1] = 1e30
    out = torch.empty(2, 1, 64, dtype=torch.bfloat16, device="cuda")
    hl.hilore_qk_norm_rope(hl.qk_norm_rope_desc(q=x.cuda(), q_out=out, w_q=torch.ones(64, dtype=torch.bfloat16, device="cuda")))
    assert not out.any()


def test_tiny_rows_without_eps(hl):
    """Values whose squares are subnormal in fp32 (2^-70: a mean of 2^-140, 512 of the smallest steps, so exact), eps 0."""
    x, go = torch.full((3, 64), 2.0 ** -70, dtype=torch.bfloat16), randn(gen(1), 3, 1, 64)
    w, out, dx = torch.ones(64, dtype=torch.bfloat16), torch.empty(3, 1, 64, dtype=torch.bfloat16, device="cuda"), torch.empty(3, 64, dtype=torch.bfloat16, device="cuda")
    hl.hilore_qk_norm_rope(hl.qk_norm_rope_desc(q=x.cuda(), q_out=out, w_q=w.cuda(), eps=0.0))
    assert bool((out == 1.0).all())
    hl.hilore_qk_norm_rope_bwd(hl.qk_norm_rope_bwd_desc(dq=go.cuda(), dq_in=dx, q=hl.unit_desc(x=x.cuda()), w_q=w.cuda(), eps=0.0))
    pos, freq = torch.arange(3), torch.empty(0)
    want, _, size, _ = R.heads_backward(x.double().reshape(3, 1, 64), w.double(), 0.0, pos, freq, False, go.double())
    close(dx.unflatten(1, (1, 64)), want, size, 2.0 ** -17, "tiny")
