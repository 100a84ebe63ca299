"""The operators between an actor's products past 2^32 elements and past the workgroups of one launch,
where each takes several turns: every row, token or pair has the bits that a small call gives it."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_heads_in_rows_behind_2_32_elements(hl):
    """Three tokens 2^31 + 64 elements apart, in and out."""
    ld, dim = (1 << 31) + 64, 64
    rows = torch.empty(2 * ld + 256, dtype=torch.bfloat16, device="cuda").as_strided((3, 128), (ld, 1))
    out = torch.empty(2 * ld + 256, dtype=torch.bfloat16, device="cuda").as_strided((3, 2, dim), (ld, dim, 1))
    g = torch.Generator(device="cuda").manual_seed(1)
    x, go, w = (torch.randn(s, generator=g, device="cuda").bfloat16() for s in ((3, 128), (3, 2, dim), (dim,)))
    freq, pos = (10000.0 ** (-torch.arange(32) / 32)).cuda(), torch.tensor([5, 70, 900]).cuda()
    small, dsmall, dw = torch.empty(3, 2, dim, dtype=torch.bfloat16, device="cuda"), torch.empty(3, 128, dtype=torch.bfloat16, device="cuda"), torch.empty(2, dim, device="cuda")
    kw = dict(inv_freq=freq, positions=pos, w_q=w)
    hl.hilore_qk_norm_rope(hl.qk_norm_rope_desc(q=x, q_out=small, **kw))
    hl.hilore_qk_norm_rope_bwd(hl.qk_norm_rope_bwd_desc(dq=go, dq_in=dsmall, q=hl.unit_desc(x=x), dw_q=dw[0], **kw))
    rows.copy_(x)
    hl.hilore_qk_norm_rope(hl.qk_norm_rope_desc(q=rows, q_out=out, **kw))
    assert torch.equal(out, small)
    out.copy_(go)  # now the gradient, and the inputs' gradient back over the rows
    hl.hilore_qk_norm_rope_bwd(hl.qk_norm_rope_bwd_desc(dq=out, dq_in=rows, q=hl.unit_desc(x=x), dw_q=dw[1], **kw))
    assert torch.equal(rows, dsmall) and torch.equal(dw[0], dw[1])
    # heads instead of tokens far apart, and saved rows far apart
    heads = out.as_strided((3, 2, dim), (dim, ld, 1))
    rows.copy_(x)
    hl.hilore_qk_norm_rope(hl.qk_norm_rope_desc(q=x, q_out=heads, **kw))
    assert torch.equal(heads, small)
    again = torch.empty_like(dsmall)
    hl.hilore_qk_norm_rope_bwd(hl.qk_norm_rope_bwd_desc(dq=go, dq_in=again, q=hl.unit_desc(x=rows), dw_q=dw[1], **kw))
    assert torch.equal(again, dsmall) and torch.equal(dw[0], dw[1])


def test_heads_of_many_tokens(hl):
    n = 4 * (1 << 22) + 77  # more than four to each workgroup of the largest grid
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn((n, 16), generator=g, device="cuda").bfloat16()
    w, freq = torch.ones(16, dtype=torch.bfloat16, device="cuda"), torch.tensor([1.0, 0.3, 0.1, 0.03, 0.01, 3e-3, 1e-3, 3e-4], device="cuda")
    out, dx = torch.zeros(n, 1, 16, dtype=torch.bfloat16, device="cuda"), torch.zeros(n, 16, dtype=torch.bfloat16, device="cuda")
    pos = torch.arange(n, device="cuda")
    hl.hilore_qk_norm_rope(hl.qk_norm_rope_desc(q=x, q_out=out, inv_freq=freq, w_q=w))
    hl.hilore_qk_norm_rope_bwd(hl.qk_norm_rope_bwd_desc(dq=out, dq_in=dx, q=hl.unit_desc(x=x), inv_freq=freq, w_q=w))
    for a in (0, n // 2, n - 300):
        part, dpart = torch.empty(300, 1, 16, dtype=torch.bfloat16, device="cuda"), torch.empty(300, 16, dtype=torch.bfloat16, device="cuda")
        kw = dict(inv_freq=freq, w_q=w, positions=pos[a:a + 300])
        xs = x[a:a + 300].clone()
        hl.hilore_qk_norm_rope(hl.qk_norm_rope_desc(q=xs, q_out=part, **kw))
        hl.hilore_qk_norm_rope_bwd(hl.qk_norm_rope_bwd_desc(dq=part, dq_in=dpart, q=hl.unit_desc(x=xs), **kw))
        assert torch.equal(part, out[a:a + 300]) and torch.equal(dpart, dx[a:a + 300])


@pytest.mark.parametrize("dim,heads", [(512, 4200), (256, 8206)])
def test_heads_backward_of_thousands_of_heads(hl, dim, heads):
    """Three tokens whose heads are more than waves take: each head's gradient as a call with fewer heads has it."""
    g = torch.Generator(device="cuda").manual_seed(8)
    x, go = (torch.randn(3, heads, dim, generator=g, device="cuda").bfloat16() for _ in range(2))
    w = torch.randn(dim, generator=g, device="cuda").bfloat16()
    dx, dw = torch.full_like(x, 9.0), torch.empty(dim, device="cuda")
    hl.hilore_qk_norm_rope_bwd(hl.qk_norm_rope_bwd_desc(dq=go, dq_in=dx.view(3, -1), q=hl.unit_desc(x=x.view(3, -1)), w_q=w, dw_q=dw))
    for a in range(0, heads, 700):
        xs, gs = x[:, a:a + 700].contiguous(), go[:, a:a + 700].contiguous()
        part, dpart = torch.full_like(xs, 9.0), torch.empty(dim, device="cuda")
        hl.hilore_qk_norm_rope_bwd(hl.qk_norm_rope_bwd_desc(dq=gs, dq_in=part.view(3, -1), q=hl.unit_desc(x=xs.view(3, -1)), w_q=w, dw_q=dpart))
        assert torch.equal(part, dx[:, a:a + 700]), a
    terms = go.double() * x.double() * torch.rsqrt(x.double().square().mean(-1, keepdim=True) + 1e-6)
    # fewer than 100 roundings on a term's way into its sum, and two units in the last place of the root
    assert ((dw.double() - terms.sum((0, 1))).abs() <= 104 * 2.0 ** -24 * terms.abs().sum((0, 1))).all()


def test_logprobs_of_many_rows(hl):
    n = (1 << 22) + 300  # more than one row to each workgroup of the largest grid
    g = torch.Generator(device="cuda").manual_seed(3)
    z = torch.randn((n, 11), generator=g, device="cuda")
    t = torch.randint(-2, 11, (n,), generator=g, device="cuda")
    f = [torch.full((n,), 9.0, device="cuda") for _ in range(4)]
    d, ones = torch.full_like(z, 9.0), torch.ones(n, device="cuda")
    hl.hilore_token_logprobs(hl.token_logprobs_desc(z, t, *f))
    hl.hilore_token_logprobs_bwd(hl.token_logprobs_bwd_desc(z, t, f[2], f[3], ones, d, entropy=f[1], dentropy=ones))
    lp = torch.log_softmax(z.double(), 1)
    live = t >= 0
    want = torch.where(live, lp.gather(1, t.clamp(min=0)[:, None])[:, 0], 0.0)
    # 2^-16 of the others and 2^-21 of a logp of at most about 12
    assert (f[0].double() - want).abs().max() < 2.0 ** -16 + 12 * 2.0 ** -21
    for a in (0, n // 2, n - 500):
        s = slice(a, a + 500)
        q = [torch.empty(500, device="cuda") for _ in range(4)]
        e = torch.empty(500, 11, device="cuda")
        hl.hilore_token_logprobs(hl.token_logprobs_desc(z[s], t[s], *q))
        hl.hilore_token_logprobs_bwd(hl.token_logprobs_bwd_desc(z[s], t[s], q[2], q[3], ones[s], e, entropy=q[1], dentropy=ones[s]))
        assert all(torch.equal(x, y[s]) for x, y in zip(q, f)) and torch.equal(e, d[s])


@pytest.mark.parametrize("sequences,length", [(60000, 31), (1500, 700), (40, 40000), (1100000, 1)])
def test_policy_of_many_tokens(hl, sequences, length):
    """With the normaliser given, a part of the sequences gives its tokens the values of the whole."""
    n = sequences * length
    g = torch.Generator(device="cuda").manual_seed(4)
    old = -torch.rand(n, generator=g, device="cuda")
    new = old + 0.3 * torch.randn(n, generator=g, device="cuda")
    ref, adv = old + 0.1, torch.randn(sequences, generator=g, device="cuda")
    mask = torch.rand(n, generator=g, device="cuda") < 0.9
    offsets = torch.arange(sequences + 1, device="cuda") * length

    def run(a, b, packed, ratio):
        s = slice(a * length, b * length)
        out = [torch.full(((b - a) * length,), 9.0, device="cuda") for _ in range(2)] + [torch.empty(8, device="cuda")]
        hl.hilore_policy_loss(hl.policy_loss_desc(new[s], old[s], adv[a:b], logp_ref=ref[s], mask=mask[s], sequences=b - a,
                                                  offsets=offsets[:b - a + 1] if packed else None, kl=2, beta=0.1, ratio=ratio,
                                                  mean="sequences", n_norm=1000.0, dlogp=out[0], token_loss=out[1], stats=out[2]))
        return out

    for ratio in ("token", "sequence"):
        whole = run(0, sequences, True, ratio)
        flat = run(0, sequences, False, ratio)
        assert torch.equal(whole[0], flat[0]) and torch.equal(whole[1], flat[1])
        assert not (whole[0] == 9.0).any()
        # sums of the same numbers in another order, in fp32 by 256: 8 roundings of their sizes
        assert abs(float(whole[2][0]) - float(whole[1].double().sum())) <= 2.0 ** -20 * float(whole[1].double().abs().sum())
        assert float(whole[2][6]) == float(mask.sum())
        for a in (0, sequences - 11):
            part = run(a, a + 11, True, ratio)
            s = slice(a * length, (a + 11) * length)
            assert torch.allclose(part[0], whole[0][s], rtol=2.0 ** -21, atol=0) and torch.allclose(part[1], whole[1][s], rtol=2.0 ** -19, atol=1e-10)


@pytest.mark.parametrize("sequences,length", [(600000, 2), (3000, 600)])
def test_preference_of_many_pairs(hl, sequences, length):
    n = sequences * length
    g = torch.Generator(device="cuda").manual_seed(5)
    new = torch.randn(n, generator=g, device="cuda")
    d, rewards, loss, stats = (torch.empty(k, device="cuda") for k in (n, sequences, sequences // 2, 6))
    hl.hilore_preference_loss(hl.preference_loss_desc(new, sequences=sequences, beta=0.5, dlogp=d, rewards=rewards, pair_loss=loss, stats=stats))
    value = new.double().reshape(sequences, length).sum(1)
    h = 0.5 * (value[0::2] - value[1::2])
    want = torch.nn.functional.softplus(-h)
    assert ((loss.double() - want).abs() <= 2.0 ** -23 * want + 1e-12).all()
    slope = -0.5 * torch.sigmoid(-h) / (sequences // 2)
    each = torch.stack((slope, -slope), 1).reshape(-1, 1).expand(-1, length).reshape(-1)
    assert ((d.double() - each).abs() <= 2.0 ** -23 * each.abs() + 1e-18).all()
    assert float(stats[0]) == pytest.approx(float(want.mean()), rel=1e-6) and float(stats[5]) == sequences // 2
    assert ((rewards.double() - 0.5 * value).abs() <= 2.0 ** -23 * value.abs() + 1e-12).all()


def test_preference_lists_of_many_pairs(hl):
    """The same pairs as lists, in another order: the same sums of the same terms."""
    sequences = 2400
    new = torch.randn(sequences, 3, generator=torch.Generator(device="cuda").manual_seed(6), device="cuda")
    order = torch.randperm(sequences // 2, device="cuda").to(torch.int32)
    a, b = torch.empty(sequences, 3, device="cuda"), torch.empty(sequences, 3, device="cuda")
    hl.hilore_preference_loss(hl.preference_loss_desc(new, dlogp=a))
    hl.hilore_preference_loss(hl.preference_loss_desc(new, chosen=2 * order, rejected=2 * order + 1, dlogp=b))
    assert torch.allclose(a, b, rtol=2.0 ** -23, atol=0)


@pytest.mark.parametrize("length", [40, 256, 1024, 4096])
def test_losses_of_the_most_tokens(hl, length):
    """2^31 - 1 tokens, whose last sequences begin fewer tokens before 2^31 than a workgroup has threads."""
    n, tail = (1 << 31) - 1, 600
    g = torch.Generator(device="cuda").manual_seed(7)
    ends = torch.tensor([n - tail, n - 300, n - 3, n], device="cuda")
    offsets = torch.cat((torch.arange(0, n - tail, length, device="cuda"), ends))
    sequences = offsets.numel() - 1
    new, old = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    new[-tail:], old[-tail:] = (torch.randn(tail, generator=g, device="cuda") for _ in range(2))
    d, stats = torch.full((n,), 9.0, device="cuda"), torch.empty(8, device="cuda")
    adv = torch.ones(sequences, device="cuda")
    few, part = slice(n - tail, n), torch.full((tail,), 9.0, device="cuda")
    kw = dict(ratio="sequence", mean="sequences", n_norm=1000.0, clip_high=5.0)
    hl.hilore_policy_loss(hl.policy_loss_desc(new, old, adv, offsets=offsets, dlogp=d, stats=stats, **kw))
    hl.hilore_policy_loss(hl.policy_loss_desc(new[few], old[few], adv[:3], offsets=ends - (n - tail), dlogp=part, **kw))
    # means and weights of one call against the other's: a rounding each of the weight, the mean, exp (2) and the product
    assert torch.allclose(d[few], part, rtol=2.0 ** -21, atol=0)
    assert float(stats[6]) == 2.0 ** 31 and float(stats[7]) == float(torch.tensor(float(sequences)))
    # equal ratios of 1 in all other sequences: weight 1 / (1000 length) each
    assert float(d[0]) == float(d[length * 5 + 3]) == pytest.approx(-1e-3 / length, rel=2.0 ** -22)
    rewards, six = torch.empty(sequences, device="cuda"), torch.empty(6, device="cuda")
    d.fill_(9.0)
    hl.hilore_preference_loss(hl.preference_loss_desc(new, old, offsets=offsets, beta=1.0, dlogp=d, rewards=rewards, stats=six))
    x = (new[few] - old[few]).double()
    want = torch.stack([x[:300].sum(), x[300:597].sum(), x[597:].sum()])
    assert ((rewards[-3:].double() - want).abs() <= 2.0 ** -23 * want.abs() + 1e-12).all()
    assert not rewards[:-3].any() and float(six[5]) == float(torch.tensor(float(sequences // 2)))
    assert not (d[few] == 9.0).any()
