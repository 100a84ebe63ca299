"""One weight for the heads of queries and keys: its gradient is the sum of both sides'.

Tolerance: the two sides apart are the same terms, in the same groups; the sums of up to 2 * 768 groups in another
order and one more addition of two roundings: 1540 steps of 2^-24 of the terms' sizes in the worst order, 2^-13.  The sizes are
those of the sides' sums of absolute values, from a call with the gradients' and the rows' signs taken off (the weight is
positive and nothing is rotated, so that dn x r is positive)."""
import pytest
import torch

from test_gpu_qk_norm_rope import gen, randn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens,hq,hk,dim", [(1, 2, 1, 16), (5, 14, 2, 64), (130, 28, 4, 128), (3, 3, 3, 512), (4000, 4, 4, 64)])
@pytest.mark.parametrize("accumulate", [False, True])
def test_one_gradient_tensor(hl, tokens, hq, hk, dim, accumulate):
    g = gen(61)
    rows, grads = randn(g, tokens, (hq + hk) * dim).cuda(), randn(g, tokens, hq + hk, dim).cuda()
    w = (1.0 + 0.2 * torch.randn(dim, generator=g)).abs().to(torch.bfloat16).cuda()

    def run(rows, grads, dw_q, dw_k, accumulate):
        desc = hl.qk_norm_rope_bwd_desc(dq=grads[:, :hq], dk=grads[:, hq:], q=hl.unit_desc(x=rows[:, :hq * dim]),
                                        k=hl.unit_desc(x=rows[:, hq * dim:]), w_q=w, w_k=w, dw_q=dw_q, dw_k=dw_k)
        hl.hilore_qk_norm_rope_bwd(desc, accumulate=accumulate)

    one, again, q, k, sq, sk = (torch.full((dim,), 0.5, device="cuda") for _ in range(6))
    run(rows, grads, one, one, accumulate)
    run(rows, grads, again, again, accumulate)
    run(rows, grads, q, k, False)
    run(rows.abs(), grads.abs(), sq, sk, False)
    want = q.double() + k.double() + (0.5 if accumulate else 0.0)
    limit = 2.0 ** -13 * (sq + sk).double() + (2.0 ** -24 if accumulate else 0.0)
    assert ((one.double() - want).abs() <= limit).all()
    assert torch.equal(one, again)
