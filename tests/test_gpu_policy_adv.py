"""The policy loss over as many packed sequences as tokens, with one advantage a token and one a sequence.
Tolerances as in test_gpu_losses."""
import pytest
import torch

import actor_reference as R
from test_gpu_losses import batch, check_policy

pytestmark = pytest.mark.gpu


# 4 tokens by one workgroup, 3000 by launches: every second sequence is empty, the others have two tokens
@pytest.mark.parametrize("n", [4, 3000])
@pytest.mark.parametrize("per_token", [True, False])
def test_as_many_sequences_as_tokens(hl, n, per_token):
    g, new, old, _, _ = batch(n, 40)
    offsets = (torch.arange(n + 1) + 1) // 2 * 2
    assert offsets[:5].tolist() == [0, 2, 2, 4, 4]
    adv = torch.randn(n, generator=g)
    out = {k: torch.full((n,), 9.0, device="cuda") for k in ("dlogp", "token_loss")}
    out["flags"], out["stats"] = torch.full((n,), 9, dtype=torch.uint8, device="cuda"), torch.empty(8, device="cuda")
    hl.hilore_policy_loss(hl.policy_loss_desc(new.cuda(), old.cuda(), adv.cuda(), offsets=offsets.cuda(), mean="sequences",
                                              adv_per_token=per_token, **out))
    got = {k: v.cpu() for k, v in out.items()}
    # the sequences that are not empty, whose number is not that of the tokens
    full = offsets[::2]
    want = R.policy_loss(new, old, adv if per_token else adv[::2], n // 2, None, None, None, full, mean="sequences")
    check_policy(got, want, n, full)
