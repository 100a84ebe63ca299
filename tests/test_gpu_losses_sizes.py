"""The losses on both sides of the sizes where their steps are shared out differently: one workgroup or three
launches, 8 or 64 lanes or a workgroup to a sequence, tiles of all tokens or of a sequence."""
import pytest
import torch

import actor_reference as R
from test_gpu_losses import batch, check_policy, check_preference, run_policy

pytestmark = pytest.mark.gpu

# sequences, length: mean lengths around 64, 512 and 4096, tokens around 2048 and 4096, sequences around 16, 256 and 1024
SIZES = [(32, 64), (32, 65), (31, 65), (64, 64), (63, 66), (5, 512), (4, 512), (4, 513), (9, 512), (9, 513), (2, 2048), (2, 2049),
         (3, 4096), (3, 4097), (17, 100), (16, 256), (17, 256), (1024, 2), (1025, 2), (1025, 3), (2, 9001), (300, 7)]


@pytest.mark.parametrize("sequences,length", SIZES)
@pytest.mark.parametrize("ragged", [False, True])
def test_policy(hl, sequences, length, ragged):
    n = sequences * length
    g, new, old, ref, ent = batch(n, sequences + length)
    mask = (torch.rand(n, generator=g) < 0.8).to(torch.uint8)
    adv = torch.randn(sequences, generator=g)
    offsets = None
    if ragged:
        cuts = torch.sort(torch.randint(0, n + 1, (sequences - 1,), generator=g)).values
        offsets = torch.cat([torch.zeros(1, dtype=torch.int64), cuts, torch.tensor([n])])
    for ratio in ("token", "sequence"):
        kw = dict(kl=3, beta=0.05, entropy_weight=0.01, ratio=ratio, mean="sequences", dual_clip=3.0)
        got = run_policy(hl, n, sequences, offsets, mask, new, old, adv, ref, ent, **kw)
        check_policy(got, R.policy_loss(new, old, adv, sequences, ref, ent, mask, offsets, **kw), n, offsets)


@pytest.mark.parametrize("sequences,length", SIZES)
@pytest.mark.parametrize("lists", [False, True])
def test_preference(hl, sequences, length, lists):
    n = sequences * length
    g, new, _, ref, _ = batch(n, sequences + length, 0.1)
    mask = (torch.rand(n, generator=g) < 0.8).to(torch.uint8)
    cuts = torch.sort(torch.randint(0, n + 1, (sequences - 1,), generator=g)).values
    offsets = torch.cat([torch.zeros(1, dtype=torch.int64), cuts, torch.tensor([n])])
    pair = [torch.randint(0, sequences, (2 * sequences + 3,), generator=g).to(torch.int32) for _ in range(2)] if lists else [None, None]
    check_preference(hl, n, sequences, offsets, mask, new, ref, *pair, beta=0.2, label_smoothing=0.05)
