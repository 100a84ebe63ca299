"""int8 products whose last round of 256 x 256 tiles goes as quarters, at the longest such rounds
(64 and 63 tiles): several rounds of whole tiles' work follow one another in one launch of quarters."""
import pytest
import torch

from test_gpu_int8_tiles import test_last_tiles_in_quarters as check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens,k,n", [(1793, 1056, 10216), (3871, 1040, 4920), (2584, 1056, 7192)])
@pytest.mark.parametrize("out_f32,accumulate", [(False, False), (True, False), (False, True), (True, True)])
def test_longest_last_rounds(hl, tokens, k, n, out_f32, accumulate):
    tiles = -(-tokens // 256) * -(-n // 256)
    assert tiles > 256 and tiles % 256 in (63, 64)
    check(hl, tokens, k, n, out_f32, accumulate)


def test_whole_rounds_and_quarters_agree(hl):
    """Tokens are independent of one another: those of a call with a quartered last round have the
    bits that they have in calls of 1000 tokens."""
    tokens, k, n = 1793, 1056, 10216
    g = torch.Generator(device="cuda").manual_seed(3)
    a, w = (torch.randint(-127, 128, s, generator=g, device="cuda", dtype=torch.int8) for s in ((tokens, k), (n, k)))
    sa, sw = torch.rand(2 * tokens, generator=g, device="cuda")[:tokens], torch.rand(n, generator=g, device="cuda")
    out = torch.full((tokens, n), float("nan"), dtype=torch.bfloat16, device="cuda")
    hl.hilore_int8_matmul(hl.int8_desc(w=w, out=out, a=a, a_scales=sa, w_scales=sw))
    for first in range(0, tokens, 1000):
        part, scales = a[first:first + 1000].contiguous(), sa[first:first + 1000].clone()
        some = torch.full((len(part), n), float("nan"), dtype=torch.bfloat16, device="cuda")
        hl.hilore_int8_matmul(hl.int8_desc(w=w, out=some, a=part, a_scales=scales, w_scales=sw))
        assert torch.equal(some, out[first:first + 1000])
