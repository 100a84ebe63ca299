"""hilore_adamw over more tensors than any launch takes (67 to 100), at lengths around the lane's, the
block's and the chunk's ends, sentinels behind every buffer, against the 64-bit reference."""
import pytest
import torch

from test_gpu_adamw import B1, B2, EPS, check, descriptor, make

pytestmark = pytest.mark.gpu
LENGTHS = [0, 1, 2, 3, 4, 5, 7, 8, 9, 63, 255, 256, 257, 259, 511, 513, 1023, 4095, 4096, 4097, 4100, 8191, 16385]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("param", ["f32", "bf16", "master"])
def test_lengths_over_launches(hl, param, bits):
    lengths = (LENGTHS + LENGTHS[::-1]) * 5
    assert len(lengths) > 2 * 100  # three launches at least
    ts = [make(n, 2000 + i, param, "bf16" if i % 2 else "f32", bits, tail=9) for i, n in enumerate(lengths)]
    hl.hilore_adamw([descriptor(hl, t) for t in ts], B1, B2, EPS, 3, seed=17)
    torch.cuda.synchronize()
    for i, t in enumerate(ts):
        check(t, i, 3, 17)
