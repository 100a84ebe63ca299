"""Arguments of hilore_block_norm_bwd that it does not read, or lacks: without an L unit its code
and block may be anything.  Each call runs in a process of its own, so that one that does not return
is a failure."""
import subprocess
import sys

import pytest

from test_abi import ROOT, lib  # noqa: F401

CALL = """
import ctypes, sys
from paper_2609_33570_amd import hilore as E
d = E.hilore_block_norm_bwd_desc(rows=0, cols=64, scale=1.0)  # nothing to launch
print(E.load().hilore_block_norm_bwd(ctypes.byref(d), int(sys.argv[1]), int(sys.argv[2]), 0, None, 0, None))
"""


@pytest.mark.parametrize("code,block", [(0, 2 ** 31 - 1), (0, 2 ** 30 + 1), (1, -(2 ** 31)), (-7, -1), (2, 128), (9, 0)])
def test_code_and_block_of_bf16_units(lib, code, block):  # noqa: F811
    out = subprocess.run([sys.executable, "-c", CALL, str(code), str(block)], cwd=ROOT, capture_output=True, text=True,
                         timeout=60)
    # 5: the runtime's own complaint where there is no device
    assert out.returncode == 0 and out.stdout.strip() in ("0", "5"), (out.stdout, out.stderr[-500:])


def test_nothing_to_launch(lib):  # noqa: F811
    """No rows and no sums over rows: HILORE_OK, whatever the runtime has to say (as without a device)."""
    out = subprocess.run([sys.executable, "-c", CALL, "0", "128"], cwd=ROOT, capture_output=True, text=True, timeout=60)
    assert out.returncode == 0 and out.stdout.strip() == "0", (out.stdout, out.stderr[-500:])


def test_a_backward_without_gradients():
    """Neither dn nor dh: refused by the binding with a message, as by the library."""
    from paper_2609_33570_amd import hilore as E

    with pytest.raises(ValueError, match="dn or dh"):
        E.block_norm_bwd_desc()
