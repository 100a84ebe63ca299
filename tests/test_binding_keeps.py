"""What descriptors keep alive: every tensor whose address a later call reads through them."""
import gc
import weakref

import pytest
import torch

from paper_2609_33570_amd import hilore as E


class Device:
    """A host tensor that says it is on the device."""

    is_cuda = True

    def __init__(self, *shape, dtype=torch.bfloat16):
        self.t = torch.zeros(shape, dtype=dtype)

    def __getattr__(self, name):
        return getattr(self.t, name)


def kept(make):
    """make(tensors) -> descriptor: which of the tensors outlive all but the descriptor."""
    tensors = {"h": Device(4, 64), "y": Device(4, 64), "codes": Device(4, 64, dtype=torch.uint8),
               "scales": Device(4, 2, dtype=torch.float32), "dn": Device(4, 64), "w": Device(64),
               "r": Device(4, dtype=torch.float32)}
    refs = {k: weakref.ref(t) for k, t in tensors.items()}
    desc = make(**tensors)
    del tensors
    gc.collect()
    alive = {k for k, r in refs.items() if r() is not None}
    del desc
    gc.collect()
    assert all(r() is None for r in refs.values())
    return alive


def test_saved_tensors_of_the_norm_backward():
    def rows(h, y, w, r, dn, **_):
        return E.block_norm_bwd_desc(h=E.unit_desc(x=h), y=E.unit_desc(x=y), w_pre=w, rstd_pre=r, dn=dn)

    def units(h, codes, scales, w, r, dn, **_):
        return E.block_norm_bwd_desc(h=E.unit_desc(x=h, codes=codes, scales=scales), w_pre=w, rstd_pre=r, dn=dn)

    assert kept(rows) == {"h", "y", "w", "r", "dn"}
    assert kept(units) == {"codes", "scales", "w", "r", "dn"}  # x beside codes is not read


def test_units():
    """A unit keeps what is read of it in backward; the activation it was encoded from may go."""
    assert kept(lambda h, codes, scales, **_: E.unit_desc(x=h, codes=codes, scales=scales)) == {"codes", "scales"}
    assert kept(lambda h, **_: E.unit_desc(x=h)) == {"h"}


@pytest.mark.parametrize("n", [1, 5])
def test_arrays_of_units_are_as_before(n):
    units = [E.unit_desc(x=Device(4, 64), rows=i) for i in range(n)]
    arr, count = E._desc_array(units)
    assert count == n and [arr[i].rows for i in range(n)] == list(range(n)) and arr[0].cols == 64
