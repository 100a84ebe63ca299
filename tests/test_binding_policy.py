"""What the binding of the policy loss makes of its arguments, on the host."""
import pytest
import torch

from paper_2609_33570_amd import hilore as E
from test_abi_actor import f, i
from test_binding_keeps import Device


class Offsets(Device):
    def __init__(self, *values):
        self.t = torch.tensor(values)


def packed(n, count, adv, **kw):
    return E.policy_loss_desc(f(n), f(n), f(adv), offsets=i(count + 1), **kw)


def test_as_many_sequences_as_tokens():
    """Some may be empty, so that neither reading of adv is the other: it has to be said."""
    with pytest.raises(ValueError, match="adv_per_token"):
        packed(4, 4, 4)
    assert packed(4, 4, 4, adv_per_token=True).adv_per_token == 1
    assert packed(4, 4, 4, adv_per_token=False).adv_per_token == 0
    assert packed(4, 4, 4, ratio="sequence").adv_per_token == 0  # takes no other
    assert packed(0, 0, 0).adv_per_token == 0
    # rows of one token: both are the same
    assert E.policy_loss_desc(f(4), f(4), f(4), sequences=4).adv_per_token == 0
    assert E.policy_loss_desc(f(4, 1), f(4, 1), f(4)).adv_per_token == 0


def test_sizes_that_differ_say_it():
    assert packed(6, 4, 4).adv_per_token == 0 and packed(6, 4, 6).adv_per_token == 1
    assert packed(6, 4, 4, adv_per_token=False).adv_per_token == 0 and packed(6, 4, 6, adv_per_token=True).adv_per_token == 1
    for adv, per_token in ((4, True), (6, False), (5, None), (5, True)):
        with pytest.raises(ValueError, match="adv needs"):
            packed(6, 4, adv, adv_per_token=per_token)


def test_flags_are_no_truth_values():
    """They have two bits: 2 or 3 in a bool tensor would be no value of its type."""
    def flags(dtype):
        return E.policy_loss_desc(f(3, 4), f(3, 4), f(3), flags=Device(12, dtype=dtype))

    with pytest.raises(TypeError, match="flags"):
        flags(torch.bool)
    assert flags(torch.uint8).flags
    assert E.policy_loss_desc(f(3, 4), f(3, 4), f(3), mask=Device(12, dtype=torch.bool)).mask


def test_packed_sequences_of_one_token_each():
    """Both readings are the same, unless one is empty and another has two tokens."""
    assert E.policy_loss_desc(f(4), f(4), f(4), offsets=Offsets(0, 1, 2, 3, 4)).adv_per_token == 0
    for offsets in (Offsets(0, 2, 2, 4, 4), Offsets(0, 1, 2, 4, 4), Offsets(0, 0, 1, 2, 3), Offsets(1, 2, 3, 4, 4)):
        with pytest.raises(ValueError, match="adv_per_token"):
            E.policy_loss_desc(f(4), f(4), f(4), offsets=offsets)
