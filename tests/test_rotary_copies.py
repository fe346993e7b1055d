"""Copies and pickles of a rotation refer to their own memory (on the CPU)."""
import copy
import pickle

import pytest
import torch

from paper_2311_14114_gb300 import soniq as sq


@pytest.mark.parametrize("again", [copy.copy, copy.deepcopy, lambda r: pickle.loads(pickle.dumps(r))])
@pytest.mark.parametrize("channels", [8, 0])
def test_copies(again, channels):
    r = sq.Rotary(channels, base=500.0, interleaved=True, scaling=("linear", 2.0), magnitude=1.5, device="cpu")
    other = again(r)
    assert torch.equal(other.turns, r.turns) and other.frequencies == r.frequencies
    assert (other.c.channels, other.c.interleaved, other.c.magnitude) == (channels, 1, 1.5)
    assert other.c is not r.c and other.c.turns == (other.turns.data_ptr() if channels else None)
    assert r.c.turns == (r.turns.data_ptr() if channels else None)


def test_a_module_that_holds_one():
    class Layer(torch.nn.Module):
        def __init__(self):
            super().__init__()
            self.rotary = sq.Rotary(4, device="cpu")

    a = Layer()
    b = copy.deepcopy(a)
    assert b.rotary.c.turns == b.rotary.turns.data_ptr() != a.rotary.c.turns
