"""The slots of a plan's tokens as a step takes them (on the CPU)."""
from types import SimpleNamespace

import pytest
import torch

from paper_2311_14114_gb300 import soniq as sq
from paper_2311_14114_gb300.decode import CachedAttention

import step_plain

PAGE, PAGES = 16, 9
NONE = PAGE * PAGES         # beyond the cache: the library reports it
layer = SimpleNamespace(cache=SimpleNamespace(page_size=PAGE, n_pages=PAGES))


def plan(lengths, targets, cap, held, free):
    """A plan from its definition; held: each sequence's pages."""
    table = [row + [-1] * (6 - len(row)) for row in held]
    starts, positions, slots, after, _, _, _ = step_plain.plan(PAGE, table, free + [0] * (PAGES - len(free)), len(free), lengths, targets, cap)
    ints = lambda x, d=torch.int32: torch.tensor(x, dtype=d)
    return sq.KVStep(ints(starts), ints(positions), ints(slots, torch.int64), ints(after))


def test_absent_sequences_have_a_row():
    """Two of five are there, in buffers of a row each: the plan's list is not the step's."""
    step = plan([-1, 20, -1, 3, -1], [-1, 21, -1, 4, -1], 5, [[], [7, 2], [], [5], []], [1])
    assert step.slots.tolist() == [36, 83, -1, -1, -1]
    assert CachedAttention.planned(layer, step, 5, 1).tolist() == [[-1], [36], [-1], [83], [-1]]
    assert CachedAttention.planned(layer, step, 3, 1).tolist() == [[-1], [36], [-1]]


def test_several_tokens():
    step = plan([14, -1, 0], [17, -1, 3], 6, [[4], [], []], [8, 6])
    assert CachedAttention.planned(layer, step, 3, 3).tolist() == [[78, 79, 96], [-1] * 3, [128, 129, 130]]


def test_sequences_that_wait():
    """The pool holds one page: the second that needs one waits, what needs none does not."""
    step = plan([16, 32, 5], [18, 34, 7], 6, [[0], [1, 2], [3]], [4])
    assert step.lengths.tolist() == [18, 32, 7]
    assert CachedAttention.planned(layer, step, 3, 2).tolist() == [[64, 65], [-1, -1], [53, 54]]
    # and those whose tokens do not fit the buffers
    step = plan([1, 1, 1], [3, 3, 3], 3, [[0], [1], [2]], [])
    assert CachedAttention.planned(layer, step, 3, 2).tolist() == [[1, 2], [-1, -1], [-1, -1]]


def test_other_numbers_of_tokens_are_reported():
    step = plan([1, 4, 2], [2, 9, 5], 9, [[0], [1], [2]], [])
    assert CachedAttention.planned(layer, step, 3, 3).tolist() == [[NONE] * 3, [NONE] * 3, [34, 35, 36]]


def test_nothing_planned():
    step = plan([3, -1], [3, -1], 0, [[0], []], [])
    assert CachedAttention.planned(layer, step, 2, 2).tolist() == [[-1, -1]] * 2


def test_refusals():
    step = plan([3, -1], [4, -1], 2, [[0], []], [])
    with pytest.raises(ValueError):
        CachedAttention.planned(layer, step, 3, 1)
    x = torch.zeros(2, 3, 8, dtype=torch.float16)
    for slots in (torch.zeros(5, dtype=torch.int64), torch.zeros(2, 2, dtype=torch.int64)):
        with pytest.raises(ValueError):
            CachedAttention.step(layer, x, torch.zeros(2, 2, dtype=torch.int32), torch.zeros(2, dtype=torch.int32), slots=slots)
