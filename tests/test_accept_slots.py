"""Where accept() puts the rows of accepted drafts (on the CPU; the write itself is recorded)."""
from types import SimpleNamespace

import pytest
import torch

from paper_2311_14114_gb300 import decode
from paper_2311_14114_gb300.decode import CachedAttention

PAGE, PAGES = 16, 8
NONE = PAGE * PAGES


@pytest.fixture
def accept(monkeypatch):
    def run(at, path, table, lengths):
        """at: the slots that the step used.  Returns where each draft's row goes, and the new lengths."""
        net, wrote = object.__new__(CachedAttention), []
        monkeypatch.setattr(decode.sq, "kv_write", lambda cache, k, v, slots: wrote.append(slots))
        net.cache = SimpleNamespace(page_size=PAGE, n_pages=PAGES)
        net.at = torch.tensor(at)
        net.k = net.v = torch.zeros(*net.at.shape, 1, 8)
        new = net.accept(torch.tensor(path), torch.tensor(table, dtype=torch.int32), torch.tensor(lengths, dtype=torch.int32))
        assert new.dtype == torch.int32 and wrote[0].is_contiguous()
        return wrote[0].view(net.at.shape).tolist(), new.tolist()
    return run


def test_accepted_rows_follow_the_context(accept):
    to, new = accept([[46, 47, 80, 81]], [[0, 2, 3]], [[0, 2, 5]], [30])
    assert to == [[46, -1, 47, 80]] and new == [33]


@pytest.mark.parametrize("T", [1, 2, 5])
def test_slots_are_contiguous(accept, T):
    """As the write wants them, also those of a step of one token."""
    to, new = accept([list(range(T)), list(range(32, 32 + T))], [[0], [0]], [[0], [2]], [0, 0])
    assert [r[0] for r in to] == [0, 32] and new == [1, 1]


def test_a_waiting_sequence_keeps_its_length_and_writes_nothing(accept):
    """Its table still names the page that it gave back, which sequence 1 holds by now."""
    to, new = accept([[-1, -1], [49, 50]], [[0, 1], [0, -1]], [[0, 1, 3], [2, 4, 3]], [32, 33])
    assert to == [[-1, -1], [49, -1]] and new == [32, 34]


def test_absent_and_beginning_sequences(accept):
    to, new = accept([[-1, -1], [16, 17], [16, 17]], [[-1, -1], [1, -1], [-1, -1]], [[7], [1], [1]], [-1, -1, 0])
    assert to == [[-1, -1], [-1, 16], [-1, -1]] and new == [-1, 1, 0]


def test_in_two_calls(accept):
    """Drafts accepted one after the other: each call's lengths say where they go."""
    at = [[46, 47, 80]]
    assert accept(at, [[1]], [[0, 2, 5]], [30]) == ([[-1, 46, -1]], [31])
    assert accept(at, [[2]], [[0, 2, 5]], [31]) == ([[-1, -1, 47]], [32])


def test_beyond_the_table(accept):
    """Reported by the write, as the step's own was."""
    to, new = accept([[63, NONE, NONE]], [[0, 1]], [[3]], [15])
    assert to == [[63, NONE, -1]] and new == [17]
