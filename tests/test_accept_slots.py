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
