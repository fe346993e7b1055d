"""The slots of a decoding step's tokens (on the CPU)."""
from types import SimpleNamespace

import pytest
import torch

from paper_2311_14114_gb300.decode import CachedAttention

PAGE, PAGES = 16, 8
NONE = PAGE * PAGES         # beyond the cache: the library reports it


def slots(table, lengths, T):
    layer = SimpleNamespace(cache=SimpleNamespace(page_size=PAGE, n_pages=PAGES))
    return CachedAttention.slots(layer, torch.tensor(table, dtype=torch.int32), torch.tensor(lengths, dtype=torch.int32), T)


def test_tokens_follow_the_context():
    got = slots([[3, 0, 7], [1, 2, 5]], [15, 30], 4)
    assert got.tolist() == [[63, 0, 1, 2], [46, 47, 80, 81]]


def test_absent_sequences_are_skipped():
    assert slots([[3, -1]], [-1], 3).tolist() == [[-1] * 3]
    assert slots([[-5, 99]], [-7], 2).tolist() == [[-1] * 2]


def test_tokens_beyond_the_table_have_no_slot():
    assert slots([[3]], [14], 4).tolist() == [[62, 63, NONE, NONE]]
    assert slots([[3]], [2 ** 31 - 1], 2).tolist() == [[NONE, NONE]]


@pytest.mark.parametrize("page", [-1, -(2 ** 31), PAGES, 2 ** 31 - 1])
def test_tokens_in_a_page_that_is_none_have_no_slot(page):
    """A negative slot would be skipped without a word, and the token lost."""
    got = slots([[3, page, 2]], [14], 20)
    assert got[0, :2].tolist() == [62, 63] and got[0, 18:].tolist() == [32, 33]
    assert (got[0, 2:18] >= NONE).all()
