"""Lengths up to the largest 32-bit number: what the page table holds is seen, and the call reports them."""
import numpy as np
import pytest

import test_gpu_kv_attend as base

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

sq = base.sq


@pytest.mark.parametrize("length", [10 ** 6, 2 ** 31 - 65, 2 ** 31 - 2, 2 ** 31 - 1])
@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("T,group", [(1, 4), (4, 4), (40, 1), (64, 4)])
def test_lengths_beyond_the_table(sq, T, group, masked, length):
    tokens, page = 208, 16
    p = base.Problem(sq, 91, base.LAYOUTS[0], [tokens - T], T, group, page, torch.float16)
    table = p.table[:, :tokens // page].contiguous()
    lens = torch.full((1,), length, dtype=torch.int32, device="cuda")
    # nothing of the drafts is within the table, so the mask hides nothing
    mask = torch.zeros(1, T, T, dtype=torch.bool, device="cuda") if masked else None
    out = sq.kv_attend(p.cache, p.q.cuda(), table, lens, mask=mask)
    assert sq.sync_status() == sq.SONIQ_ERR_INVALID_ARG and sq.sync_status() == 0
    p.check(out, np.ones((1, T, T), dtype=bool), p.cache.k.D ** -0.5)
