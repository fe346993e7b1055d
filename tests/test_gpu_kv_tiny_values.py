"""Values far below 1 while a row's scores rise: what was summed before keeps its share."""
import numpy as np
import pytest

import kv_shaped
import test_gpu_kv_attend as base

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

sq = base.sq

ONE = (2, 128, 128, ([128], [8]), ([128], [4]))
TWO = (2, 64, 64, ([51, 13], [4, 8]), ([51, 13], [4, 8]))


@pytest.mark.parametrize("log2", [-60.0, -90.0, -100.0, -106.0])
@pytest.mark.parametrize("rise", [3.0, 12.0, 25.0])
@pytest.mark.parametrize("shape", [ONE, TWO])
@pytest.mark.parametrize("T,group", [(1, 4), (3, 4), (40, 1), (40, 4)])
def test_tiny_values_under_rising_scores(sq, T, group, shape, rise, log2):
    """Scores rise by `rise` in steps, and values get larger by as much less that early and late tokens weigh alike."""
    context = 500
    n = context + T
    step = np.floor(np.arange(n) / 70.0) / 7.0
    score = rise * step
    size = log2 + rise / np.log(2.0) * (0.7 - step)
    p = kv_shaped.problem(sq, 99, shape, context, T, group, torch.bfloat16, score, [size, size - 1.0])
    out = sq.kv_attend(p.cache, p.q.cuda(), p.table, p.dlens, scale=1.0)
    assert sq.sync_status() == 0
    kv_shaped.check_rows(p, out, None, 1.0)
