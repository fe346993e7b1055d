"""Values near the end of bf16's range: sums of them are formed, their average is representable."""
import numpy as np
import pytest

import kv_shaped
import test_gpu_kv_attend as base

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

sq = base.sq

ONE = (1, 64, 64, ([64], [8]), ([64], [4]))
TWO = (1, 64, 64, ([51, 13], [4, 8]), ([51, 13], [4, 8]))


@pytest.mark.parametrize("T,group", [(1, 4), (4, 4), (40, 1), (40, 4)])
@pytest.mark.parametrize("context", [0, 90, 400, 3000])
@pytest.mark.parametrize("shape", [ONE, TWO])
def test_large_values_do_not_overflow(sq, shape, context, T, group):
    n = context + T
    size = np.full(n, 127.9)
    p = kv_shaped.problem(sq, 61, shape, context, T, group, torch.bfloat16, np.zeros(n), [size, size])
    out = sq.kv_attend(p.cache, p.q.cuda(), p.table, p.dlens, scale=1.0)
    kv_shaped.check_rows(p, out, None, 1.0)
    assert sq.sync_status() == 0


@pytest.mark.parametrize("T,group", [(1, 4), (40, 1), (40, 4)])
def test_infinite_values_count_as_the_largest(sq, T, group):
    """Written infinities are the type's largest finite value; so is the average of nothing else."""
    context = 130
    n = context + T
    p = kv_shaped.problem(sq, 62, ONE, context, T, group, torch.bfloat16, np.zeros(n), [np.zeros(n)])
    v = torch.full((n, 1, 64), float("-inf"), dtype=torch.bfloat16)
    k = torch.zeros(n, 1, 64, dtype=torch.bfloat16)
    sq.kv_write(p.cache, k.cuda(), v.cuda(), p.slots)
    p.k, p.v = [np.zeros((n, 1, 64))], [base.plain.values(p.cache.v, v.double().numpy(), torch.bfloat16)]
    out = sq.kv_attend(p.cache, p.q.cuda(), p.table, p.dlens, scale=1.0)
    kv_shaped.check_rows(p, out, None, 1.0)
