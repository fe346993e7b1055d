"""A token that takes a row's whole weight gives its values, rounded once: the largest weight is exactly 1."""
import numpy as np
import pytest

import kv_shaped
import test_gpu_kv_attend as base

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

sq = base.sq

LN2 = float(np.log(2.0))


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("shape", [(2, 128, 128, ([128], [8]), ([128], [4])), (2, 64, 64, ([51, 13], [4, 8]), ([51, 13], [4, 8])),
                                   (1, 192, 192, ([187, 5], [4, 8]), ([160, 32], [2, 8]))])
@pytest.mark.parametrize("at", [0, 33, 299])
@pytest.mark.parametrize("T,group", [(1, 4), (3, 4), (40, 1), (40, 4)])
def test_a_single_weight(sq, T, group, at, shape, dtype):
    """The others' weights are below 2^-40 together; the leading score is no round number, and rises in steps."""
    context = 300
    n = context + T
    score = np.full(n, -60.0)
    score[:at] += np.linspace(0.0, 20.0, at) if at else 0.0
    score[at] = 11.37 + LN2
    p = kv_shaped.problem(sq, 97, shape, context, T, group, dtype, score, [np.zeros(n), np.full(n, 1.3)])
    out = sq.kv_attend(p.cache, p.q.cuda(), p.table, p.dlens, scale=1.0)
    assert sq.sync_status() == 0
    want = torch.from_numpy(np.repeat(p.v[0][at], group, 0)[None, None] * np.ones((1, T, 1, 1)))
    got = out.double().cpu()
    # one rounding, of a number that fp32 sums and the division leave within 2^-19
    half_ulp = 2.0 ** -11 if dtype == torch.float16 else 2.0 ** -8
    assert ((got - want).abs() <= want.abs() * (half_ulp + 2.0 ** -19) + 2.0 ** -25).all()
