"""Queries near the end of bf16's range: the token with the largest score takes the whole weight."""
import numpy as np
import pytest

import test_gpu_kv_attend as base

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

sq = base.sq


@pytest.mark.parametrize("log2", [60, 105, 118, 119])
@pytest.mark.parametrize("shape", [(2, 128, 128, ([128], [8]), ([128], [4])), (2, 64, 64, ([51, 13], [2, 8]), ([64], [8]))])
@pytest.mark.parametrize("T,group", [(1, 4), (3, 4), (40, 1), (40, 4)])
def test_large_queries(sq, T, group, shape, log2):
    p = base.Problem(sq, 98, shape, [200], T, group, 16, torch.bfloat16)
    p.q = torch.clamp(p.q.double(), -4.0, 4.0).mul(2.0 ** log2).to(torch.bfloat16)
    out = sq.kv_attend(p.cache, p.q.cuda(), p.table, p.dlens)
    assert sq.sync_status() == 0
    got, q = out.double().cpu().numpy(), p.q.double().numpy()
    assert np.isfinite(got).all()
    for t in range(T):
        for h in range(q.shape[2]):
            k, v = p.k[0][:201 + t, h // group], p.v[0][:201 + t, h // group]
            s = k @ q[0, t, h]
            assert np.abs(s).max() < np.finfo(np.float32).max        # fp32 holds the products
            order = np.argsort(s)
            # fp32 tells the two largest scores apart (a row where it may not is left out)
            if s[order[-1]] - s[order[-2]] < 2.0 ** -18 * np.abs(q[0, t, h]).sum() * np.abs(k).max():
                continue
            want = v[order[-1]]
            assert (np.abs(got[0, t, h] - want) <= np.abs(want) * (2.0 ** -8 + 2.0 ** -19)).all()
