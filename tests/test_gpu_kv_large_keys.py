"""Keys near the end of the type's range, written infinities among them: scores that fp32 holds give their softmax."""
import numpy as np
import pytest

import test_gpu_kv_attend as base

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

sq = base.sq


@pytest.mark.parametrize("dtype,value", [(torch.float16, np.inf), (torch.bfloat16, 2.0 ** 105), (torch.bfloat16, -2.0 ** 120),
                                         (torch.bfloat16, np.inf), (torch.bfloat16, -np.inf)])
@pytest.mark.parametrize("shape", [0, 1, 6])
@pytest.mark.parametrize("at", [0, 70, 299])
@pytest.mark.parametrize("T,group", [(3, 4), (40, 1), (40, 4)])
def test_one_large_key(sq, T, group, at, shape, dtype, value):
    """Half of the rows give all their weight to the token with the large key, the others none."""
    context, page = 300, 16
    p = base.Problem(sq, 95, base.LAYOUTS[shape], [context], T, group, page, dtype)
    c, n = p.cache, context + T
    channel = 3
    sign = np.where(np.arange(T * c.heads * group).reshape(1, T, -1) % 2 == 0, 1.0, -1.0)
    p.q[..., channel] = torch.from_numpy(0.5 * sign).to(dtype)
    rng = np.random.default_rng(96)
    k, v = base.rows(rng, n, c.heads, c.k.D, dtype), base.rows(rng, n, c.heads, c.v.D, dtype)
    k[at] = 0.0
    k[at, :, channel] = value
    pos = np.arange(n)
    table = p.table[0].cpu().numpy()
    sq.kv_write(c, k.cuda(), v.cuda(), torch.from_numpy(table[pos // page].astype(np.int64) * page + pos % page).cuda())
    kk, vv = (base.plain.values(lay, x.double().numpy(), dtype) for lay, x in ((c.k, k), (c.v, v)))
    out = sq.kv_attend(c, p.q.cuda(), p.table, p.dlens)
    assert sq.sync_status() == 0
    got = out.double().cpu().numpy()
    assert np.isfinite(got).all()
    takes = sign * np.sign(value) > 0
    # all weight on one token: its value, rounded as a product with a weight of 1 and once more at the end
    want = np.repeat(vv[at], group, 0)[None, None] * np.ones((1, T, 1, 1))
    half_ulp = 2.0 ** -11 if dtype == torch.float16 else 2.0 ** -8
    assert (np.abs(got - want) <= np.abs(want) * (2.0 ** -10 + half_ulp) + 2.0 ** -24)[takes].all()
    # none: as if the token were not there
    rest = np.arange(n) != at
    o, mag, ds, total = base.plain.attend(p.q.double().numpy(), [kk[rest]], [vv[rest]], [context - 1], None, group, c.k.D ** -0.5)
    tol = base.plain.tolerance(o, mag, ds, total, n, np.abs(vv).max(), dtype)
    assert (np.abs(got - o) <= tol)[~takes].all()
