"""How the attention kernels share work among CTAs: sequences without work, many
short items beside long ones, items in one part and in many, on both kernels."""
import numpy as np
import pytest

import test_gpu_kv_attend as base

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

sq = base.sq


def attend_into_nan(sq, p, mask=None):
    out = torch.full(p.q.shape[:3] + (p.cache.v.D,), float("nan"), dtype=p.cache.dtype, device="cuda")
    m = None if mask is None else torch.from_numpy(mask).cuda()
    got = sq.kv_attend(p.cache, p.q.cuda(), p.table, p.dlens, mask=m, out=out)
    assert got.data_ptr() == out.data_ptr()
    p.check(out, mask, p.cache.k.D ** -0.5)
    assert sq.sync_status() == 0
    return out


@pytest.mark.parametrize("T,group", [(1, 4), (40, 4), (70, 2)])
@pytest.mark.parametrize("lens", [[-1], [-1] * 9, [-1] * 5 + [40] + [-3] * 200, [0] + [-1] * 170])
def test_absent_sequences_are_written(sq, lens, T, group):
    """Zeros for absent sequences whichever CTAs have other work, none of them included."""
    p = base.Problem(sq, 41, base.LAYOUTS[0], lens, T, group, 16, torch.float16)
    attend_into_nan(sq, p)


@pytest.mark.parametrize("shape", [0, 1])
@pytest.mark.parametrize("T,group", [(1, 8), (13, 1), (24, 4), (64, 4)])
def test_short_items_beside_long_ones(sq, shape, T, group):
    rng = np.random.default_rng(42 + T)
    lens = [int(n) for n in rng.integers(0, 90, 60)]
    lens[7], lens[33], lens[59] = 2600, 1900, 1111
    p = base.Problem(sq, 42, base.LAYOUTS[shape], lens, T, group, 32, torch.float16)
    mask = base.tree(p.rng, len(lens), T)
    first = attend_into_nan(sq, p, mask)
    assert torch.equal(first, attend_into_nan(sq, p, mask))


@pytest.mark.parametrize("T,group", [(1, 4), (24, 4), (64, 8)])
@pytest.mark.parametrize("length", [63, 64, 65, 255, 1000, 6000])
def test_items_in_parts(sq, length, T, group):
    p = base.Problem(sq, 43, base.LAYOUTS[0], [length], T, group, 64, torch.bfloat16)
    attend_into_nan(sq, p)


def test_one_group_a_side_over_long_contexts(sq):
    """Two score buffers, many blocks: the outputs are the same bits every time."""
    rng = np.random.default_rng(44)
    perm = np.stack([rng.permutation(128) for _ in range(2)])
    lay = sq.KVLayout(perm, (128, 0), (4, 8))
    cache = sq.KVCache(lay, lay, 80, 64)
    n = 80 * 64 - 64
    k, v = (torch.from_numpy(rng.standard_normal((n + 64, 2, 128)).astype(np.float16)).cuda() for _ in range(2))
    sq.kv_write(cache, k, v, torch.arange(n + 64, device="cuda"))
    q = torch.from_numpy(rng.standard_normal((1, 64, 16, 128)).astype(np.float16)).cuda()
    table = torch.arange(80, dtype=torch.int32, device="cuda").view(1, 80)
    lens = torch.tensor([n], dtype=torch.int32, device="cuda")
    first = sq.kv_attend(cache, q, table, lens)
    for _ in range(20):
        assert torch.equal(sq.kv_attend(cache, q, table, lens), first)
    assert sq.sync_status() == 0
    kk, vv = (base.plain.values(lay, t.double().cpu().numpy(), torch.float16) for t in (k, v))
    for t in (0, 31, 63):      # a row of the chain alone: one token over a context of n + t
        o, mag, ds, total = base.plain.attend(q[:, t:t + 1].double().cpu().numpy(), [kk[:n + t + 1]], [vv[:n + t + 1]], [n + t], None, 8,
                                              128 ** -0.5)
        tol = base.plain.tolerance(o, mag, ds, total, n + t + 1, np.abs(vv).max(), torch.float16)
        assert (np.abs(first[:, t:t + 1].double().cpu().numpy() - o) <= tol).all()


@pytest.mark.parametrize("T,group", [(40, 4), (9, 16)])
@pytest.mark.parametrize("shape", [(1, 256, 64, ([256], [2]), ([64], [4])), (2, 256, 128, ([256], [4]), ([128], [4])),
                                   (1, 256, 128, ([256], [4]), ([128], [8])), (1, 256, 256, ([192, 64], [4, 8]), ([256], [8]))])
def test_many_rows_of_wide_heads(sq, shape, T, group):
    """More than 128 rows per key head of 256 channels: two tiles of queries leave no room for a ring of operands."""
    p = base.Problem(sq, 45, shape, [0, 130, 777], T, group, 16, torch.float16)
    attend_into_nan(sq, p)
