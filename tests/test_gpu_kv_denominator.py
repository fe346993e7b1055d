"""The softmax sum counts every visible token, whatever its value's size."""
import numpy as np
import pytest

import kv_shaped
import test_gpu_kv_attend as base

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

sq = base.sq

ONE = (2, 128, 128, ([128], [8]), ([128], [4]))
TWO = (2, 128, 128, ([96, 32], [4, 8]), ([96, 32], [4, 8]))
LN2 = float(np.log(2.0))


def where(n, blocks, keep):
    """True for the tokens of 64-token blocks whose number modulo `blocks` is in `keep`."""
    return np.isin(np.arange(n) // 64 % blocks, keep)


@pytest.mark.parametrize("T,group", [(3, 2), (40, 1), (40, 4)])
@pytest.mark.parametrize("dtype,log2", [(torch.float16, 15), (torch.bfloat16, 30), (torch.bfloat16, 100)])
@pytest.mark.parametrize("shape", [ONE, TWO])
@pytest.mark.parametrize("blocks,keep", [(4, (0, 1)), (2, (0,)), (3, (1, 2))])
def test_blocks_of_zero_values_count(sq, blocks, keep, shape, dtype, log2, T, group):
    """Large values, then blocks of exact zeros whose tokens together weigh about a tenth as much as the first token."""
    context = 400
    n = context + T
    score = np.full(n, -11.0 * LN2)
    score[0] = score[70] = 0.0
    size = np.where(where(n, blocks, keep), float(log2), -np.inf)
    p = kv_shaped.problem(sq, 51, shape, context, T, group, dtype, score, [size, size])
    base.run(sq, p, scale=1.0)


@pytest.mark.parametrize("T,group", [(3, 2), (40, 1), (40, 4)])
@pytest.mark.parametrize("dtype,log2", [(torch.float16, 15), (torch.bfloat16, 40)])
@pytest.mark.parametrize("zero", [0, 1])
def test_a_group_of_zeros_leaves_the_other(sq, zero, dtype, log2, T, group):
    """One value group is large first and zero later, the other holds values of ordinary size throughout."""
    context = 400
    n = context + T
    score = np.full(n, -11.0 * LN2)
    score[0] = score[70] = 0.0
    size = [np.zeros(n), np.zeros(n)]
    size[zero] = np.where(where(n, 4, (0, 1)), float(log2), -np.inf)
    p = kv_shaped.problem(sq, 52, TWO, context, T, group, dtype, score, size)
    out = base.run(sq, p, scale=1.0)
    # the bound above grows with the larger group; the other one alone, at its own size
    o, mag, ds, total = base.plain.attend(p.q.double().numpy(), p.k, p.v, p.lens, None, group, 1.0)
    got = out.double().cpu().numpy()
    for h in range(p.cache.heads):
        at, count, _ = base.plain.groups(p.cache.v)[1 - zero]
        ch = p.cache.v.perm_host[h][at:at + count]
        rows = slice(h * group, (h + 1) * group)
        tol = base.plain.tolerance(o, mag, ds, total, n, np.abs(p.v[0][:, h, ch]).max(), dtype)
        assert (np.abs(got - o)[:, :, rows][..., ch] <= tol[:, :, rows][..., ch]).all()


@pytest.mark.parametrize("T,group", [(3, 2), (40, 1), (40, 4)])
@pytest.mark.parametrize("dtype,log2", [(torch.float16, 15), (torch.bfloat16, 100)])
def test_a_page_outside_the_cache_counts_as_zeros(sq, dtype, log2, T, group):
    """Its 64 keys are zero and weigh 2^-12 of the first token, each; its values add nothing."""
    context, page = 400, 64
    n = context + T
    score = np.full(n, -20.0 * LN2)
    score[0] = 12.0 * LN2
    p = kv_shaped.problem(sq, 53, ONE, context, T, group, dtype, score, [np.full(n, float(log2))], page)
    p.table[0, 2] = p.cache.n_pages
    p.k[0][128:192] = 0.0
    p.v[0][128:192] = 0.0
    out = sq.kv_attend(p.cache, p.q.cuda(), p.table, p.dlens, scale=1.0)
    assert sq.sync_status() == sq.SONIQ_ERR_INVALID_ARG
    p.check(out, None, 1.0)
