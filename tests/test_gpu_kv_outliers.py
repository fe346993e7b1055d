"""A token's large value disturbs no row that gives it little weight, or none."""
import numpy as np
import pytest

import kv_shaped
import test_gpu_kv_attend as base

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

sq = base.sq

F16, BF16 = torch.float16, torch.bfloat16
LN2 = float(np.log(2.0))
TOP = {F16: 65504.0, BF16: float(torch.finfo(BF16).max)}

ONE = (2, 128, 128, ([128], [8]), ([128], [4]))
MIXED = (2, 128, 128, ([96, 32], [4, 8]), ([128], [4]))
TWO = (2, 64, 64, ([51, 13], [4, 8]), ([51, 13], [4, 8]))
WIDE = (1, 192, 192, ([187, 5], [4, 8]), ([160, 32], [2, 8]))       # values that no tile kernel takes
SHAPES = [ONE, MIXED, TWO, WIDE]
# T, group: 4 and 12 query rows per key head, and 40, 160 and 264
FEW = [(4, 1), (3, 4)]
MANY = [(40, 1), (40, 4), (33, 8)]


def attend(sq, p, mask=None, scale=None):
    m = None if mask is None else torch.from_numpy(mask).cuda()
    out = sq.kv_attend(p.cache, p.q.cuda(), p.table, p.dlens, mask=m, scale=scale)
    assert sq.sync_status() == 0
    return out


@pytest.mark.parametrize("dtype,poison", [(F16, 4096.0), (F16, TOP[F16]), (BF16, 2.0 ** 100), (BF16, TOP[BF16])])
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("T,group", FEW + MANY)
def test_hidden_drafts_of_any_size(sq, T, group, shape, dtype, poison):
    """A draft that no row sees, in contexts of none, one and several blocks."""
    p = base.Problem(sq, 71, shape, [70, 0, 400], T, group, 16, dtype)
    m = base.tree(p.rng, 3, T)
    m[:, :, 2] = False
    for b in range(3):
        pos = int(p.lens[b]) + 2
        page, at = int(p.table[b, pos // 16]), pos % 16
        for codes, scales in ((p.cache.k_codes, p.cache.k_scales), (p.cache.v_codes, p.cache.v_scales)):
            codes[page, :, at] = 0x81
            scales[page, :, at] = poison
    kv_shaped.check_rows(p, attend(sq, p, m), m, p.cache.k.D ** -0.5)


@pytest.mark.parametrize("dtype,log2", [(F16, 15), (BF16, 60), (BF16, 127)])
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("T,group", FEW[:1] + MANY[:2])
def test_a_draft_disturbs_only_its_own_rows(sq, T, group, shape, dtype, log2):
    """Draft 1's values are large; it sees itself, the others do not see it."""
    context = 70
    n = context + T
    size = np.zeros(n)
    size[context + 1] = log2
    p = kv_shaped.problem(sq, 72, shape, context, T, group, dtype, p_scores(n), [size, size])
    m = np.tril(np.ones((1, T, T), dtype=bool))
    m[0, 2:, 1] = False
    kv_shaped.check_rows(p, attend(sq, p, m, 1.0), m, 1.0)


def p_scores(n):
    return np.random.default_rng(n).standard_normal(n)


# tokens of size 2^log2 weigh 2^-weight of the others'
@pytest.mark.parametrize("dtype,log2,weight", [(F16, 12, 20), (F16, 15, 24), (BF16, 40, 48), (BF16, 100, 110), (BF16, 127, 130)])
@pytest.mark.parametrize("at", [(0,), (5, 66, 130), (399,)])
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("T,group", [(1, 4), (3, 4)] + MANY[:2])
def test_large_values_of_little_weight(sq, T, group, shape, at, dtype, log2, weight):
    context = 400
    n = context + T
    score, size = p_scores(n), np.zeros(n)
    for t in at:
        score[t], size[t] = -weight * LN2, log2
    p = kv_shaped.problem(sq, 73, shape, context, T, group, dtype, score, [size, size])
    kv_shaped.check_rows(p, attend(sq, p, None, 1.0), None, 1.0)


# the token that takes the weight has small values, or none
@pytest.mark.parametrize("log2", [-np.inf, -8.0])
@pytest.mark.parametrize("dtype,lead", [(F16, 18), (BF16, 18), (BF16, 60)])
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("at", [0, 70, 399])
@pytest.mark.parametrize("T,group", [(1, 4)] + MANY[:2])
def test_small_values_of_much_weight(sq, T, group, at, shape, dtype, lead, log2):
    context = 400
    n = context + T
    score, size = p_scores(n), np.full(n, 12.0)
    score[at], size[at] = lead * LN2, log2
    p = kv_shaped.problem(sq, 74, shape, context, T, group, dtype, score, [size, size])
    kv_shaped.check_rows(p, attend(sq, p, None, 1.0), None, 1.0)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("T,group", [(1, 4)] + MANY[:2])
def test_sizes_that_rise_and_fall(sq, T, group, dtype):
    """Scores and sizes that climb by more than fp16's range, and fall, over a context in many parts."""
    context = 3000
    n = context + T
    t = np.arange(n)
    for score in (t * 0.02, -t * 0.02, 20.0 * np.sin(t / 300.0)):
        for size in (6.0 * np.cos(t / 200.0), 8.0 * np.sign(np.sin(t / 77.0))):
            p = kv_shaped.problem(sq, 75, TWO, context, T, group, dtype, score, [size, -size], 64)
            kv_shaped.check_rows(p, attend(sq, p, None, 1.0), None, 1.0)
