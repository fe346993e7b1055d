"""Attention over the quantized cache against its definition in fp64."""
import numpy as np
import pytest
import torch

import kv_plain as plain
from test_gpu_kv_cache import LAYOUTS, make_cache, rows

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sq():
    from paper_2311_14114_gb300 import soniq
    return soniq


def tree(rng, B, T):
    m = np.zeros((B, T, T), dtype=bool)
    for b in range(B):
        for i in range(T):
            p = int(rng.integers(-1, i))
            if p >= 0:
                m[b, i] = m[b, p]
            m[b, i, i] = True
    return m


class Problem:
    """Sequences in randomly ordered pages; what no sequence shows is filled with
    bytes that decode to NaN or infinite scales."""

    def __init__(self, sq, seed, shape, lens, T, group, page, dtype, gain=1.0, vgain=1.0):
        rng = self.rng = np.random.default_rng(seed)
        heads, D, Dv = shape[:3]
        self.lens, self.T, self.group, self.B = np.asarray(lens), T, group, len(lens)
        need = [0 if n < 0 else -(-(n + T) // page) for n in lens]
        n_pages = sum(need) + 2
        self.cache = c = make_cache(sq, rng, shape, n_pages, page, dtype)
        for codes in (c.k_codes, c.v_codes):
            codes.copy_(torch.from_numpy(rng.integers(0, 256, codes.shape, dtype=np.uint8)))
        c.k_scales.fill_(float("nan"))
        c.v_scales.fill_(float("inf"))
        order = rng.permutation(n_pages)
        table = rng.integers(-2 ** 31, 2 ** 31, (self.B, max(need + [0]) + 1)).astype(np.int32)
        self.k, self.v, at = [], [], 0
        for b, n in enumerate(lens):
            m = max(n, 0) + T if n >= 0 else 0
            pages = order[at:at + need[b]]
            table[b, :need[b]] = pages
            at += need[b]
            k, v = rows(rng, m, heads, D, dtype) * gain, rows(rng, m, heads, Dv, dtype) * vgain
            k, v = k.to(dtype), v.to(dtype)
            pos = np.arange(m)
            slots = torch.from_numpy((pages[pos // page] * page + pos % page).astype(np.int64) if m else pos).cuda()
            sq.kv_write(c, k.cuda(), v.cuda(), slots)
            self.k.append(plain.values(c.k, k.double().numpy(), dtype))
            self.v.append(plain.values(c.v, v.double().numpy(), dtype))
        self.table = torch.from_numpy(table).cuda()
        self.dlens = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.q = rows(rng, self.B * T, heads * group, D, dtype).view(self.B, T, heads * group, D)

    def check(self, out, mask, scale):
        o, mag, ds, total = plain.attend(self.q.double().numpy(), self.k, self.v, self.lens, mask, self.group, scale)
        v_max = max([np.abs(v).max() for v in self.v if v.size] + [0.0])
        n_seen = max(int(self.lens.max()), 0) + self.T
        tol = plain.tolerance(o, mag, ds, total, n_seen, v_max, self.cache.dtype)
        got = out.double().cpu().numpy()
        assert np.isfinite(got).all()
        err = np.abs(got - o)
        assert (err <= tol).all(), (float((err / tol).max()), np.unravel_index((err / tol).argmax(), err.shape))


def run(sq, p, mask=None, scale=None):
    m = None if mask is None else torch.from_numpy(mask).cuda()
    out = sq.kv_attend(p.cache, p.q.cuda(), p.table, p.dlens, mask=m, scale=scale)
    p.check(out, mask, p.cache.k.D ** -0.5 if scale is None else scale)
    assert sq.sync_status() == 0
    return out


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("shape", LAYOUTS)
@pytest.mark.parametrize("group", [1, 4])
def test_layouts(sq, shape, group, dtype):
    p = Problem(sq, 11, shape, [70, 0, 33], 3, group, 16, dtype)
    run(sq, p, tree(p.rng, 3, 3))


@pytest.mark.parametrize("length", [0, 1, 15, 16, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 1000])
@pytest.mark.parametrize("page", [16, 64, 256])
def test_one_token_lengths(sq, length, page):
    p = Problem(sq, length, LAYOUTS[0], [length], 1, 4, page, torch.float16)
    run(sq, p)


@pytest.mark.parametrize("T", [1, 2, 5, 8, 9, 16, 17, 31, 33, 64])
@pytest.mark.parametrize("group", [1, 2, 5, 8])
def test_trees(sq, T, group):
    p = Problem(sq, T, (2, 64, 64, ([51, 13], [4, 8]), ([64], [4])), [97, 40], T, group, 32, torch.bfloat16)
    run(sq, p, tree(p.rng, 2, T))


@pytest.mark.parametrize("T,group", [(1, 1), (7, 3), (65, 2), (200, 1), (130, 4)])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_chains(sq, T, group, dtype):
    p = Problem(sq, T, (2, 128, 128, ([112, 16], [4, 8]), ([128], [4])), [70, 0], T, group, 64, dtype)
    run(sq, p)


@pytest.mark.parametrize("group", [1, 8])
def test_ragged_batch_with_absent_sequences(sq, group):
    lens = [0, 511, -1, 3, 64, 1200, 31, -7, 90]
    p = Problem(sq, 21, LAYOUTS[1], lens, 1, group, 32, torch.float16)
    out = run(sq, p)
    assert not out[2].any() and not out[7].any()


@pytest.mark.parametrize("T,group", [(4, 1), (40, 2)])
def test_rows_that_see_nothing(sq, T, group):
    """No context and a mask whose rows are empty: zeros, beside rows that see something."""
    p = Problem(sq, 22, LAYOUTS[0], [0, 5], T, group, 16, torch.float16)
    m = tree(p.rng, 2, T)
    m[:, 1] = False
    m[0, T - 1] = False
    out = run(sq, p, m)
    assert not out[0, 1].any() and not out[0, T - 1].any() and out[1, 1].any()
    m[:] = False
    out = run(sq, p, m)
    assert not out[0].any() and out[1].any()


@pytest.mark.parametrize("T", [3, 33])
def test_any_mask(sq, T):
    """Masks that are no trees, one for all sequences or one each."""
    p = Problem(sq, 23, LAYOUTS[2], [45, 100], T, 2, 16, torch.bfloat16)
    m = p.rng.random((2, T, T)) < 0.4
    run(sq, p, m)
    one = m[:1].repeat(2, 0)
    out = sq.kv_attend(p.cache, p.q.cuda(), p.table, p.dlens, mask=torch.from_numpy(m[0]).cuda())
    p.check(out, one, p.cache.k.D ** -0.5)


def test_long_context_is_split(sq):
    p = Problem(sq, 24, (1, 128, 128, ([96, 32], [4, 8]), ([128], [4])), [5003], 1, 8, 64, torch.float16)
    run(sq, p)
    p = Problem(sq, 25, (1, 128, 128, ([128], [4]), ([128], [4])), [4001], 16, 8, 64, torch.float16)
    run(sq, p, tree(p.rng, 1, 16))


@pytest.mark.parametrize("scale", [0.0, -0.3, 1.0])
def test_scale(sq, scale):
    p = Problem(sq, 26, LAYOUTS[0], [100], 2, 4, 16, torch.float16)
    run(sq, p, scale=scale)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("gain,vgain", [(1.0, 2.0 ** -12), (1.0, 4000.0), (20.0, 1.0), (2.0 ** -10, 1.0)])
@pytest.mark.parametrize("T", [2, 40])
def test_magnitudes(sq, T, gain, vgain, dtype):
    """Small and large values (their scales leave fp16's normal range without normalisation), peaked and flat softmax."""
    p = Problem(sq, 27, LAYOUTS[0], [300], T, 2, 16, dtype, gain, vgain)
    run(sq, p)


def test_bf16_beyond_fp16_range(sq):
    for vgain in (1e30, 1e-30):
        p = Problem(sq, 28, LAYOUTS[0], [150, 20], 2, 4, 16, torch.bfloat16, 1.0, vgain)
        run(sq, p)
        p = Problem(sq, 28, LAYOUTS[0], [150, 20], 40, 4, 16, torch.bfloat16, 1.0, vgain)
        run(sq, p)


@pytest.mark.parametrize("T", [1, 20])
def test_query_strides_and_streams(sq, T):
    p = Problem(sq, 29, LAYOUTS[0], [77, 30], T, 4, 16, torch.float16)
    q = p.q.cuda()
    want = sq.kv_attend(p.cache, q, p.table, p.dlens)
    wide = torch.full((2, T, 50, 131), float("nan"), dtype=q.dtype, device="cuda")
    wide[:, :, 5:37, 3:] = q
    assert torch.equal(sq.kv_attend(p.cache, wide[:, :, 5:37, 3:], p.table, p.dlens), want)
    heads_first = q.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)
    assert torch.equal(sq.kv_attend(p.cache, heads_first, p.table, p.dlens), want)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    out = sq.kv_attend(p.cache, q, p.table, p.dlens, stream=s)
    s.synchronize()
    assert torch.equal(out, want)


@pytest.mark.parametrize("T,n", [(1, 3000), (24, 900)])
def test_same_bits_every_time_and_in_graphs(sq, T, n):
    p = Problem(sq, 30, LAYOUTS[0], [n, n // 3], T, 4, 64, torch.float16)
    q = p.q.cuda()
    want = sq.kv_attend(p.cache, q, p.table, p.dlens)
    for _ in range(5):
        assert torch.equal(sq.kv_attend(p.cache, q, p.table, p.dlens), want)
    out = torch.empty_like(want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        sq.kv_attend(p.cache, q, p.table, p.dlens, out=out)
    for _ in range(3):
        out.zero_()
        g.replay()
        assert torch.equal(out, want)
    # lengths are read on the device: the captured call follows them
    p.dlens.fill_(n // 4)
    p.lens[:] = n // 4
    g.replay()
    direct = sq.kv_attend(p.cache, q, p.table, p.dlens)
    assert torch.equal(out, direct) and not torch.equal(out, want)


def test_bad_pages_and_lengths_are_reported(sq):
    p = Problem(sq, 31, LAYOUTS[0], [40, 20], 1, 4, 16, torch.float16)
    good = sq.kv_attend(p.cache, p.q.cuda(), p.table, p.dlens)
    table = p.table.clone()
    table[0, 1] = p.cache.n_pages
    out = sq.kv_attend(p.cache, p.q.cuda(), table, p.dlens)
    assert sq.sync_status() == sq.SONIQ_ERR_INVALID_ARG
    assert torch.equal(out[1], good[1]) and torch.isfinite(out).all()
    # the page counts as zero keys and values
    p.k[0][16:32] = 0.0
    p.v[0][16:32] = 0.0
    p.check(out, None, 128 ** -0.5)
    # a length beyond the table: what the table holds is seen
    lens = p.dlens.clone()
    lens[1] = 10 ** 6
    table = p.table[:, :1].contiguous()
    lens[0] = -1
    out = sq.kv_attend(p.cache, p.q.cuda(), table, lens)
    assert sq.sync_status() == sq.SONIQ_ERR_INVALID_ARG and sq.sync_status() == 0
    assert not out[0].any() and torch.isfinite(out).all()


def test_no_rows(sq):
    p = Problem(sq, 32, LAYOUTS[0], [40], 1, 4, 16, torch.float16)
    q = p.q.cuda()
    assert sq.kv_attend(p.cache, q[:0], p.table[:0], p.dlens[:0]).shape == (0, 1, 32, 128)
    assert sq.kv_attend(p.cache, q[:, :0], p.table, p.dlens).shape == (1, 0, 32, 128)


def test_refusals(sq):
    p = Problem(sq, 33, LAYOUTS[0], [40], 2, 4, 16, torch.float16)
    q = p.q.cuda()
    m = torch.ones(1, 2, 2, dtype=torch.bool, device="cuda")
    for kw in (dict(q=q[0]), dict(q=q.float()), dict(q=q[:, :, :31]), dict(q=q[..., :64]), dict(q=q.cpu()),
               dict(page_table=p.table.long()), dict(page_table=p.table[0]), dict(lengths=p.dlens.long()),
               dict(lengths=torch.cat([p.dlens, p.dlens])), dict(mask=m.float()), dict(mask=m[:, :1]),
               dict(mask=m.transpose(1, 2)), dict(out=torch.empty(3, dtype=q.dtype, device="cuda"))):
        args = dict(q=q, page_table=p.table, lengths=p.dlens)
        args.update(kw)
        with pytest.raises(ValueError):
            sq.kv_attend(p.cache, **args)
    with pytest.raises(sq.SoniqError):
        sq.kv_attend(p.cache, q, p.table, p.dlens, scale=float("nan"))


def test_lost_copy_is_reported(sq):
    """A copy that never comes: the bounded wait runs out, the status says so, and the next call is right."""
    p = Problem(sq, 34, LAYOUTS[0], [200, 31], 1, 4, 16, torch.float16)
    want = run(sq, p)
    sq.test_drop_barrier_arrival()
    sq.kv_attend(p.cache, p.q.cuda(), p.table, p.dlens)
    assert sq.sync_status() == sq.SONIQ_ERR_TIMEOUT
    assert torch.equal(run(sq, p), want)


def test_nan_query_stays_in_its_row(sq):
    p = Problem(sq, 35, LAYOUTS[0], [100], 3, 4, 16, torch.float16)
    want = run(sq, p)
    q = p.q.clone()
    q[0, 1, 6, 3] = float("nan")
    out = sq.kv_attend(p.cache, q.cuda(), p.table, p.dlens)
    assert torch.isnan(out[0, 1, 6]).all()
    out[0, 1, 6] = want[0, 1, 6]
    assert torch.equal(out, want)


@pytest.mark.parametrize("poison", [float("nan"), float("inf"), -1.0])
@pytest.mark.parametrize("shape", [0, 1])
@pytest.mark.parametrize("T,group", [(4, 1), (40, 4)])
def test_hidden_drafts_may_hold_anything(sq, T, group, shape, poison):
    """A draft that no row sees: whatever stands in its slot, the outputs are those without it."""
    p = Problem(sq, 36, LAYOUTS[shape], [70, 0], T, group, 16, torch.float16)
    m = tree(p.rng, 2, T)
    m[:, :, 2] = False
    run(sq, p, m)
    for b in range(2):
        pos = int(p.lens[b]) + 2
        page, at = int(p.table[b, pos // 16]), pos % 16
        for codes, scales in ((p.cache.k_codes, p.cache.k_scales), (p.cache.v_codes, p.cache.v_scales)):
            codes[page, :, at] = 0x81
            scales[page, :, at] = poison
    run(sq, p, m)
