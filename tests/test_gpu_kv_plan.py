"""Pages, slots and positions of a step on the GPU against lists worked through one
sequence after the other.  Every output is a whole number and has to be equal."""
import random

import numpy as np
import pytest

import step_plain

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def sq():
    from paper_2311_14114_gb300 import build, soniq
    build.build()
    soniq.lib()
    return soniq


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Pool:
    """A pool whose sequences hold random pages, and the same as lists."""

    def __init__(self, sq, lengths, page, spare, width, seed=0):
        rng = random.Random(seed)
        has = [min(-(-max(n, 0) // page), width) for n in lengths]
        n_pages = sum(has) + spare
        order = rng.sample(range(n_pages), n_pages)
        self.table, at = [], 0
        for h in has:
            self.table.append(order[at:at + h] + [rng.randint(-9, n_pages + 9) for _ in range(width - h)])
            at += h
        self.free, self.n_free = order[at:] + [rng.randint(-9, 9) for _ in range(at)], spare
        self.page, self.lengths = page, list(lengths)
        self.pages = sq.KVPages(max(n_pages, 1), page, len(lengths), width)
        if lengths and width:
            self.pages.table.copy_(ints(self.table))
        if n_pages:
            self.pages.free.copy_(ints(self.free))
        self.pages.count[0] = spare

    def step(self, sq, targets, cap, **kw):
        """One step on both sides, and their comparison."""
        want = step_plain.plan(self.page, self.table, self.free, self.n_free, self.lengths, targets, cap)
        got = sq.kv_plan(self.pages, ints(self.lengths), ints(targets), cap, **kw)
        torch.cuda.synchronize()
        self.compare(got, want)
        self.lengths, self.table, self.free, self.n_free = want[3], want[4], want[5], want[6]
        return got

    def compare(self, got, want):
        assert got.starts.tolist() == want[0]
        assert got.positions.tolist() == want[1]
        assert got.slots.tolist() == want[2]
        assert got.lengths.tolist() == want[3]
        assert self.pages.table.tolist() == want[4]
        if want[5]:
            assert self.pages.free.tolist() == want[5]
        assert self.pages.count.tolist() == [want[6], 0]


@pytest.mark.parametrize("B,page,new,ctx", [(1, 16, 1, 0), (1, 256, 5000, 0), (7, 64, 1, 1000), (33, 16, 40, 300),
                                            (511, 32, 3, 100), (513, 128, 70, 999), (2049, 16, 5, 64), (8192, 16, 2, 40)])
@pytest.mark.parametrize("spare", [1.0, 0.5, 0.0])
def test_random_steps(sq, B, page, new, ctx, spare):
    rng = random.Random(B * 1000 + page)
    lengths = [rng.randint(-1, ctx) for _ in range(B)]
    width = -(-(ctx + 3 * new) // page) + 1
    pool = Pool(sq, lengths, page, int(spare * (B * (new // page + 1))), width, seed=B)
    for step in range(3):
        targets = []
        for n in pool.lengths:
            what = rng.random()
            targets.append(max(n, 0) + rng.randint(1, new) if what < 0.7 else (rng.randint(0, max(n, 0)) if what < 0.9 else -1))
        tokens = sum(max(max(t, 0) - max(n, 0), 0) for n, t in zip(pool.lengths, targets))
        pool.step(sq, targets, tokens + rng.choice([0, 1, 300]) if step != 1 else tokens // 2)
    assert sq.sync_status() == 0


def test_shrinking_undoes_growing(sq):
    pool = Pool(sq, [5, -1, 100, 0, 17], 16, 40, 12)
    before = (pool.table, pool.free[:pool.n_free], pool.n_free)
    pool.step(sq, [90, 33, 101, 16, 17], 400)
    pool.step(sq, [5, -1, 100, 0, 17], 0)
    assert (pool.free[:pool.n_free], pool.n_free) == before[1:]
    assert sq.sync_status() == 0


def test_pages_given_back_are_taken_first(sq):
    pool = Pool(sq, [64, 64, -1, 3], 16, 2, 8)
    given = pool.table[0][1:4] + pool.table[1][:4]
    got = pool.step(sq, [16, -1, 48, 35], 100)
    assert pool.table[2][:3] + pool.table[3][1:3] == given[:5]
    assert got.lengths.tolist() == [16, -1, 48, 35]


def test_when_the_pool_is_too_small(sq):
    """The first that does not fit waits, and all later ones that need pages; those that need none do not."""
    pool = Pool(sq, [0, 10, 0, 10, 0, 20], 16, 3, 8)
    got = pool.step(sq, [32, 12, 33, 16, 1, 5], 200)
    assert got.lengths.tolist() == [32, 12, 0, 16, 0, 5]
    assert got.starts.tolist() == [0, 32, 34, 67, 73, 74, 74]
    assert (got.slots[34:67] == -1).all() and (got.slots[73:74] == -1).all() and (got.slots[:34] >= 0).all()


def test_rows_and_buffers_that_are_too_short(sq):
    pool = Pool(sq, [0, 30, 5, 0], 16, 20, 3)
    got = pool.step(sq, [49, 48, 2 ** 31 - 1, 10], 60)      # the first and third: more pages than the row holds
    assert got.lengths.tolist() == [0, 30, 5, 0]            # and their tokens take the buffer's places
    got = pool.step(sq, [48, 40, 5, 3], 60)
    assert got.lengths.tolist() == [48, 40, 5, 0] and got.starts.tolist() == [0, 48, 58, 58, 60]
    pool.step(sq, [2 ** 31 - 1] * 4, 7)
    pool.step(sq, [-2 ** 31] * 4, 1)
    assert sq.sync_status() == 0


def test_nothing_to_do(sq):
    Pool(sq, [], 16, 4, 3).step(sq, [], 5)
    Pool(sq, [3, -1], 16, 0, 4).step(sq, [3, -1], 0)
    Pool(sq, [-1, 0], 16, 2, 0).step(sq, [1, 0], 3)
    assert sq.sync_status() == 0


def test_in_place_lengths_and_given_outputs(sq):
    pool = Pool(sq, [40] * 600, 16, 700, 8, seed=3)
    lengths = ints(pool.lengths)
    cap = 2500
    out = sq.KVStep(torch.full((601,), -7, dtype=torch.int32, device="cuda"), torch.full((cap,), -7, dtype=torch.int32, device="cuda"),
                    torch.full((cap,), -7, dtype=torch.int64, device="cuda"), lengths)
    for grow in (1, 3, 20):
        targets = [n + grow if i % 3 else n for i, n in enumerate(pool.lengths)]
        want = step_plain.plan(16, pool.table, pool.free, pool.n_free, pool.lengths, targets, cap)
        t = ints(targets)
        sq.kv_plan(pool.pages, lengths, t, cap, out=out)
        torch.cuda.synchronize()
        pool.compare(out, want)
        pool.lengths, pool.table, pool.free, pool.n_free = want[3], want[4], want[5], want[6]
    left = torch.zeros(1, dtype=torch.int32, device="cuda")
    before = pool.pages.count.tolist()
    sq.kv_plan(pool.pages, lengths, ints([-1] * 600), cap, count_out=left)
    assert left.item() == pool.pages.n_pages and pool.pages.count.tolist() == before


def test_captured_decoding_steps(sq):
    """A graph whose replays each append a token: lengths and the pool in place."""
    pool = Pool(sq, [14, -1, 31], 16, 12, 5)
    lengths, one = ints([14, 0, 31]), torch.ones(3, dtype=torch.int32, device="cuda")
    pool.lengths = [14, 0, 31]
    targets = torch.zeros(3, dtype=torch.int32, device="cuda")
    out = sq.KVStep(*(torch.zeros(n, dtype=d, device="cuda") for n, d in ((4, torch.int32), (8, torch.int32), (8, torch.int64))), lengths)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        torch.add(lengths, one, out=targets)
        sq.kv_plan(pool.pages, lengths, targets, 8, out=out)
    for _ in range(40):
        want = step_plain.plan(16, pool.table, pool.free, pool.n_free, pool.lengths, [n + 1 for n in pool.lengths], 8)
        graph.replay()
        torch.cuda.synchronize()
        pool.compare(out, want)
        pool.lengths, pool.table, pool.free, pool.n_free = want[3], want[4], want[5], want[6]
    assert pool.lengths == [54, 40, 71] and sq.sync_status() == 0


def test_own_stream(sq):
    pool = Pool(sq, [0] * 50, 32, 100, 4)
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    pool.step(sq, [33] * 50, 2000, stream=st)


def test_bad_pages_and_counts_are_reported(sq):
    pool = Pool(sq, [20, 20], 16, 4, 4)
    pool.pages.table[0, 1] = 99
    got = sq.kv_plan(pool.pages, ints([20, 20]), ints([22, 22]), 4)
    n = pool.pages.n_pages * 16
    assert got.slots.tolist()[:2] == [n, n] and all(0 <= s < n for s in got.slots.tolist()[2:])
    assert sq.sync_status() == 0                         # (kv_write reports such a slot)
    pool.pages.free[3] = -4
    got = sq.kv_plan(pool.pages, ints([32, 20]), ints([34, 20]), 2)
    assert got.slots.tolist() == [n, n]
    assert sq.sync_status() == sq.SONIQ_ERR_INVALID_ARG
    for bad in (-3, 1 << 30):
        pool.pages.count[0] = bad
        sq.kv_plan(pool.pages, ints([5, 5]), ints([5, -1]), 0)
        assert sq.sync_status() == sq.SONIQ_ERR_INVALID_ARG
        assert 0 <= pool.pages.count[0].item() <= pool.pages.n_pages
    assert sq.sync_status() == 0


def test_what_is_planned_is_written(sq):
    """The step's rows through kv_write: padding and sequences that wait leave the cache alone."""
    D, page = 64, 16
    lay = sq.KVLayout(np.arange(D)[None], (D, 0), (8, 8))
    pages = sq.KVPages(5, page, 3, 4)
    cache = sq.KVCache(lay, lay, 5, page)
    step = sq.kv_plan(pages, ints([-1, -1, -1]), ints([40, 20, 33]), 120)
    rows = torch.randn(120, 1, D, device="cuda").half()
    cache.k_codes.fill_(77)
    sq.kv_write(cache, rows, rows, step.slots)
    assert step.lengths.tolist() == [40, 20, -1]
    k, _ = sq.kv_read(cache, step.slots[:60].clone())
    assert (k - rows[:60]).abs().max() <= rows.abs().max() / 127
    used = (cache.k_codes != 77).any(-1).sum().item()
    assert used == 60 and sq.sync_status() == 0
