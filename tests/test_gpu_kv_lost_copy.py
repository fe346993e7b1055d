"""A copy that never comes ends the call on the tensor-core path too: within its
bound, with a status, and with nothing left behind for the next call."""
import time

import pytest

import test_gpu_kv_attend as base

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

sq = base.sq

BOUND = 2.0         # seconds of a wait


@pytest.mark.parametrize("shape", [0, 1, 7])
@pytest.mark.parametrize("lens,T,group", [
    ([200, 31], 20, 4),         # one row tile as two streams
    ([70], 40, 1),              # ... whose second stream has one block
    ([200, 31], 40, 4),         # two row tiles
    ([3000], 24, 4),            # an item in parts, which the second kernel would join
    ([3000, 900, -1, 40], 64, 8)])
def test_lost_copy_is_reported(sq, lens, T, group, shape):
    p = base.Problem(sq, 81, base.LAYOUTS[shape], lens, T, group, 16, torch.float16)
    q = p.q.cuda()
    want = sq.kv_attend(p.cache, q, p.table, p.dlens)
    assert sq.sync_status() == 0
    sq.test_drop_barrier_arrival()
    start = time.monotonic()
    sq.kv_attend(p.cache, q, p.table, p.dlens)
    assert sq.sync_status() == sq.SONIQ_ERR_TIMEOUT
    # one wait runs out; the waits for copies and MMAs in flight that follow have nothing to wait for
    assert BOUND <= time.monotonic() - start < 2 * BOUND
    for _ in range(2):
        assert torch.equal(sq.kv_attend(p.cache, q, p.table, p.dlens), want)
    assert sq.sync_status() == 0
