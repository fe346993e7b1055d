"""Plans of different sizes from several threads at once: none changes what another's launch needs."""
import threading

import pytest

from test_gpu_kv_plan import Pool, ints, sq  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def test_threads_with_their_own_pools(sq):  # noqa: F811
    sizes, errors = (8192, 2400, 5000, 3000), []
    pools = [Pool(sq, [5] * B, 16, 0, 2, seed=B) for B in sizes]
    lengths = [ints([5] * B) for B in sizes]
    targets = [ints([6 + b % 3 for b in range(B)]) for B in sizes]
    torch.cuda.synchronize()
    begin = threading.Barrier(len(sizes))

    def work(i):
        try:
            begin.wait(10)
            for _ in range(1500):
                got = sq.kv_plan(pools[i].pages, lengths[i], targets[i], 4 * sizes[i])
            assert torch.equal(got.lengths, targets[i])
        except Exception as e:  # noqa: BLE001
            errors.append(f"{sizes[i]}: {e}")

    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(sizes))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert errors == []
    assert sq.sync_status() == 0
