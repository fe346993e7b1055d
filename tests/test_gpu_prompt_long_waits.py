"""A role of the prompts' kernel that waits while others work waits for as long as they
do: over units, and over rows done again, that take longer than the limit of a wait."""
import pytest

import step_plain
from test_gpu_prompt_attend import BF16, F16, check, draw, ints, sq  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("lens,heads,G,D,causal", [([4096, 300], 6, 2, 128, True), ([4096], 6, 1, 256, True), ([4096, 70], 6, 2, 64, True)])
def test_rows_done_again(sq, lens, heads, G, D, causal):  # noqa: F811
    """A NaN in the last token's values has all rows of its prompt done again: some
    2 us a token of the prompt, which holds up a unit for 8 ms.  (There are more units
    than SMs, so other roles wait with the next one.)"""
    q, k, v, starts = draw(21, lens, heads, G, D, D, BF16)
    last = starts[1] - 1
    ref = step_plain.attend(q.double(), k.double(), v.double(), starts, causal, D ** -0.5)
    tol = step_plain.attend_tolerance(*ref, max(lens), BF16)
    v[last] = float("nan")
    sq.test_wait_limit(2_000_000)
    got = sq.prompt_attend(q, k, v, ints(starts), causal)
    assert sq.sync_status() == 0
    ok = (got.double() - ref[0]).abs() <= tol
    ok[last] = got[last].isnan()
    assert ok.all()


@pytest.mark.parametrize("n,D", [(400000, 8), (150000, 256)])
def test_units_longer_than_a_wait(sq, n, D):  # noqa: F811
    """A unit at the end of 400000 tokens goes over 3125 blocks: 4 ms."""
    q, k, v, starts = draw(22, [n], 1, 1, D, D, F16)
    sq.test_wait_limit(1_000_000)
    out = sq.prompt_attend(q, k, v, ints(starts))
    assert sq.sync_status() == 0
    # some rows against fp64: as the only queries of their prefix
    for t in (0, 1000, n // 2, n - 1):
        s = (k[:t + 1, 0].double() @ q[t, 0].double()) * D ** -0.5
        p = torch.softmax(s, 0)
        ref, mag = p @ v[:t + 1, 0].double(), p @ v[:t + 1, 0].double().abs()
        dscore = ((k[:t + 1, 0].double().abs() @ q[t, 0].double().abs()) * D ** -0.5).max()
        total, top = torch.exp(s - s.max()).sum(), v[:t + 1, 0].double().abs().max()
        tol = step_plain.attend_tolerance(ref, mag, dscore, total, top, n, F16)
        assert ((out[t, 0].double() - ref).abs() <= tol).all()


def test_a_lost_copy_is_given_up_all_the_same(sq):  # noqa: F811
    args = draw(23, [700, 20], 2, 4, 128, 128, BF16)
    sq.test_wait_limit(5_000_000)
    sq.test_drop_barrier_arrival()
    sq.prompt_attend(*args[:3], ints(args[3]))
    assert sq.sync_status() == sq.SONIQ_ERR_TIMEOUT
    check(sq, *args)
