"""Where prompts are short on the average two CTAs of one tile share an SM.  Sequences
without tokens bring every batch there: what the other instances are tested on, this one
is too, with prompts of several blocks, rows done again, and a lost copy."""
import pytest

import step_plain
import test_gpu_prompt_attend as full
from test_gpu_prompt_attend import BF16, F16, check, compare, ints, sq  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
with_tokens = full.draw


def draw(seed, lens, heads, G, D, Dv, dtype, pad=0, size=1.0):
    """The same with so many empty sequences behind that there are at most 128 rows a sequence."""
    q, k, v, starts = with_tokens(seed, lens, heads, G, D, Dv, dtype, pad, size)
    assert max(D, Dv) <= 128
    return q, k, v, starts + [starts[-1]] * max(0, q.shape[0] * min(G, 128) // 128 + 1 - len(lens))


@pytest.fixture
def small(monkeypatch):
    monkeypatch.setattr(full, "draw", draw)


@pytest.mark.parametrize("D,Dv", [(64, 64), (128, 128), (8, 8), (80, 80), (72, 104), (128, 24)])
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("causal", [True, False])
def test_widths(sq, small, D, Dv, dtype, causal):  # noqa: F811
    full.test_widths(sq, D, Dv, dtype, causal)


@pytest.mark.parametrize("G", [1, 3, 7, 16, 71, 200])
@pytest.mark.parametrize("causal", [True, False])
def test_shared_heads(sq, small, G, causal):  # noqa: F811
    full.test_shared_heads(sq, G, causal)


@pytest.mark.parametrize("lens", [[1], [127], [128], [129], [257], [1500], [3001]])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("causal", [True, False])
def test_one_prompt(sq, small, lens, D, causal):  # noqa: F811
    full.test_one_prompt(sq, lens, D, causal)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_what_a_row_does_not_see(sq, small, D, dtype, bad):  # noqa: F811
    full.test_what_a_row_does_not_see(sq, D, dtype, bad)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("causal", [True, False])
def test_nothing_behind_a_prompt_matters(sq, D, dtype, causal):  # noqa: F811
    """NaN in all keys and values behind each prompt alone, and in the padding."""
    lens = [129, 40, 300, 1, 255]
    q, k, v, starts = draw(41, lens, 2, 2, D, D, dtype, pad=30)
    want = check(sq, q, k, v, starts, causal)
    for s, e in zip(starts, starts[1:6]):
        y = [k.clone(), v.clone()]
        for x in y:
            x[e:] = float("nan")
            x[:s] = float("nan")
        got = sq.prompt_attend(q, *y, ints(starts), causal)
        assert torch.equal(got[s:e], want[s:e])


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_tokens_of_no_weight(sq, small, D, dtype):  # noqa: F811
    full.test_tokens_of_no_weight(sq, D, dtype)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_scores_of_any_size(sq, small, D, dtype):  # noqa: F811
    full.test_scores_of_any_size(sq, dtype, D)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("D", [64, 128])
def test_values_near_the_ends_of_their_types(sq, small, causal, D):  # noqa: F811
    full.test_values_near_the_ends_of_their_types(sq, causal, D)


def test_more_units_than_places(sq):  # noqa: F811
    """Long prompts among empty sequences: each CTA takes several units, of many blocks."""
    for causal in (True, False):
        check(sq, *draw(42, [1200, 0, 700, 2100, 33], 6, 4, 128, 128, BF16), causal)
        check(sq, *draw(43, [900] * 9, 4, 3, 64, 64, F16), causal)


@pytest.mark.parametrize("D", [64, 128])
def test_the_same_bits_every_time(sq, D):  # noqa: F811
    q, k, v, starts = draw(44, [700, 20, 3, 900, 128], 2, 4, D, D, BF16)
    want = check(sq, q, k, v, starts)
    for _ in range(5):
        assert torch.equal(sq.prompt_attend(q, k, v, ints(starts)), want)


def test_streams_and_graphs(sq):  # noqa: F811
    q, k, v, starts = draw(45, [300, 41, 150], 2, 2, 128, 128, BF16)
    want = check(sq, q, k, v, starts)
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    st = ints(starts)
    outs = [sq.prompt_attend(q, k, v, st, stream=s) for s in streams for _ in range(3)]
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)
    graphs = []
    for _ in range(2):
        out, g = torch.full_like(want, 7.0), torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            sq.prompt_attend(q, k, v, st, out=out)
        graphs.append((g, out))
    new = [0, 10, 10, 444] + [444] * (len(starts) - 4)
    st.copy_(ints(new))
    torch.cuda.synchronize()
    for _ in range(5):
        for (g, _), s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for _, out in graphs:
        compare(out, q, k, v, new)
    assert sq.sync_status() == 0


def test_rows_done_again_take_their_time(sq):  # noqa: F811
    """All rows of a prompt, for longer than the limit of a wait."""
    lens = [3000, 100]
    q, k, v, starts = draw(46, lens, 12, 2, 128, 128, BF16)
    ref = step_plain.attend(q.double(), k.double(), v.double(), starts, True, 128 ** -0.5)
    tol = step_plain.attend_tolerance(*ref, max(lens), BF16)
    v[2999] = float("nan")
    sq.test_wait_limit(2_000_000)
    got = sq.prompt_attend(q, k, v, ints(starts))
    assert sq.sync_status() == 0
    ok = (got.double() - ref[0]).abs() <= tol
    ok[2999] = got[2999].isnan()
    assert ok.all()


@pytest.mark.parametrize("lens,D,causal", [([40, 0, 0], 64, True), ([700, 20], 128, True), ([900] * 8, 128, False)])
def test_lost_copy(sq, lens, D, causal):  # noqa: F811
    args = draw(47, lens, 2, 4, D, D, BF16)
    sq.test_wait_limit(20_000_000)
    sq.test_drop_barrier_arrival()
    sq.prompt_attend(*args[:3], ints(args[3]), causal)
    assert sq.sync_status() == sq.SONIQ_ERR_TIMEOUT
    assert sq.sync_status() == 0
    check(sq, *args, causal)
