"""Attention of packed prompts against fp64."""
import numpy as np
import pytest

import step_plain

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
F16, BF16 = torch.float16, torch.bfloat16


@pytest.fixture(scope="module")
def sq():
    from paper_2311_14114_gb300 import build, soniq
    build.build()
    soniq.lib()
    return soniq


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def draw(seed, lens, heads, G, D, Dv, dtype, pad=0, size=1.0):
    g, n = gen(seed), sum(lens) + pad
    r = lambda h, d: torch.randn(n, h, d, generator=g, device="cuda") * torch.exp(0.3 * torch.randn(n, h, 1, generator=g, device="cuda"))
    starts = [0]
    for x in lens:
        starts.append(starts[-1] + x)
    return (r(heads * G, D) * size).to(dtype), r(heads, D).to(dtype), r(heads, Dv).to(dtype), starts


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def check(sq, q, k, v, starts, causal=True, scale=None, **kw):
    out = torch.full((q.shape[0], q.shape[1], v.shape[2]), 7.0, dtype=q.dtype, device="cuda")
    got = sq.prompt_attend(q, k, v, ints(starts), causal, scale, out=out, **kw)
    torch.cuda.synchronize()
    assert got is out and sq.sync_status() == 0
    compare(got, q, k, v, starts, causal, scale)
    return got


def compare(got, q, k, v, starts, causal=True, scale=None):
    n = starts[-1]
    ref = step_plain.attend(q[:n].double(), k[:n].double(), v[:n].double(), starts, causal, q.shape[2] ** -0.5 if scale is None else scale)
    tol = step_plain.attend_tolerance(*ref, max([b - a for a, b in zip(starts, starts[1:])] + [0]), q.dtype)
    first = starts[0]
    err = (got[:n].double() - ref[0]).abs()
    assert (err <= tol)[first:].all(), ((err / tol)[first:].max().item(), (err > tol)[first:].nonzero()[:5].tolist())
    assert (got[n:] == 7).all() and (got[:first] == 7).all()


EDGES = [1, 2, 63, 64, 65, 0, 127, 128, 129, 200, 255, 256, 257, 300]


@pytest.mark.parametrize("D,Dv", [(64, 64), (128, 128), (256, 256), (8, 8), (40, 40), (80, 80), (96, 96), (192, 192), (72, 136), (192, 128),
                                  (256, 64), (64, 256), (128, 24)])
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("causal", [True, False])
def test_widths(sq, D, Dv, dtype, causal):
    check(sq, *draw(D + Dv, EDGES, 2, 2, D, Dv, dtype, pad=11), causal)


@pytest.mark.parametrize("G", [1, 2, 3, 4, 5, 6, 7, 8, 12, 16, 32, 64, 71, 128, 200])
@pytest.mark.parametrize("causal", [True, False])
def test_shared_heads(sq, G, causal):
    check(sq, *draw(G, [40, 1, 77, 130, 0, 261], 2 if G < 64 else 1, G, 64, 64, BF16), causal)


@pytest.mark.parametrize("lens", [[1], [2], [63], [64], [65], [128], [129], [256], [257], [777], [1500], [3001]])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("causal", [True, False])
def test_one_prompt(sq, lens, D, causal):
    check(sq, *draw(lens[0], lens, 2, 4, D, D, F16), causal)


def test_heads_alone(sq):
    """As many query heads as key heads, in every number of row tiles."""
    for n in (1, 100, 128, 129, 256, 300, 513, 1030):
        check(sq, *draw(n, [n, 3], 3, 1, 128, 128, BF16))


def test_a_long_prompt(sq):
    check(sq, *draw(3, [9000], 1, 2, 128, 128, F16))


def test_many_prompts(sq):
    rng = np.random.default_rng(4)
    check(sq, *draw(4, rng.integers(0, 12, 3000).tolist(), 2, 3, 64, 64, F16, pad=5))
    check(sq, *draw(5, rng.integers(0, 400, 100).tolist(), 2, 2, 128, 128, BF16))
    check(sq, *draw(6, [0] * 40 + [700] + [1] * 40, 2, 1, 64, 64, F16))


def test_none(sq):
    q, k, v, _ = draw(0, [5], 1, 1, 64, 64, F16)
    check(sq, q, k, v, [0])
    check(sq, q, k, v, [0, 0, 0])
    check(sq, q, k, v, [2, 2, 4])
    check(sq, q[:0], k[:0], v[:0], [0, 0])


@pytest.mark.parametrize("D,Dv", [(1, 1), (7, 5), (33, 33), (50, 250), (255, 12)])
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_odd_widths(sq, D, Dv, dtype):
    check(sq, *draw(D, [1, 0, 40, 70], 2, 2, D, Dv, dtype, pad=2))


def test_strides(sq):
    lens, heads, G, D, Dv = [100, 33, 290], 2, 4, 64, 128
    q, k, v, starts = draw(7, lens, heads, G, D, Dv, F16)
    want, n = check(sq, q, k, v, starts), q.shape[0]
    fused = torch.full((n, heads * (G * D + D + Dv) + 8), float("nan"), dtype=F16, device="cuda")
    fused[:, :-8] = torch.cat([q.flatten(1), k.flatten(1), v.flatten(1)], 1)
    fq, fk, fv = fused[:, :-8].split([heads * G * D, heads * D, heads * Dv], 1)
    assert torch.equal(sq.prompt_attend(fq.unflatten(1, (-1, D)), fk.unflatten(1, (-1, D)), fv.unflatten(1, (-1, Dv)), ints(starts)), want)
    flip = lambda x: x.transpose(0, 1).contiguous().transpose(0, 1)
    assert torch.equal(sq.prompt_attend(flip(q), flip(k), flip(v), ints(starts)), want)
    wide = lambda x, by: torch.nn.functional.pad(x, (8, by), value=float("nan"))[:, :, 8:8 + x.shape[2]]
    assert torch.equal(sq.prompt_attend(wide(q, 8), wide(k, 16), wide(v, 24), ints(starts)), want)
    # rows off their 16 bytes, and one head's row for all: other kernels or copies, the same values within the tolerance
    for x in ((wide(q, 1), k, v), (q, wide(k, 3), v), (q, k, wide(v, 5))):
        out = sq.prompt_attend(*x, ints(starts))
        compare(out, q, k, v, starts)
    one = k[:, :1].expand(n, heads, D)
    check(sq, q, one, v, starts)
    same = k[:1].expand(n, heads, D)
    check(sq, q, same, v, starts)


def test_offsets_past_32_bits(sq):
    """A token stride of 2^26 elements: keys lie up to 2^32 elements apart."""
    q, k, v, starts = draw(8, [40], 1, 1, 64, 64, F16)
    big = torch.empty(39 * 2 ** 26 + 64, dtype=F16, device="cuda")
    far = big.as_strided((40, 1, 64), (2 ** 26, 64, 1))
    far.copy_(k)
    want = check(sq, q, k, v, starts)
    assert torch.equal(sq.prompt_attend(q, far, v, ints(starts)), want)
    far.copy_(v)
    assert torch.equal(sq.prompt_attend(q, k, far, ints(starts)), want)


@pytest.mark.parametrize("D", [64, 128, 256, 33])
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_what_a_row_does_not_see(sq, D, dtype, bad):
    """Anything in later tokens, other prompts and rows of none.  Other prompts keep their
    bits.  Earlier rows of the same prompt may be done by other arithmetic (from the
    definition in fp32, weights not rounded, sums in another order), which is within
    the tolerance of the same fp64 values: it counts the rounding of weights, which that
    leaves out, and any order of sums in fp32."""
    lens = [70, 200, 1, 150]
    q, k, v, starts = draw(9, lens, 2, 2, D, D, dtype, pad=40)
    want = check(sq, q, k, v, starts)
    ref = step_plain.attend(q.double(), k.double(), v.double(), starts, True, D ** -0.5)
    tol = step_plain.attend_tolerance(*ref, max(lens), dtype)
    for x in (k, v):
        for t, seen_from in ((60, 70), (120, 270), (269, 270), (270, 271), (starts[-1] + 3, None), (430, starts[-1])):
            y = [a.clone() for a in (q, k, v)]
            y[1 if x is k else 2][t] = bad
            got = sq.prompt_attend(*y, ints(starts), out=torch.full_like(want, 7.0))
            hit, before = torch.zeros(q.shape[0], dtype=torch.bool), torch.zeros(q.shape[0], dtype=torch.bool)
            if t < starts[-1]:
                s, e = next((s, e) for s, e in zip(starts, starts[1:]) if s <= t < e)
                hit[t:e] = True
                before[s:t] = True
            assert torch.equal(got[~hit & ~before], want[~hit & ~before])
            assert ((got.double() - ref[0]).abs() <= tol)[before].all()
            if x is v and bad == bad and t < starts[-1]:        # an infinity of any weight
                assert (got[hit] == bad).all() or dtype == F16 and not got[hit].isfinite().any()
            elif bad != bad and t < starts[-1]:
                assert got[hit].isnan().all()
    y = q.clone()
    y[100, 1], y[300] = bad, bad
    got = sq.prompt_attend(y, k, v, ints(starts), out=torch.full_like(want, 7.0))
    keep = torch.ones(q.shape[:2], dtype=torch.bool)
    keep[100, 1] = keep[300] = False
    assert torch.equal(got[keep], want[keep])
    assert got[100, 1].isnan().all() and got[300].isnan().all()


@pytest.mark.parametrize("D", [64, 128, 256, 33])
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_tokens_of_no_weight(sq, D, dtype):
    """The first 100 tokens' scores are minus infinity: they add nothing, the rows that
    see no others are NaN, and so is what sees a NaN or an infinity in their values
    (0 times it), wherever that stands among them."""
    lens = [170, 5]
    q, k, v, starts = draw(15, lens, 2, 2, D, D, dtype)
    q[:, :, 0] = 1.0
    k[:100, :, 0] = -float("inf")
    for t in (None, 0, 31, 63, 64, 96, 99):
        for bad in (float("nan"), float("inf")):
            y = v.clone()
            if t is not None:
                y[t, :, 0] = bad
            got = sq.prompt_attend(q, k, y, ints(starts))
            assert got[:100].isnan().all()
            ref = step_plain.attend(q[100:].double(), k[100:].double(), v[100:].double(), [0, 70, 75], True, D ** -0.5)
            ok = (got[100:].double() - ref[0]).abs() <= step_plain.attend_tolerance(*ref, 170, dtype)
            seen = torch.zeros_like(ok)
            if t is not None:
                seen[:70, :, 0] = True
            assert ok[~seen].all() and got[100:][seen].isnan().all()


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_scores_of_any_size(sq, dtype, D):
    lens = [300, 150]
    for size in (0.0, 0.01, 10.0, 100.0):
        check(sq, *draw(10, lens, 2, 2, D, D, dtype, size=size))
    q, k, v, starts = draw(11, lens, 2, 2, D, D, dtype)
    # rising and falling along the prompt, by more than the weights' range at every step
    ramp = torch.arange(starts[-1], device="cuda")[:, None, None]
    for way in (1, -1):
        r = (q.abs() + 0.1, (0.05 * way * ramp * torch.ones_like(k)).to(dtype), v)
        check(sq, *r, starts)
        check(sq, *r, starts, scale=30.0 / D)
    check(sq, q, k, v, starts, scale=0.0)
    check(sq, q, k, v, starts, scale=3.0)


def test_scores_near_the_end_of_fp32(sq):
    """Products of 2^126, which times the factor of the exponent would pass it."""
    q, k, v, starts = draw(12, [200], 1, 2, 64, 64, BF16)
    q, k = torch.zeros_like(q), torch.zeros_like(k)
    q[:, :, 0] = 2.0 ** 63
    k[:, :, 0] = 2.0 ** 63 * torch.tensor([1.0, -1.0, 0.5, 0.25], device="cuda").repeat(50)[:, None]
    got = sq.prompt_attend(q, k, v, ints(starts), scale=1.9)
    best = torch.zeros(200, 1, 64, dtype=torch.float64, device="cuda")
    for t in range(200):
        best[t] = v[0:t + 1:4].double().mean(0)
    assert ((got.double() - best).abs() <= 2.0 ** -7 * best.abs() + 2.0 ** -8 * 4).all()


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_values_near_the_ends_of_their_types(sq, causal, D):
    lens = [200, 90]
    q, k, v, starts = draw(13, lens, 2, 2, D, D, BF16)
    for size in (1e38, 1e30, 1e-30):
        big = (v.float().clamp(-3, 3) * size).to(BF16)
        check(sq, q, k, big, starts, causal)
    full = torch.full_like(v, torch.finfo(BF16).max)
    got = sq.prompt_attend(q, k, full, ints(starts), causal)
    assert ((got.double() / torch.finfo(BF16).max - 1).abs() <= 2.0 ** -8).all()
    q, k, v, starts = draw(14, lens, 2, 2, D, D, F16)
    check(sq, q, k, (v.float() * 1e4).clamp(-6e4, 6e4).half(), starts, causal)
    check(sq, q, k, (v.float() * 1e-5).half(), starts, causal)


def test_small_weights_count(sq):
    """One token with nearly all of the weight and little in its value, many with little: 2^-20 each."""
    n = 400
    q = torch.zeros(n, 1, 64, dtype=F16, device="cuda")
    k, v = torch.zeros_like(q), torch.zeros_like(q)
    q[:, :, 0], k[0, :, 0] = 1.0, 20 * np.log(2.0)
    v[1:] = 1000.0
    check(sq, q, k, v, [0, n], scale=1.0)


@pytest.mark.parametrize("D", [128, 256, 33])
def test_the_same_bits_every_time(sq, D):
    q, k, v, starts = draw(15, [700, 20, 3, 900, 128], 2, 4, D, D, BF16)
    want = check(sq, q, k, v, starts)
    for _ in range(5):
        assert torch.equal(sq.prompt_attend(q, k, v, ints(starts)), want)
    # and whatever stands beside a prompt
    for a, b in zip(starts, starts[1:]):
        alone = sq.prompt_attend(q[a:b].contiguous(), k[a:b].contiguous(), v[a:b].contiguous(), ints([0, b - a]))
        assert torch.equal(alone, want[a:b])


def test_prompts_behind_the_first_rows(sq):
    q, k, v, _ = draw(16, [300], 2, 2, 64, 64, F16)
    check(sq, q, k, v, [37, 100, 100, 260])


@pytest.mark.parametrize("D", [128, 33])
@pytest.mark.parametrize("starts,good", [([-5, 50, 100], [1]), ([0, 50, 1000], [0]), ([0, 90, 60, 120], [0]), ([0, 90, 60, 80, 95, 120], [0, 4]),
                                         ([0, 2 ** 31 - 1, 100], []), ([-2 ** 31, 2 ** 31 - 1, 2 ** 31 - 1], []),
                                         ([0, 30] * 40 + [30, 77], [0, 80])])
def test_bad_starts_are_reported(sq, D, starts, good):
    """What begins in front of the end of a prompt before it is left out, so no row is written twice."""
    q, k, v, _ = draw(17, [200], 2, 2, D, D, F16)
    out = torch.full((200, 4, D), 7.0, dtype=F16, device="cuda")
    sq.prompt_attend(q, k, v, ints(starts), out=out)
    assert sq.sync_status() == sq.SONIQ_ERR_INVALID_ARG
    assert sq.sync_status() == 0
    left = torch.ones(200, dtype=torch.bool)
    for b in good:
        s, e = starts[b], starts[b + 1]
        compare(out[s:e], q[s:e], k[s:e], v[s:e], [0, e - s])
        left[s:e] = False
    assert (out[left] == 7).all()


@pytest.mark.parametrize("D", [128, 50])
def test_streams_and_graphs(sq, D):
    q, k, v, starts = draw(18, [300, 41, 150], 2, 2, D, D, BF16)
    want = check(sq, q, k, v, starts)
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    st = ints(starts)
    outs = [sq.prompt_attend(q, k, v, st, stream=s) for s in streams for _ in range(3)]
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)
    # graphs replayed side by side, with other prompts than they were captured with
    graphs = []
    for _ in range(2):
        out, g = torch.full_like(want, 7.0), torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            sq.prompt_attend(q, k, v, st, out=out)
        graphs.append((g, out))
    new = [0, 10, 10, 444]
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
