"""Normed and turned heads against fp64, angles reduced exactly."""
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


def rows(rng, shape, dtype, spread=0.5):
    x = rng.standard_normal(shape) * np.exp(spread * rng.standard_normal(shape[:-1] + (1,)))
    return torch.from_numpy(x).to(dtype).cuda()


def check(sq, q, k, rotary, positions, gains=(None, None), eps=1e-6, **kw):
    before = [t.clone() if t is not None else None for t in (q, k)]
    got = sq.rotate_heads(rotary, q, k, positions, gains[0], gains[1], eps, **kw)
    torch.cuda.synchronize()
    freq = rotary.frequencies if rotary is not None else []
    for y, x, gain in zip(got, before, gains):
        if x is None:
            assert y is None
            continue
        ref, mag = step_plain.rotate(x.double().cpu().numpy(), freq, positions.tolist() if positions is not None else [0] * len(x),
                                     rotary.interleaved if rotary else False, gain.double().cpu().numpy() if gain is not None else None,
                                     eps, rotary.magnitude if rotary else 1.0)
        err = np.abs(y.double().cpu().numpy() - ref)
        assert (err <= step_plain.rotate_tolerance(ref, mag, x.dtype)).all(), err.max()
    return got


def positions_of(rng, n, far=5000):
    return torch.from_numpy(rng.integers(0, far, n).astype(np.int32)).cuda()


@pytest.mark.parametrize("D,channels", [(128, 128), (128, 64), (128, 32), (128, 122), (64, 64), (64, 16), (40, 40), (40, 32), (80, 80),
                                        (96, 96), (96, 48), (192, 192), (192, 64), (256, 256), (256, 128), (1, 0), (2, 2), (7, 6),
                                        (33, 20), (255, 254)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("norm", [False, True])
def test_heads(sq, D, channels, interleaved, dtype, norm):
    rng = np.random.default_rng(D * 7 + channels)
    n, Hq, Hk = 37, 6, 3
    gains = [torch.from_numpy((1 + 0.3 * rng.standard_normal(D)).astype(np.float32)).cuda() for _ in range(2)] if norm else (None, None)
    rotary = sq.Rotary(channels, interleaved=interleaved, magnitude=1.25) if channels else None
    check(sq, rows(rng, (n, Hq, D), dtype), rows(rng, (n, Hk, D), dtype), rotary, positions_of(rng, n), gains)


@pytest.mark.parametrize("n", [1, 2, 3, 1001, 5003])
@pytest.mark.parametrize("Hq,Hk", [(1, 1), (32, 8), (5, 0), (0, 3), (71, 1)])
def test_numbers_of_tokens_and_heads(sq, n, Hq, Hk):
    rng = np.random.default_rng(n + Hq)
    q, k = (rows(rng, (n, h, 128), BF16) if h else None for h in (Hq, Hk))
    gains = [torch.from_numpy((1 + 0.3 * rng.standard_normal(128)).astype(np.float32)).cuda() if h else None for h in (Hq, Hk)]
    check(sq, q, k, sq.Rotary(128, scaling=("wavelength", 8, 1, 4, 512)), positions_of(rng, n), gains)


@pytest.mark.parametrize("D,channels", [(128, 128), (128, 90)])
@pytest.mark.parametrize("norm", [False, True])
def test_slices_in_place_and_other_strides(sq, D, channels, norm):
    rng = np.random.default_rng(5)
    n, Hq, Hk = 50, 8, 2
    rotary, pos = sq.Rotary(channels, base=500000.0), positions_of(rng, n)
    gain = torch.from_numpy((1 + 0.3 * rng.standard_normal(D)).astype(np.float32)).cuda() if norm else None
    fused = rows(rng, (n, Hq + 2 * Hk, D), F16)
    kept = fused.clone()
    want = check(sq, fused[:, :Hq], fused[:, Hq:Hq + Hk], rotary, pos, (gain, gain))
    assert torch.equal(fused, kept)
    # in place, and nothing beside them touched
    q, k = fused[:, :Hq], fused[:, Hq:Hq + Hk]
    got = sq.rotate_heads(rotary, q, k, pos, gain, gain, q_out=q, k_out=k)
    assert got[0].data_ptr() == q.data_ptr() and torch.equal(q, want[0]) and torch.equal(k, want[1])
    assert torch.equal(fused[:, Hq + Hk:], kept[:, Hq + Hk:])
    # heads in front of tokens, and rows that begin off their 16 bytes
    first = kept[:, :Hq].transpose(0, 1).contiguous().transpose(0, 1)
    assert torch.equal(sq.rotate_heads(rotary, first, None, pos, gain)[0], want[0])
    wide = torch.zeros(n, Hq, D + 3, dtype=F16, device="cuda")
    wide[:, :, 3:] = kept[:, :Hq]
    off = sq.rotate_heads(rotary, wide[:, :, 3:], None, pos, gain)[0]
    ref = want[0].double()
    assert ((off.double() - ref).abs() <= 2 * 2.0 ** -11 * ref.abs() + 2.0 ** -18).all()      # another order of sums
    # a row broadcast to all tokens
    one = kept[:1, :Hq].expand(n, Hq, D)
    check(sq, one, None, rotary, pos, (gain, None))


@pytest.mark.parametrize("scaling", [None, ("linear", 3.0), ("wavelength", 8.0, 1.0, 4.0, 8192)])
def test_far_and_negative_positions(sq, scaling):
    rng = np.random.default_rng(9)
    pos = [0, 1, -1, 4095, 131071, 1000003, 2 ** 24 + 1, 2 ** 31 - 1, -(2 ** 31), -(2 ** 20) - 7]
    check(sq, rows(rng, (len(pos), 4, 128), F16), None, sq.Rotary(128, base=1e6, scaling=scaling),
          torch.tensor(pos, dtype=torch.int32, device="cuda"))


def test_given_frequencies(sq):
    """Zero, negative, more than a turn a position."""
    rng = np.random.default_rng(10)
    check(sq, rows(rng, (9, 2, 16), BF16), None, sq.Rotary(16, frequencies=[0.0, -0.3, 7.5, 100.0, 1e-9, 3.0, -6.4, 0.01]),
          positions_of(rng, 9, 100000))


@pytest.mark.parametrize("D", [128, 50])
def test_rows_whose_squares_leave_fp32(sq, D):
    rng = np.random.default_rng(11)
    ones = torch.ones(D, device="cuda")
    base = rng.standard_normal((6, 3, D))
    for dtype, size in ((BF16, 3e37), (BF16, 1e25), (BF16, 1e-20), (BF16, 1e-36), (F16, 6000.0), (F16, 1e-6)):
        for eps in (0.0, 1e-6):
            check(sq, torch.from_numpy(base * size).to(dtype).cuda(), None, None, None, (ones, None), eps)
    zero = torch.zeros(2, 1, D, dtype=BF16, device="cuda")
    assert (sq.rotate_heads(None, zero, None, None, ones, eps=1e-6)[0] == 0).all()
    # no eps: 0 / 0
    assert sq.rotate_heads(None, zero, None, None, ones, eps=0.0)[0].isnan().all()


@pytest.mark.parametrize("D,channels", [(128, 64), (50, 20)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_infinities_stay_in_their_pairs(sq, D, channels, interleaved):
    rng = np.random.default_rng(12)
    rotary = sq.Rotary(channels, interleaved=interleaved)
    x = rows(rng, (4, 2, D), F16)
    pos = torch.tensor([1, 2, 3, 4], dtype=torch.int32, device="cuda")
    want = sq.rotate_heads(rotary, x, None, pos)[0]
    y = x.clone()
    y[0, 0, 3], y[1, 1, D - 1], y[2, 0, D - 2] = float("inf"), float("-inf"), float("nan")
    got = sq.rotate_heads(rotary, y, None, pos)[0]
    mate = 2 if interleaved else 3 + channels // 2
    assert not got[0, 0, 3].isfinite() and not got[0, 0, mate].isfinite()
    assert got[1, 1, D - 1] == float("-inf") and got[2, 0, D - 2].isnan()
    same = torch.ones_like(x, dtype=torch.bool)
    same[0, 0, 3] = same[0, 0, mate] = same[1, 1, D - 1] = same[2, 0, D - 2] = False
    assert torch.equal(got[same], want[same])
    # with a norm, a row that holds an infinity or a NaN, and no other
    ones = torch.ones(D, device="cuda")
    a, b = sq.rotate_heads(rotary, x, None, pos, ones)[0], sq.rotate_heads(rotary, y, None, pos, ones)[0]
    whole = torch.ones(4, 2, dtype=torch.bool)
    whole[0, 0] = whole[1, 1] = whole[2, 0] = False
    assert torch.equal(a[whole], b[whole]) and b[2, 0].isnan().all() and b[0, 0, 3].isnan() and (b[1, 1, channels:D - 1] == 0).all()


def test_streams_and_graphs(sq):
    rng = np.random.default_rng(13)
    x, rotary, pos = rows(rng, (100, 4, 64), F16), sq.Rotary(64), positions_of(rng, 100)
    want = sq.rotate_heads(rotary, x, x, pos)
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = sq.rotate_heads(rotary, x, x, pos, stream=st)
    st.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    graph, y = torch.cuda.CUDAGraph(), torch.empty_like(x)
    with torch.cuda.graph(graph):
        sq.rotate_heads(rotary, x, None, pos, q_out=y)
    pos.add_(5)
    x.mul_(0.5)
    graph.replay()
    assert torch.equal(y, sq.rotate_heads(rotary, x, None, pos)[0])


def test_offsets_past_32_bits(sq):
    """A token stride of 2^31 elements."""
    rng = np.random.default_rng(14)
    big = torch.zeros(2 ** 31 + 4 * 64, dtype=F16, device="cuda")
    x = big.as_strided((2, 4, 64), (2 ** 31, 64, 1))
    x.copy_(rows(rng, (2, 4, 64), F16))
    rotary, pos = sq.Rotary(64), torch.tensor([7, 8], dtype=torch.int32, device="cuda")
    want = check(sq, x.contiguous(), None, rotary, pos)[0]
    sq.rotate_heads(rotary, x, None, pos, q_out=x)
    assert torch.equal(x, want)


def test_a_rotary_made_elsewhere_is_refused(sq):
    x, pos = torch.zeros(2, 3, 16, dtype=F16, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):
        sq.rotate_heads(sq.Rotary(4, device="cpu"), x, None, pos)
    sq.rotate_heads(sq.Rotary(0, device="cpu"), x, None)        # turns nothing
