"""The C entry points of a step reject bad arguments on the host, before any CUDA
call (so these run on CPU; no pointer here is ever read), and so does the binding."""
import ctypes
import math

import pytest
import torch

OK, INVALID, UNSUPPORTED, ALIGNMENT = 0, 1, 2, 3
FAKE = 1 << 20                  # an aligned address that no check reads


@pytest.fixture(scope="module")
def sq():
    from paper_2311_14114_gb300 import build, soniq
    build.build()
    soniq.lib()
    return soniq


def plan(sq, **kw):
    a = dict(page=16, n_pages=4, table=FAKE, stride=4, width=4, free=FAKE, count=FAKE, count_out=FAKE, lengths=FAKE,
             targets=FAKE, B=2, cap=8, starts=FAKE, positions=FAKE, slots=FAKE, lengths_out=FAKE)
    assert set(kw) <= set(a)
    a.update(kw)
    return sq.lib().soniq_kv_plan(*a.values(), None)


@pytest.mark.parametrize("kw,want", [
    (dict(page=0), INVALID), (dict(page=24), INVALID), (dict(page=8), UNSUPPORTED), (dict(page=512), UNSUPPORTED),
    (dict(n_pages=0), INVALID), (dict(n_pages=1 << 31), UNSUPPORTED), (dict(width=-1), INVALID), (dict(B=-1), INVALID),
    (dict(B=8193), UNSUPPORTED), (dict(B=8192, width=1 << 20), UNSUPPORTED), (dict(cap=-1), INVALID),
    (dict(count=None), INVALID), (dict(count_out=None), INVALID), (dict(free=None), INVALID), (dict(starts=None), INVALID),
    (dict(lengths=None), INVALID), (dict(targets=None), INVALID), (dict(lengths_out=None), INVALID), (dict(table=None), INVALID),
    (dict(positions=None), INVALID), (dict(slots=None), INVALID), (dict(slots=FAKE + 4), ALIGNMENT),
    (dict(table=FAKE + 2), ALIGNMENT), (dict(free=FAKE + 1), ALIGNMENT), (dict(count=FAKE + 2), ALIGNMENT),
    (dict(lengths=FAKE + 1), ALIGNMENT), (dict(starts=FAKE + 2), ALIGNMENT), (dict(positions=FAKE + 2), ALIGNMENT),
    (dict(lengths_out=FAKE + 3), ALIGNMENT)])
def test_bad_plans(sq, kw, want):
    assert plan(sq, **kw) == want


def rotate(sq, **kw):
    a = dict(channels=8, magnitude=1.0, turns=FAKE, positions=FAKE, n=1, D=16, dtype=0, heads=2, in_=FAKE, out=FAKE, gain=None,
             eps=1e-6, q=True, k=False)
    assert set(kw) <= set(a)
    a.update(kw)
    r = sq.CRotary(a["channels"], 0, a["magnitude"], a["turns"])
    h = sq.CHeads(a["heads"], a["in_"], 32, 16, a["out"], 32, 16, a["gain"])
    return sq.lib().soniq_rotate_heads(ctypes.byref(r), a["positions"], a["n"], a["D"], a["dtype"],
                                       ctypes.byref(h) if a["q"] else None, ctypes.byref(h) if a["k"] else None, a["eps"], None)


@pytest.mark.parametrize("kw,want", [
    (dict(n=0), OK), (dict(q=False), OK), (dict(heads=0), OK), (dict(n=-1), INVALID), (dict(n=1 << 40), UNSUPPORTED),
    (dict(D=0, channels=0), INVALID), (dict(D=257), UNSUPPORTED), (dict(dtype=2), INVALID), (dict(channels=7), INVALID),
    (dict(channels=18), INVALID), (dict(channels=-2), INVALID), (dict(magnitude=math.inf), INVALID),
    (dict(magnitude=math.nan), INVALID), (dict(eps=-1.0), INVALID), (dict(eps=math.nan), INVALID), (dict(turns=None), INVALID),
    (dict(positions=None), INVALID), (dict(turns=FAKE + 4), ALIGNMENT), (dict(positions=FAKE + 2), ALIGNMENT),
    (dict(heads=-1), INVALID), (dict(heads=4097), UNSUPPORTED), (dict(in_=None), INVALID), (dict(out=None), INVALID),
    (dict(in_=FAKE + 1), ALIGNMENT), (dict(out=FAKE + 1), ALIGNMENT), (dict(gain=FAKE + 2), ALIGNMENT),
    (dict(q=False, k=True, in_=None), INVALID)])
def test_bad_rotations(sq, kw, want):
    assert rotate(sq, **kw) == want


def test_frequencies(sq):
    r = sq.Rotary(8, base=100.0, device="cpu")
    assert r.frequencies == [100.0 ** (-2.0 * p / 8) for p in range(4)]
    # turns of 2^64 parts, to the nearest
    assert all(abs(t % 2 ** 64 - f / (2 * math.pi) * 2.0 ** 64) <= 2.0 ** 64 * f * 2.0 ** -53 for t, f in zip(r.turns.tolist(), r.frequencies))
    assert sq.Rotary(8, base=100.0, scaling=("linear", 4), device="cpu").frequencies == [f / 4 for f in r.frequencies]
    # 6.28 turns over 2 pi * 10 positions a radian: kept above 4 turns, slowed below 1, halfway at 2.5
    got = sq.Rotary(8, frequencies=None, base=100.0, scaling=("wavelength", 8, 1, 4, 2 * math.pi * 5), device="cpu").frequencies
    turns = [5 * f for f in r.frequencies]
    for f, t, g in zip(r.frequencies, turns, got):
        keep = min(max((t - 1) / 3, 0), 1)
        assert g == pytest.approx(f * (keep + (1 - keep) / 8), rel=1e-12)
    assert sq.Rotary(4, frequencies=[-1.0, 0.0], device="cpu").turns.tolist()[1] == 0


@pytest.mark.parametrize("kw", [dict(channels=3), dict(channels=-2), dict(scaling=("linear", 0)), dict(scaling=("other", 2)),
                                dict(scaling=("linear", 2, 3)), dict(scaling=("wavelength", 8, 4, 1, 100)),
                                dict(frequencies=[1.0]), dict(frequencies=[1.0, math.inf])])
def test_bad_rotaries(sq, kw):
    with pytest.raises(ValueError):
        sq.Rotary(**{**dict(channels=4, device="cpu"), **kw})


def test_the_binding_refuses(sq):
    x = torch.zeros(2, 3, 16, dtype=torch.float16)
    for call in (lambda: sq.rotate_heads(None, x, None), lambda: sq.rotate_heads(None, x.float(), None),
                 lambda: sq.rotate_heads(None, x[0], None), lambda: sq.rotate_heads(sq.Rotary(4, device="cpu"), x, None),
                 lambda: sq.kv_plan(sq.KVPages(4, 16, 2, 3, device="cpu"), torch.zeros(2, dtype=torch.int32),
                                    torch.zeros(2, dtype=torch.int32), 4)):
        with pytest.raises(ValueError):
            call()
    assert sq.rotate_heads(None, None, None) == (None, None)


def attend(sq, **kw):
    a = dict(Q=FAKE, qt=512, qh=64, K=FAKE, kt=128, kh=64, V=FAKE, vt=128, vh=64, starts=FAKE, B=1, n=4, q_heads=8, k_heads=2,
             D=64, Dv=64, dtype=0, causal=1, scale=0.1, out=FAKE, scratch=FAKE, bytes=256)
    assert set(kw) <= set(a)
    a.update(kw)
    return sq.lib().soniq_prompt_attend(*a.values(), None)


@pytest.mark.parametrize("kw,want", [
    (dict(B=0), OK), (dict(n=0), OK), (dict(B=-1), INVALID), (dict(n=-1), INVALID), (dict(n=(1 << 30) + 1), UNSUPPORTED),
    (dict(q_heads=7), INVALID), (dict(q_heads=0), INVALID), (dict(k_heads=0), INVALID), (dict(q_heads=4098), UNSUPPORTED),
    (dict(D=0), INVALID), (dict(Dv=0), INVALID), (dict(D=257), UNSUPPORTED), (dict(Dv=264), UNSUPPORTED), (dict(dtype=3), INVALID),
    (dict(scale=math.inf), INVALID), (dict(scale=math.nan), INVALID), (dict(scale=-0.1), INVALID), (dict(Q=None), INVALID),
    (dict(K=None), INVALID), (dict(V=None), INVALID), (dict(starts=None), INVALID), (dict(out=None), INVALID),
    (dict(Q=FAKE + 1), ALIGNMENT), (dict(K=FAKE + 1), ALIGNMENT), (dict(V=FAKE + 1), ALIGNMENT), (dict(out=FAKE + 1), ALIGNMENT),
    (dict(starts=FAKE + 2), ALIGNMENT), (dict(scratch=None), INVALID), (dict(bytes=255), INVALID), (dict(scratch=FAKE + 8), ALIGNMENT)])
def test_bad_prompts(sq, kw, want):
    assert attend(sq, **kw) == want


def test_prompt_scratch(sq):
    assert sq.lib().soniq_prompt_attend_scratch_bytes() == sq.PROMPT_SCRATCH


def test_the_binding_refuses_prompts(sq):
    x, st = torch.zeros(4, 2, 16, dtype=torch.float16), torch.zeros(2, dtype=torch.int32)
    for args in ((x, x, x, st), (x.float(), x, x, st), (x[0], x, x, st), (x, x[:3], x, st), (x, x[:, :0], x[:, :0], st)):
        with pytest.raises(ValueError):
            sq.prompt_attend(*args)
