"""The cache's C entry points reject bad arguments on the host, before any CUDA
call: bad layouts, caches, sizes, alignments and scratch (so these run on CPU;
no pointer here is ever read)."""
import ctypes

import numpy as np
import pytest

OK, INVALID, UNSUPPORTED, ALIGNMENT = 0, 1, 2, 3
FAKE = 1 << 20                  # an aligned address that no check reads


@pytest.fixture(scope="module")
def sq():
    from paper_2311_14114_gb300 import build, soniq
    build.build()
    soniq.lib()
    return soniq


def rows(sq, D=128, count=(112, 16), bits=(4, 8), n_groups=None, perm=FAKE):
    n = (2 if count[1] else 1) if n_groups is None else n_groups
    return sq.CKvRows(D, n, (ctypes.c_int32 * 2)(*count), (ctypes.c_int32 * 2)(*bits), perm)


def cache(sq, **kw):
    k = kw.pop("k", None) or rows(sq)
    v = kw.pop("v", None) or rows(sq)
    c = sq.CKvCache(kw.pop("heads", 2), kw.pop("page", 16), kw.pop("n_pages", 4), kw.pop("dtype", sq.OUT_F16), k, v)
    for name in ("k_codes", "v_codes", "k_scales", "v_scales"):
        setattr(c, name, kw.pop(name, FAKE))
    assert not kw
    return c


@pytest.mark.parametrize("kw,want", [
    (dict(), 16 * 4 + 32), (dict(D=64, count=(64, 0), bits=(4, 0)), 32), (dict(D=80, count=(67, 13), bits=(2, 8)), 64),
    (dict(D=33, count=(33, 0), bits=(2, 0)), 16), (dict(D=256, count=(256, 0), bits=(8, 8)), 256),
    (dict(D=0, count=(0, 0)), -1), (dict(D=128, count=(128, 16)), -1), (dict(count=(0, 128)), -1),
    (dict(count=(129, -1)), -1), (dict(bits=(3, 8)), -1), (dict(bits=(4, 16)), -1), (dict(n_groups=1), -1),
    (dict(n_groups=3), -1), (dict(D=257, count=(257, 0)), -1), (dict(D=250, count=(249, 1)), -1),
    (dict(D=1 << 30, count=(1 << 30, 0)), -1), (dict(count=(2 ** 31 - 1, 2 ** 31 - 1)), -1)])
def test_row_bytes(sq, kw, want):
    assert sq.lib().soniq_kv_row_bytes(ctypes.byref(rows(sq, **kw))) == want


@pytest.mark.parametrize("kw,want", [
    (dict(), OK), (dict(heads=0), INVALID), (dict(heads=4097), UNSUPPORTED), (dict(page=24), INVALID),
    (dict(page=8), UNSUPPORTED), (dict(page=512), UNSUPPORTED), (dict(page=-16), INVALID), (dict(n_pages=0), INVALID),
    (dict(n_pages=1 << 31), UNSUPPORTED), (dict(dtype=7), INVALID)])
def test_validate(sq, kw, want):
    c = cache(sq, **kw)
    assert sq.lib().soniq_kv_validate(ctypes.byref(c), None, None) == want


def test_validate_permutations(sq):
    good = np.stack([np.random.default_rng(0).permutation(128) for _ in range(2)]).astype(np.int32)
    c = cache(sq)
    check = lambda k, v: sq.lib().soniq_kv_validate(ctypes.byref(c), k.ctypes.data_as(ctypes.c_void_p),
                                                     v.ctypes.data_as(ctypes.c_void_p))
    assert check(good, good) == OK
    for at, value in ((0, -1), (130, 128), (255, good[1, 0])):
        bad = good.copy()
        bad.flat[at] = value
        assert check(bad, good) == INVALID and check(good, bad) == INVALID


def write(sq, c, **kw):
    a = dict(K=FAKE, ks=256, kh=128, V=FAKE, vs=256, vh=128, slots=FAKE, n=0)
    a.update(kw)
    return sq.lib().soniq_kv_write(ctypes.byref(c), *a.values(), None)


def read(sq, c, **kw):
    a = dict(slots=FAKE, n=0, K=FAKE, V=FAKE)
    a.update(kw)
    return sq.lib().soniq_kv_read(ctypes.byref(c), *a.values(), None)


def attend(sq, c, **kw):
    a = dict(Q=FAKE, qs=1024, qt=1024, qh=128, table=FAKE, ts=4, pages=4, lengths=FAKE, mask=None, ms=0, B=1, T=1,
             heads=8, scale=0.1, out=FAKE, scratch=FAKE, bytes=0)
    a.update(kw)
    return sq.lib().soniq_kv_attend(ctypes.byref(c), *a.values(), None)


@pytest.mark.parametrize("call", [write, read, attend])
@pytest.mark.parametrize("kw,want", [
    (dict(k_codes=None), INVALID), (dict(v_scales=None), INVALID), (dict(v_codes=FAKE + 8), ALIGNMENT),
    (dict(k_scales=FAKE + 2), ALIGNMENT), (dict(page=3), INVALID)])
def test_bad_caches(sq, call, kw, want):
    assert call(sq, cache(sq, **kw)) == want


def test_bad_permutation_pointers(sq):
    assert write(sq, cache(sq, k=rows(sq, perm=None))) == INVALID
    assert write(sq, cache(sq, v=rows(sq, perm=FAKE + 2))) == ALIGNMENT


@pytest.mark.parametrize("kw,want", [
    (dict(), OK), (dict(n=-1), INVALID), (dict(n=1 << 41), UNSUPPORTED), (dict(n=1, slots=None), INVALID),
    (dict(n=1, K=None), INVALID), (dict(n=1, V=FAKE + 1), ALIGNMENT), (dict(n=1, slots=FAKE + 4), ALIGNMENT)])
def test_bad_writes(sq, kw, want):
    assert write(sq, cache(sq), **kw) == want


@pytest.mark.parametrize("kw,want", [
    (dict(), OK), (dict(n=5, K=None, V=None), OK), (dict(n=-1), INVALID), (dict(n=1 << 41), UNSUPPORTED),
    (dict(n=1, slots=None), INVALID), (dict(n=1, K=FAKE + 1), ALIGNMENT), (dict(n=1, slots=FAKE + 4), ALIGNMENT)])
def test_bad_reads(sq, kw, want):
    assert read(sq, cache(sq), **kw) == want


@pytest.mark.parametrize("kw,want", [
    (dict(B=0), OK), (dict(T=0), OK), (dict(B=-1), INVALID), (dict(T=-1), INVALID), (dict(heads=0), INVALID),
    (dict(heads=7), INVALID), (dict(pages=-1), INVALID), (dict(scale=float("inf")), INVALID),
    (dict(scale=float("nan")), INVALID), (dict(T=1 << 26), UNSUPPORTED), (dict(pages=1 << 27), UNSUPPORTED),
    (dict(Q=None), INVALID), (dict(out=None), INVALID), (dict(lengths=None), INVALID), (dict(table=None), INVALID),
    (dict(Q=FAKE + 1), ALIGNMENT), (dict(lengths=FAKE + 2), ALIGNMENT), (dict(table=FAKE + 2), ALIGNMENT)])
def test_bad_attends(sq, kw, want):
    assert attend(sq, cache(sq), **kw) == want


def test_scratch(sq):
    size = lambda B, T, heads: sq.lib().soniq_kv_attend_scratch_bytes(ctypes.byref(cache(sq)), B, T, heads)
    assert size(-1, 1, 8) == -1 and size(1, -1, 8) == -1 and size(1, 1, 7) == -1 and size(1, 1, 0) == -1
    for T in (1, 4, 64):
        assert size(1, T, 8) > 0
        assert attend(sq, cache(sq), T=T, bytes=size(1, T, 8) - 1) == INVALID
        assert attend(sq, cache(sq), T=T, scratch=None, bytes=size(1, T, 8)) == INVALID
        assert attend(sq, cache(sq), T=T, scratch=FAKE + 8, bytes=size(1, T, 8)) == ALIGNMENT


def test_python_layouts(sq):
    perm = np.arange(64).reshape(1, 64)
    assert sq.KVLayout(perm, (48, 16), (4, 8)).row_bytes == 64
    for bad in (dict(perm=np.arange(64)), dict(perm=perm, count=(48, 15)), dict(perm=perm, bits=(5, 8))):
        kw = dict(perm=perm, count=(48, 16), bits=(4, 8))
        kw.update(bad)
        with pytest.raises((ValueError, sq.SoniqError)):
            sq.KVLayout(**kw)
    lay, two = sq.KVLayout(perm, (64, 0), (8, 8)), sq.KVLayout(np.stack([perm[0]] * 2), (64, 0), (8, 8))
    import torch
    for kw in (dict(v=two), dict(page_size=20), dict(n_pages=0), dict(dtype=torch.float32)):
        a = dict(k=lay, v=lay, n_pages=1, page_size=16)
        a.update(kw)
        with pytest.raises((ValueError, sq.SoniqError)):
            sq.KVCache(**a, device="cpu")
    dup = perm.copy()
    dup[0, 3] = 4
    with pytest.raises(sq.SoniqError):
        sq.KVCache(sq.KVLayout(dup, (64, 0), (8, 8)), lay, 1, 16, device="cpu")
