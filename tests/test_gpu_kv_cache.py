"""Key / value cache: rows written as codes, and read back, bit for bit."""
import numpy as np
import pytest
import torch

import kv_plain as plain

pytestmark = pytest.mark.gpu

# heads, D, Dv, (k counts, bits), (v counts, bits)
LAYOUTS = [
    (8, 128, 128, ([96, 32], [4, 8]), ([128], [4])),
    (2, 64, 64, ([51, 13], [2, 8]), ([59, 5], [4, 8])),
    (3, 80, 80, ([67, 13], [4, 8]), ([75, 5], [2, 4])),
    (1, 256, 256, ([192, 64], [4, 8]), ([256], [8])),
    (5, 40, 64, ([8, 32], [8, 4]), ([64], [2])),
    (2, 1, 3, ([1], [8]), ([2, 1], [4, 2])),
    (1, 97, 33, ([97], [2]), ([33], [4])),
    (12, 192, 128, ([187, 5], [4, 8]), ([112, 16], [4, 8])),
]


@pytest.fixture(scope="module")
def sq():
    from paper_2311_14114_gb300 import soniq
    return soniq


def make_layout(sq, rng, heads, D, spec):
    perm = np.stack([rng.permutation(D) for _ in range(heads)]).astype(np.int32)
    return sq.KVLayout(perm, *spec)


def make_cache(sq, rng, shape, n_pages, page, dtype):
    heads, D, Dv, ks, vs = shape
    return sq.KVCache(make_layout(sq, rng, heads, D, ks), make_layout(sq, rng, heads, Dv, vs), n_pages, page, dtype)


def rows(rng, n, heads, D, dtype):
    x = rng.standard_normal((n, heads, D)) * np.exp(0.5 * rng.standard_normal((n, heads, 1)))
    return torch.from_numpy(x).to(dtype)


def check_rows(cache, slots, k, v):
    """Packed bytes and scales of every written slot."""
    for x, lay, codes, scales in ((k, cache.k, cache.k_codes, cache.k_scales), (v, cache.v, cache.v_codes, cache.v_scales)):
        codes, scales = codes.cpu().numpy(), scales.double().cpu().numpy()
        x = x.double().numpy()
        for i, slot in enumerate(slots):
            if slot < 0 or slot >= cache.n_pages * cache.page_size:
                continue
            p, t = divmod(int(slot), cache.page_size)
            for h in range(cache.heads):
                want, s = plain.row_bytes(lay, h, x[i, h], cache.dtype)
                assert np.array_equal(codes[p, h, t], want), (i, h)
                assert np.array_equal(scales[p, h, t], s), (i, h)


def check_values(cache, x, lay, got):
    want = torch.from_numpy(plain.values(lay, x.double().numpy(), cache.dtype)).to(cache.dtype)
    assert torch.equal(got.cpu(), want)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("shape", LAYOUTS)
@pytest.mark.parametrize("n,page", [(1, 16), (37, 16), (50, 64)])
def test_write_then_read(sq, shape, n, page, dtype):
    rng = np.random.default_rng(n + shape[1])
    heads, D, Dv = shape[:3]
    cache = make_cache(sq, rng, shape, 6, page, dtype)
    k, v = rows(rng, n, heads, D, dtype), rows(rng, n, heads, Dv, dtype)
    slots = rng.permutation(6 * page)[:n].astype(np.int64)
    dslots = torch.from_numpy(slots).cuda()
    sq.kv_write(cache, k.cuda(), v.cuda(), dslots)
    check_rows(cache, slots, k, v)
    gk, gv = sq.kv_read(cache, dslots)
    check_values(cache, k, cache.k, gk)
    check_values(cache, v, cache.v, gv)
    assert sq.sync_status() == 0


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("shape", [LAYOUTS[0], LAYOUTS[2]])
@pytest.mark.parametrize("offset", [0, 1, 8])
def test_slices_of_a_fused_projection(sq, shape, offset, dtype):
    """Token and head strides, rows off every alignment but two bytes; nothing beside them is read into a row."""
    rng = np.random.default_rng(offset)
    heads, D, Dv = shape[:3]
    n, page = 77, 32
    cache = make_cache(sq, rng, shape, 4, page, dtype)
    width = offset + heads * (D + Dv) + 3
    qkv = torch.full((n, width), float("nan"), dtype=dtype)
    k, v = rows(rng, n, heads, D, dtype), rows(rng, n, heads, Dv, dtype)
    qkv[:, offset:offset + heads * D] = k.reshape(n, -1)
    qkv[:, offset + heads * D:offset + heads * (D + Dv)] = v.reshape(n, -1)
    dev = qkv.cuda()
    slots = rng.permutation(4 * page)[:n].astype(np.int64)
    dslots = torch.from_numpy(slots).cuda()
    sq.kv_write(cache, dev[:, offset:offset + heads * D].view(n, heads, D),
                dev[:, offset + heads * D:offset + heads * (D + Dv)].view(n, heads, Dv), dslots)
    check_rows(cache, slots, k, v)
    # heads before tokens
    cache2 = sq.KVCache(cache.k, cache.v, 4, page, dtype)
    kt, vt = k.transpose(0, 1).contiguous().cuda(), v.transpose(0, 1).contiguous().cuda()
    sq.kv_write(cache2, kt.transpose(0, 1), vt.transpose(0, 1), dslots)
    for name in ("k_codes", "v_codes", "k_scales", "v_scales"):
        assert torch.equal(getattr(cache, name), getattr(cache2, name)), name


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_special_values(sq, dtype):
    """Zero rows, NaN, infinities, subnormals, the largest values, ties between two codes."""
    rng = np.random.default_rng(3)
    shape = LAYOUTS[0]
    heads, D, Dv = shape[:3]
    cache = make_cache(sq, rng, shape, 2, 16, dtype)
    n = 12
    k, v = rows(rng, n, heads, D, dtype), rows(rng, n, heads, Dv, dtype)
    tiny = 2.0 ** -24 if dtype == torch.float16 else 2.0 ** -133
    for x in (k, v):
        x[0] = 0
        x[1, :, 5] = float("nan")
        x[2] = float("nan")
        x[3, :, 7] = float("inf")
        x[4, :, 9] = float("-inf")
        x[5] = torch.from_numpy(rng.integers(-9, 10, (heads, x.shape[-1])) * tiny).to(dtype)
        x[6] = x[6] * (3e4 if dtype == torch.float16 else 1e38) / x[6].abs().amax().clamp(min=1)
        x[7] = torch.from_numpy(rng.integers(-16, 17, (heads, x.shape[-1])) / 16.0).to(dtype)     # ties of 4-bit codes
        x[8] = torch.from_numpy(rng.integers(-256, 257, (heads, x.shape[-1])) / 256.0).to(dtype)  # and of 8-bit ones
        x[9] = torch.finfo(dtype).max
        x[10] = -0.0
        x[11] = x[11] * tiny * 100
    slots = np.arange(n, dtype=np.int64)[::-1].copy() + 3
    dslots = torch.from_numpy(slots).cuda()
    sq.kv_write(cache, k.cuda(), v.cuda(), dslots)
    check_rows(cache, slots, k, v)
    gk, gv = sq.kv_read(cache, dslots)
    check_values(cache, k, cache.k, gk)
    check_values(cache, v, cache.v, gv)
    assert torch.isfinite(gk).all() and torch.isfinite(gv).all()


def test_skipped_and_bad_slots(sq):
    rng = np.random.default_rng(4)
    shape = LAYOUTS[1]
    cache = make_cache(sq, rng, shape, 2, 16, torch.float16)
    k, v = rows(rng, 4, 2, 64, torch.float16), rows(rng, 4, 2, 64, torch.float16)
    sq.kv_write(cache, k.cuda(), v.cuda(), torch.tensor([3, -1, 31, -5], device="cuda"))
    assert sq.sync_status() == 0
    check_rows(cache, [3, -1, 31, -5], k, v)
    gk, gv = sq.kv_read(cache, torch.tensor([-1, 3], device="cuda"))
    assert not gk[0].any() and not gv[0].any() and gk[1].any()
    assert sq.sync_status() == 0
    before = cache.k_codes.clone()
    sq.kv_write(cache, k.cuda(), v.cuda(), torch.tensor([32, 3, 1 << 40, -1], device="cuda"))
    assert sq.sync_status() == sq.SONIQ_ERR_INVALID_ARG
    assert sq.sync_status() == 0
    check_rows(cache, [32, 3, 1 << 40, -1], k, v)
    changed = (cache.k_codes != before).any(-1).nonzero()
    assert {tuple(c.tolist()) for c in changed} <= {(0, 0, 3), (0, 1, 3)}
    gk, _ = sq.kv_read(cache, torch.tensor([1 << 33, 3], device="cuda"))
    assert sq.sync_status() == sq.SONIQ_ERR_INVALID_ARG and not gk[0].any() and gk[1].any()


def test_no_tokens_and_one_side(sq):
    rng = np.random.default_rng(5)
    cache = make_cache(sq, rng, LAYOUTS[0], 2, 16, torch.float16)
    none = torch.empty(0, dtype=torch.int64, device="cuda")
    e = torch.empty(0, 8, 128, dtype=torch.float16, device="cuda")
    sq.kv_write(cache, e, e, none)
    gk, gv = sq.kv_read(cache, none)
    assert gk.shape == (0, 8, 128) and gv.shape == (0, 8, 128)


def test_rows_beyond_32_bit_offsets(sq):
    """Slots whose codes lie more than 2^32 bytes into the cache."""
    rng = np.random.default_rng(6)
    shape = (8, 128, 128, ([96, 32], [4, 8]), ([128], [8]))
    pages = (1 << 32) // (8 * 16 * 80) + 300
    cache = make_cache(sq, rng, shape, pages, 16, torch.float16)
    k, v = rows(rng, 3, 8, 128, torch.float16), rows(rng, 3, 8, 128, torch.float16)
    slots = torch.tensor([pages * 16 - 1, 5, pages * 16 - 4000], device="cuda")
    sq.kv_write(cache, k.cuda(), v.cuda(), slots)
    gk, gv = sq.kv_read(cache, slots)
    check_values(cache, k, cache.k, gk)
    check_values(cache, v, cache.v, gv)
    table = torch.tensor([[pages - 1]], dtype=torch.int32, device="cuda")
    q = rows(rng, 1, 8, 128, torch.float16).view(1, 1, 8, 128)
    # the last page holds one token: attention over it alone gives its value
    cache.k_codes[pages - 1, :, 0] = cache.k_codes[pages - 1, :, 15]
    cache.k_scales[pages - 1, :, 0] = cache.k_scales[pages - 1, :, 15]
    cache.v_codes[pages - 1, :, 0] = cache.v_codes[pages - 1, :, 15]
    cache.v_scales[pages - 1, :, 0] = cache.v_scales[pages - 1, :, 15]
    o = sq.kv_attend(cache, q.cuda(), table, torch.zeros(1, dtype=torch.int32, device="cuda"))
    # one weight of 1: the value's own rounding, and fp16's of the weight times its scale
    want = gv[0].double()
    assert ((o[0, 0].double() - want).abs() <= want.abs() * 2.0 ** -10 + 2.0 ** -24).all()
    assert sq.sync_status() == 0


def test_refusals(sq):
    rng = np.random.default_rng(7)
    eye = np.arange(64, dtype=np.int32)[None]
    with pytest.raises(sq.SoniqError):
        sq.KVLayout(eye, [64], [3])            # a width outside 2, 4, 8
    with pytest.raises(sq.SoniqError):
        sq.KVLayout(eye, [60], [4])            # groups that miss channels
    with pytest.raises(sq.SoniqError):
        sq.KVLayout(eye, [0, 64], [4, 8])
    with pytest.raises(sq.SoniqError):
        sq.KVLayout(np.arange(257, dtype=np.int32)[None], [257], [4])
    with pytest.raises(sq.SoniqError):
        sq.KVLayout(np.arange(256, dtype=np.int32)[None], [243, 13], [4, 8])   # 288 padded codes
    ok = sq.KVLayout(eye, [64], [4])
    bad = sq.KVLayout(np.zeros((1, 64), np.int32), [64], [4])
    with pytest.raises(sq.SoniqError):
        sq.KVCache(bad, ok, 2, 16)             # not a permutation
    for page in (0, 8, 24, 512):
        with pytest.raises(sq.SoniqError):
            sq.KVCache(ok, ok, 2, page)
    with pytest.raises(ValueError):
        sq.KVCache(ok, ok, 2, 16, dtype=torch.float32)
    two = sq.KVLayout(np.concatenate([eye, eye]), [64], [4])
    with pytest.raises(ValueError):
        sq.KVCache(ok, two, 2, 16)
    cache = sq.KVCache(ok, ok, 2, 16)
    x = torch.zeros(3, 1, 64, dtype=torch.float16, device="cuda")
    slots = torch.arange(3, device="cuda")
    for bad_args in ((x.float(), x, slots), (x, x[:2], slots), (x, x, slots.int()), (x.cpu(), x, slots),
                     (x.transpose(1, 2).contiguous().transpose(1, 2)[:, :, ::2], x, slots)):
        with pytest.raises(ValueError):
            sq.kv_write(cache, *bad_args)
    with pytest.raises(ValueError):
        sq.kv_read(cache, slots, k=torch.empty(2, 1, 64, dtype=torch.float16, device="cuda"))


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_many_rows_of_unequal_sides(sq, dtype):
    """Keys' rows take more lanes than values': many tokens at once equal the same tokens in small calls."""
    rng = np.random.default_rng(16)
    n, shape = 16384 + 21, (8, 128, 128, ([112, 16], [4, 8]), ([128], [4]))
    caches = [make_cache(sq, np.random.default_rng(17), shape, n // 16 + 2, 16, dtype) for _ in range(2)]
    k, v = (torch.from_numpy(rng.standard_normal((n, 8, 128)).astype(np.float32)).to(dtype).cuda() for _ in range(2))
    slots = torch.from_numpy(rng.permutation(n + 16)[:n]).cuda()
    slots[5] = -1
    sq.kv_write(caches[0], k, v, slots)
    for i in range(0, n, 4001):
        sq.kv_write(caches[1], k[i:i + 4001], v[i:i + 4001], slots[i:i + 4001])
    for name in ("k_codes", "k_scales", "v_codes", "v_scales"):
        assert torch.equal(getattr(caches[0], name), getattr(caches[1], name))
    got = sq.kv_read(caches[0], slots)
    for i in range(0, n, 4001):
        part = sq.kv_read(caches[1], slots[i:i + 4001].contiguous())
        for a, b in zip(got, part):
            assert torch.equal(a[i:i + 4001], b)
    assert sq.sync_status() == 0
