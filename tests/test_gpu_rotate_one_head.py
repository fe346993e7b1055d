"""One head, whose stride may be any number: rows stay on their 16 bytes, whatever it says."""
import numpy as np
import pytest

from test_gpu_rotate import BF16, F16, check, positions_of, rows, sq  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def strided(x, head_stride):
    """The rows [n][1][D] in memory of their own, with that stride of their one head."""
    n, _, D = x.shape
    y = torch.empty(n * D, dtype=x.dtype, device="cuda").as_strided((n, 1, D), (D, head_stride, 1))
    return y.copy_(x)


@pytest.mark.parametrize("D,channels,interleaved", [(128, 128, False), (64, 40, False), (80, 32, True), (256, 256, False)])
@pytest.mark.parametrize("stride", [0, 1, 3, 2 ** 33 + 1])
@pytest.mark.parametrize("n", [1, 2, 700])
def test_a_lone_head_of_any_stride(sq, D, channels, interleaved, stride, n):  # noqa: F811
    rng = np.random.default_rng(D + n)
    rotary, pos = sq.Rotary(channels, interleaved=interleaved), positions_of(rng, n)
    gain = torch.from_numpy((1 + 0.3 * rng.standard_normal(D)).astype(np.float32)).cuda()
    q, k = rows(rng, (n, 1, D), BF16), rows(rng, (n, 1, D), BF16)
    want = check(sq, q, k, rotary, pos, (gain, None))
    to = [strided(torch.zeros_like(x), stride) for x in (q, k)]
    got = check(sq, strided(q, stride), strided(k, stride), rotary, pos, (gain, None), q_out=to[0], k_out=to[1])
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and got[0].data_ptr() == to[0].data_ptr()
    # beside a side of several heads, and in place
    many = rows(rng, (n, 5, D), F16)
    alone = sq.rotate_heads(rotary, many, None, pos)[0]
    one = strided(q.half(), stride)
    got = check(sq, many, one, rotary, pos, k_out=one)
    assert torch.equal(got[0], alone) and got[1].data_ptr() == one.data_ptr()
    assert sq.sync_status() == 0
