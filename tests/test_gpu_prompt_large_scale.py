"""Scales whose product with log2(e) passes fp32: the softmax of scores that are tiny, all
the same, or far apart, is what its definition says."""
import pytest

from test_gpu_prompt_attend import BF16, check, draw, ints, sq  # noqa: F401

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("scale", [1e38, 2.2e38, 2.4e38, 3.4e38])
@pytest.mark.parametrize("D", [64, 256, 33])
def test_large_scales(sq, scale, D):  # noqa: F811
    lens = [150, 1, 70]
    q, k, v, starts = draw(31, lens, 2, 2, D, D, BF16)
    tiny = (5 / scale) ** 0.5           # products of 5 / scale, which are normal numbers: scores of some 40
    check(sq, (q.float() * tiny).to(BF16), (k.float() * tiny).to(BF16), v, starts, scale=scale)
    check(sq, torch.zeros_like(q), k, v, starts, scale=scale)
    # one key of all the weight, in the definition: scores 1 and 0
    q, k = torch.zeros_like(q), torch.zeros_like(k)
    q[:, :, 0], k[::10, :, 0] = 1.0, 1.0
    check(sq, q, k, v, starts, scale=scale)
    check(sq, q, -k, v, starts, False, scale=scale)
