"""A copy of keys and values that never comes: the waits run out, the CTA gives up,
and the next call is right."""
import pytest

from test_gpu_prompt_attend import check, draw

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def sq():
    from paper_2311_14114_gb300 import build, soniq
    build.build()
    soniq.lib()
    return soniq


@pytest.mark.parametrize("lens,D,causal", [([40], 64, True), ([700, 20], 128, True), ([300], 256, False), ([900] * 8, 128, False)])
def test_lost_copy(sq, lens, D, causal):
    args = draw(D, lens, 2, 4, D, D, torch.bfloat16)
    st = torch.tensor(args[3], dtype=torch.int32, device="cuda")
    sq.test_drop_barrier_arrival()
    sq.prompt_attend(*args[:3], st, causal)
    assert sq.sync_status() == sq.SONIQ_ERR_TIMEOUT
    assert sq.sync_status() == 0
    check(sq, *args, causal)
