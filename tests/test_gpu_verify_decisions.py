"""GPU tests of the verification of drafted tokens where a decision or a draw hangs on one
number: drafted ids outside the vocabulary, rows whose largest logits are far apart, logits
whose difference is no fp32 number, residuals that leave nothing."""
import pytest
import torch

from tests.gpu_util import require_gpu
from tests.test_gpu_verify import TD, call

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    require_gpu()
    yield
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [50, 28672, 50001])
def test_drafted_ids_far_outside_the_vocabulary(V, dtype):
    """Such an id has p = 0 and takes nothing from p: the token that its lowest 32 bits name,
    which has nearly all of the probability, is drawn."""
    S, k = 5, 2
    v = torch.tensor([0, V // 3, V - 1, V // 2, 7])
    x = torch.zeros((S, k + 1, V))
    x[torch.arange(S), :, v] = 30.0
    high = torch.tensor([2 ** 32, 2 ** 40, 2 ** 62, 2 ** 32 * 5, 2 ** 33])
    ids = torch.stack([high + v, v], 1)
    u = torch.zeros((S, k))
    e = 0.5 + torch.rand((S, V), generator=torch.Generator().manual_seed(V))
    op = call(S, k, V, dtype, (x.view(-1, V).to(TD[dtype]), ids, u, e, None), "tokens", least=S)
    assert op.accepted.tolist() == [0] * S
    assert op.tokens[:, 0].cpu().tolist() == v.tolist()
