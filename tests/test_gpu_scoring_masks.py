"""Divergences where logits are masked."""
import pytest
import torch

from paper_2605_30574_gb300 import build as B
from paper_2605_30574_gb300 import decoder as K
from paper_2605_30574_gb300.decoder import scoring

pytestmark = pytest.mark.gpu
INF = float("inf")


@pytest.fixture(scope="module", autouse=True)
def _built():
    B.build()
    yield
    K.check_device_error()


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("top", [5, 33, 40, 64, 65, 128])
def test_tokens_that_cannot_be_said_among_many(top, rest):
    """One alternative of -inf among others: the loss is +inf wherever it stands."""
    V = 3001
    g = torch.Generator(device="cuda")
    g.manual_seed(top)
    x = torch.randn(top + 1, V, generator=g, device="cuda")
    ids = torch.rand(top + 1, V, generator=g, device="cuda").topk(top, -1).indices
    teacher = torch.log_softmax(torch.randn(top + 1, top, generator=g, device="cuda"), -1) - 0.1
    at = torch.arange(top, device="cuda")
    x[at, ids[at, at]] = -INF
    loss, grad = scoring.distill_loss_and_grad(x, ids, teacher, rest=rest)
    assert bool((loss[:top] == INF).all()), loss
    assert bool(loss[top].isfinite()) and bool(grad.isfinite().all())
    assert torch.equal(scoring.distill_loss(x, ids, teacher, rest=rest), loss)
