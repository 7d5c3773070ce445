"""Arguments without memory are refused, whichever it is."""
import pytest
import torch

from paper_2605_30574_gb300 import build as B
from paper_2605_30574_gb300 import decoder as K
from paper_2605_30574_gb300.decoder import attention as A
from paper_2605_30574_gb300.decoder import scoring

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def _built():
    B.build()
    yield
    K.check_device_error()


def zeros(like):
    return torch._efficientzerotensor(tuple(like.shape), dtype=like.dtype, device="cuda")


def freed(like):
    t = like.clone()
    t.untyped_storage().resize_(0)
    return t


@pytest.mark.parametrize("nothing", [zeros, freed])
def test_arguments_without_memory(nothing):
    x, tokens = torch.zeros(4, 300, device="cuda"), torch.zeros(4, dtype=torch.long, device="cuda")
    ids, teacher, weight = torch.zeros(4, 3, dtype=torch.long, device="cuda"), torch.zeros(4, 3, device="cuda"), torch.ones(4, device="cuda")
    q, k, v = (torch.zeros(*s, dtype=BF, device="cuda") for s in ((5, 4, 64), (2, 7, 64), (2, 7, 64)))
    out, lse = A.attention_forward(q, k, v)
    args = {scoring.token_logprobs: (x, tokens), scoring.distill_loss: (x, ids, teacher), scoring.distill_loss_and_grad: (x, ids, teacher),
            A.attention: (q, k, v), A.attention_forward: (q, k, v), A.attention_backward: (q, q, k, v, out, lse)}
    for f, a in args.items():
        f(*a)
        for i in range(len(a)):
            with pytest.raises(ValueError, match="no memory"):
                f(*a[:i], nothing(a[i]), *a[i + 1:])
    with pytest.raises(ValueError, match="no memory"):
        scoring.distill_loss(x, ids, teacher, weight=nothing(weight))
