"""The prefill's causal attention over more heads than attention with log sums
takes.  Of one key, the output is its value, bit for bit."""
import pytest
import torch

from paper_2605_30574_gb300 import build as B
from paper_2605_30574_gb300 import decoder as K

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def test_a_million_heads():
    B.build()
    g = torch.Generator(device="cuda")
    g.manual_seed(0)
    H = (1 << 20) + 3
    q = torch.randn(1, H, 64, generator=g, device="cuda").to(BF)
    k, v = (torch.randn(1, 1, 64, generator=g, device="cuda").to(BF) for _ in range(2))
    out = K.causal(q, k, v, 0.125)
    assert torch.equal(out, v.expand_as(out.transpose(0, 1)).transpose(0, 1))
    K.check_device_error()
