"""The gradients' scratch is as large as the library says."""
import pytest
import torch

from paper_2605_30574_gb300 import build as B
from paper_2605_30574_gb300 import decoder as K
from paper_2605_30574_gb300.decoder import attention as A

pytestmark = pytest.mark.gpu


def test_scratch_is_the_librarys(monkeypatch):
    B.build()
    L, asked, made = K.lib(), [], []
    size, empty = L.decoder_attention_scratch, torch.empty
    monkeypatch.setattr(L, "decoder_attention_scratch", lambda *a: asked.append(a) or size(*a))
    q, k = (torch.randn(2, *s, device="cuda").bfloat16() for s in ((130, 4, 64), (2, 200, 64)))
    out, lse = A.attention_forward(q, k, k)
    monkeypatch.setattr(torch, "empty", lambda *a, **b: made.append(a[0]) or empty(*a, **b))
    A.attention_backward(q, q, k, k, out, lse)
    assert asked == [(2, 130, 4)] and size(2, 130, 4) in made
    K.check_device_error()
