"""Tracers are refused by the calls that launch kernels on their own: what they
record would never fill the outputs.  (No kernel is reached: without a GPU the
calls would refuse the tensors next.)"""
import pytest
import torch
from torch.fx.experimental.proxy_tensor import make_fx

from paper_2605_30574_gb300 import decoder as K
from paper_2605_30574_gb300.decoder import attention as A
from paper_2605_30574_gb300.decoder import scoring

X, T = torch.zeros(2, 9), torch.zeros(2, 3)
Q, KV, LSE = torch.zeros(3, 4, 64, dtype=torch.bfloat16), torch.zeros(2, 5, 64, dtype=torch.bfloat16), torch.zeros(4, 3)
IDS = torch.zeros(2, 3, dtype=torch.long)
CALLS = {"token_logprobs": (lambda x: scoring.token_logprobs(x, top=1)[1], X),
         "distillation": (lambda x: scoring._distill(x, IDS, T, None, False, 1.0, True, False)[1], X),
         "attention_forward": (lambda q: A.attention_forward(q, KV, KV)[0], Q),
         "attention_backward": (lambda q: A.attention_backward(q, q, KV, KV, q, LSE)[0], Q)}


@pytest.fixture(autouse=True)
def no_device(monkeypatch):
    monkeypatch.setattr(K, "_current_device", lambda: None)
    monkeypatch.setattr(scoring, "_current_device", lambda: None)
    monkeypatch.setattr(scoring, "_launch", lambda *a: None)


@pytest.mark.parametrize("name", CALLS)
def test_a_trace(name):
    f, x = CALLS[name]
    with pytest.raises(RuntimeError, match=f"{name}.*tracer"):
        torch.jit.trace(f, (x,), check_trace=False)


@pytest.mark.parametrize("mode", ["real", "fake", "symbolic"])
@pytest.mark.parametrize("name", CALLS)
def test_a_proxys_graph(name, mode):
    f, x = CALLS[name]
    with pytest.raises(RuntimeError, match=f"{name}.*tracer"):
        make_fx(f, tracing_mode=mode)(x)


def test_other_modes_are_not():
    """A mode that only watches sees the allocations and no more."""
    from torch.utils.flop_counter import FlopCounterMode
    K.untraced("a call")
    with FlopCounterMode(display=False):
        K.untraced("a call")
    with torch.device("cpu"):
        K.untraced("a call")
