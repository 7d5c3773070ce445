"""Scores, divergences and attention under tracers and compilers: refused, or the
values that the call itself gives."""
import pytest
import torch
from torch.fx.experimental.proxy_tensor import make_fx

from paper_2605_30574_gb300 import build as B
from paper_2605_30574_gb300 import decoder as K
from paper_2605_30574_gb300.decoder import attention as A
from paper_2605_30574_gb300.decoder import scoring

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def calls():
    B.build()
    g = torch.Generator(device="cuda")
    g.manual_seed(0)
    x, y = (torch.randn(4, 300, generator=g, device="cuda") for _ in range(2))
    q, k, v = (torch.randn(*s, generator=g, device="cuda").bfloat16() for s in ((9, 4, 64), (2, 9, 64), (2, 9, 64)))
    ids = torch.tensor([[3, 250]], device="cuda").repeat(4, 1)
    t = torch.full((4, 2), 0.4, device="cuda").log()
    out, lse = A.attention_forward(q, k, v)
    r = q.flip(0).contiguous()
    yield {"scores": (lambda z: scoring.token_logprobs(z, top=3)[1], x, y),
           "loss": (lambda z: scoring.distill_loss(z, ids, t), x, y),
           "loss and gradient": (lambda z: scoring.distill_loss_and_grad(z, ids, t)[1], x, y),
           "attention": (lambda z: A.attention(z, k, v), q, r),
           "forward": (lambda z: A.attention_forward(z, k, v)[0], q, r),
           "backward": (lambda z: A.attention_backward(z, q, k, v, out, lse)[0], q, r)}
    K.check_device_error()


NAMES = ["scores", "loss", "loss and gradient", "attention", "forward", "backward"]


@pytest.mark.parametrize("name", NAMES)
def test_what_a_tracer_makes_is_right_or_refused(calls, name):
    f, x, y = calls[name]
    want = f(y)
    if name in ("loss", "attention"):       # (recorded as the functions that they are)
        g = torch.jit.trace(f, (x,), check_trace=False)
        assert torch.equal(g(y), want) and torch.equal(g(x), f(x))
    else:
        with pytest.raises(RuntimeError, match="tracer"):
            torch.jit.trace(f, (x,), check_trace=False)
    with pytest.raises(RuntimeError, match="tracer"):
        make_fx(f)(x)


@pytest.mark.parametrize("backend", ["eager", "aot_eager"])
@pytest.mark.parametrize("name", NAMES)
def test_compilers_run_the_calls(calls, name, backend):
    f, x, y = calls[name]
    torch._dynamo.reset()
    g = torch.compile(f, backend=backend)
    assert torch.equal(g(x), f(x)) and torch.equal(g(y), f(y))
    if name in ("loss", "attention"):
        grads = []
        for h in (f, g):
            leaf = y.clone().requires_grad_()
            grads += torch.autograd.grad(h(leaf).float().square().sum(), leaf)
        assert torch.equal(*grads)
    torch._dynamo.reset()
