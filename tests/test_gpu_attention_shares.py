"""Attention whose keys several CTAs share, against the definition in fp64.

P goes into its product in two bf16 terms, so what is left is fp32 and the
output's own rounding: scores of size s are off by about 2^-20 (1 + s), and P by
as much, relatively; 2^-16 of P |V| covers that, and 2^-18 (1 + |lse|) the log
sums.  The output is rounded to 8 bits: 2^-8 of it.
"""
import math

import pytest
import torch

from paper_2605_30574_gb300 import build as B
from paper_2605_30574_gb300 import decoder as K
from paper_2605_30574_gb300.decoder import attention as A

pytestmark = pytest.mark.gpu
NONE = float("-inf")


@pytest.fixture(scope="module", autouse=True)
def _built():
    B.build()
    yield
    K.check_device_error()


# one token; a few blocks; shares that early rows see nothing of; rows that see
# nothing at all; tiles of unlike length; keys that end inside a block
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("batch,Tq,Tk,Hq,Hkv", [(1, 1, 256, 2, 1), (1, 1, 2049, 4, 2), (2, 128, 512, 2, 2), (1, 300, 300, 4, 1),
                                                (1, 400, 300, 2, 2), (3, 100, 4001, 8, 2), (1, 1000, 1000, 2, 1)])
def test_forward(batch, Tq, Tk, Hq, Hkv, d):
    g = torch.Generator(device="cuda")
    g.manual_seed(Tq + 10 * Tk + d)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
    q, k, v = r(batch, Tq, Hq, d) * 2, r(batch, Hkv, Tk, d), r(batch, Hkv, Tk, d)
    scale, G = 1.0 / math.sqrt(d), Hq // Hkv
    out, lse = A.attention_forward(q, k, v)
    again = A.attention_forward(q, k, v)
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])
    qh, kh, vh = q.double().transpose(1, 2), k.double().repeat_interleave(G, 1), v.double().repeat_interleave(G, 1)
    seen = torch.arange(Tk, device="cuda")[None] <= torch.arange(Tq, device="cuda")[:, None] + (Tk - Tq)
    s = (scale * (qh @ kh.transpose(-1, -2))).masked_fill(~seen, NONE)
    want = torch.logsumexp(s, -1)
    some = want != NONE
    p = torch.where(seen, (s - want.masked_fill(~some, 0.0)[..., None]).exp(), torch.zeros_like(s))
    o = p @ vh
    assert torch.equal(lse == NONE, ~some)
    assert bool(((lse.double() - want).abs()[some] <= 2.0 ** -18 * (1 + want.abs()[some])).all())
    off = 2.0 ** -16 * (p @ vh.abs()) + 2.0 ** -8 * o.abs() + 1e-30
    assert float(((out.double().transpose(1, 2) - o).abs() / off).max()) <= 1.0


def test_masked_lowest_scores():
    # scores down to about -1e37, whole shares of them
    q = torch.full((1, 1, 1, 64), 1e18, device="cuda").to(torch.bfloat16)
    k = torch.full((1, 1, 512, 64), -1e18, device="cuda").to(torch.bfloat16)
    k[:, :, 130:140] = 0
    v = torch.randn(1, 1, 512, 64, device="cuda").to(torch.bfloat16)
    out, lse = A.attention_forward(q, k, v)
    want = v[0, 0, 130:140].double().mean(0)
    assert abs(float(lse) - math.log(10)) <= 2.0 ** -18 * (1 + math.log(10))
    off = 2.0 ** -8 * want.abs() + 2.0 ** -16 * v[0, 0, 130:140].double().abs().mean(0)
    assert bool(((out[0, 0, 0].double() - want).abs() <= off).all())
