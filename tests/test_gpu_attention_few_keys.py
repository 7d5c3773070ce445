"""The gradients of attention over a few keys, from an output that is wrong.

Up to 32 keys, the row's delta = dO . O is put right by the row's own sum of dS,
so it does not matter what the output was rounded to, or whether it is there.
With P and dS rounded to bf16 (u = 2^-8) and fp32 elsewhere, dS is then off by
u |dS|, and by what fp32 leaves of P (|dP| + sum P |dP|) and of the sums |dO| |V|
that dP is made of: scores of size s, and so P, are off by about 2^-20 (1 + s),
and 2^-16 of these covers that.  dK and dQ add it up with |Q| and |K|, and have
their own rounding, u |value|, on top.
"""
import math

import pytest
import torch

from paper_2605_30574_gb300 import build as B
from paper_2605_30574_gb300 import decoder as K
from paper_2605_30574_gb300.decoder import attention as A

pytestmark = pytest.mark.gpu
U, FP32 = 2.0 ** -8, 2.0 ** -16


@pytest.fixture(scope="module", autouse=True)
def _built():
    B.build()
    yield
    K.check_device_error()


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("batch,Tq,Tk,Hq,Hkv", [(1, 1, 2, 2, 1), (2, 3, 3, 4, 4), (1, 17, 17, 8, 1), (3, 5, 31, 6, 2), (1, 32, 32, 4, 2),
                                                (2, 150, 32, 4, 1), (1, 64, 9, 2, 2)])
def test_output_does_not_matter(batch, Tq, Tk, Hq, Hkv, d):
    g = torch.Generator(device="cuda")
    g.manual_seed(Tq * 100 + Tk)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
    q, k, v, dout = r(batch, Tq, Hq, d), r(batch, Hkv, Tk, d), r(batch, Hkv, Tk, d), r(batch, Tq, Hq, d)
    scale, G = 1.0 / math.sqrt(d), Hq // Hkv
    out, lse = A.attention_forward(q, k, v)
    qh, gh = q.double().transpose(1, 2), dout.double().transpose(1, 2)
    kh, vh = k.double().repeat_interleave(G, 1), v.double().repeat_interleave(G, 1)
    seen = torch.arange(Tk, device="cuda")[None] <= torch.arange(Tq, device="cuda")[:, None] + (Tk - Tq)
    p = torch.softmax((scale * (qh @ kh.transpose(-1, -2))).masked_fill(~seen, -1e300), -1) * seen
    dp = gh @ vh.transpose(-1, -2)
    ds = p * (dp - (p * dp).sum(-1, keepdim=True))
    sums = gh.abs() @ vh.abs().transpose(-1, -2)
    off = U * ds.abs() + FP32 * p * (sums + (p * sums).sum(-1, keepdim=True))
    fold = lambda x: x.unflatten(1, (Hkv, G)).sum(2)  # noqa: E731
    dq, e_q = scale * (ds @ kh), scale * (off @ kh.abs())
    dk, e_k = fold(scale * (ds.transpose(-1, -2) @ qh)), fold(scale * (off.transpose(-1, -2) @ qh.abs()))
    for o in (out, torch.zeros_like(out), -out):
        got = A.attention_backward(dout, q, k, v, o, lse)
        for x, y, e in ((got[0].transpose(1, 2), dq, e_q), (got[1], dk, e_k)):
            assert bool(((x.double() - y).abs() <= e + U * y.abs() + 1e-30).all()), float(((x.double() - y).abs() / (e + U * y.abs() + 1e-30)).max())
