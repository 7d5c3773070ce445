"""Causal attention and its gradients against the definition in fp64.

Tolerances.  P and dS are rounded to bf16 (8 bits: 2^-8 relative each) for their
products, whose sums are in fp32; O, rounded to bf16, goes into delta.  With
u = 2^-8, and |.| element by element, the errors are at most

  dV: u P^T |dO|
  dP - delta: u |dO| . |O| (delta's, for the row)
  dS: u |dS| + P u (|dO| . |O|)
  dK: scale (that)^T |Q|      dQ: scale (that) |K|

plus the output's own rounding, u |value|, and what fp32 leaves: scores of size
s are off by about 2^-20 (1 + s), which moves P by as much, relatively: 2^-16
of the sums of absolute terms covers it (P |dP| + P |delta| for dS).
"""
import math

import pytest
import torch

from paper_2605_30574_gb300 import build as B
from paper_2605_30574_gb300 import decoder as K
from paper_2605_30574_gb300.decoder import attention as A

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
U, FP32 = 2.0 ** -8, 2.0 ** -16
NONE = float("-inf")


@pytest.fixture(scope="module", autouse=True)
def _built():
    B.build()
    yield
    K.check_device_error()


def gen(seed=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def inputs(batch, Tq, Tk, Hq, Hkv, d, seed=0):
    g = gen(seed + 1000 * Tq + Tk)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda").to(BF)  # noqa: E731
    lead = () if batch is None else (batch,)
    return r(*lead, Tq, Hq, d), r(*lead, Hkv, Tk, d), r(*lead, Hkv, Tk, d), r(*lead, Tq, Hq, d)


def definition(q, k, v, dout, scale):
    """fp64 output, log sums and gradients, with the bounds of their errors."""
    q, k, v, go = (t.double() if t.dim() == 4 else t.double()[None] for t in (q, k, v, dout))
    G = q.shape[2] // k.shape[1]
    qh, gh = q.transpose(1, 2), go.transpose(1, 2)
    kh, vh = k.repeat_interleave(G, 1), v.repeat_interleave(G, 1)
    Tq, Tk = q.shape[1], k.shape[2]
    seen = torch.arange(Tk, device="cuda")[None] <= torch.arange(Tq, device="cuda")[:, None] + (Tk - Tq)
    s = (scale * (qh @ kh.transpose(-1, -2))).masked_fill(~seen, NONE)
    lse = torch.logsumexp(s, -1)
    p = torch.where(seen, (s - torch.where(lse == NONE, torch.zeros_like(lse), lse)[..., None]).exp(), torch.zeros_like(s))
    o = p @ vh
    dp = gh @ vh.transpose(-1, -2)
    delta = (gh * o).sum(-1, keepdim=True)
    ds = p * (dp - delta)
    fold = lambda x: x.unflatten(1, (k.shape[1], G)).sum(2)  # noqa: E731
    back = lambda x: x.transpose(1, 2)  # noqa: E731
    e_ds = U * ds.abs() + p * (U * (gh.abs() * o.abs()).sum(-1, keepdim=True)) \
        + FP32 * p * (dp.abs() + delta.abs() + gh.abs() @ vh.abs().transpose(-1, -2))
    a = abs(scale)
    got = dict(out=back(o), lse=lse, dq=back(scale * (ds @ kh)), dk=fold(scale * (ds.transpose(-1, -2) @ qh)),
               dv=fold(p.transpose(-1, -2) @ gh))
    off = dict(out=back((U + FP32) * (p @ vh.abs())), lse=2.0 ** -18 * (1 + lse.abs().masked_fill(lse == NONE, 0)),
               dq=back(a * (e_ds @ kh.abs())), dk=fold(a * (e_ds.transpose(-1, -2) @ qh.abs())),
               dv=fold((U + FP32) * (p.transpose(-1, -2) @ gh.abs())))
    for n in ("out", "dq", "dk", "dv"):
        off[n] = off[n] + U * got[n].abs() + 1e-30
    return got, off


def near(name, got, want, off):
    got = got.double().reshape(want.shape)
    same = got == want
    bad = ((got - want).abs() / off).masked_fill(same, 0.0)
    assert bool(got.isfinite().logical_or(same).all()), name
    assert float(bad.max()) <= 1.0, (name, float(bad.max()))


def check(q, k, v, dout, scale=None):
    want, off = definition(q, k, v, dout, 1.0 / math.sqrt(q.shape[-1]) if scale is None else scale)
    out, lse = A.attention_forward(q, k, v, scale)
    assert out.shape == q.shape and out.dtype is BF
    near("out", out, want["out"], off["out"])
    near("lse", lse, want["lse"], off["lse"])
    grads = A.attention_backward(dout, q, k, v, out, lse, scale)
    for n, t, like in zip(("dq", "dk", "dv"), grads, (q, k, v)):
        assert t.shape == like.shape and t.dtype is BF and t.is_contiguous()
        near(n, t, want[n], off[n])
    return out, lse, grads


SHAPES = [
    # batch, Tq, Tk, Hq, Hkv: one token of one key; of several; either side of a
    # block and of a tile; a group of heads; odd ones; a long span; a batch
    (None, 1, 1, 2, 1), (None, 1, 37, 4, 2), (1, 1, 700, 8, 2), (None, 63, 63, 2, 2), (None, 64, 64, 1, 1),
    (None, 65, 65, 2, 1), (None, 127, 129, 2, 2), (2, 128, 128, 4, 1), (3, 129, 129, 2, 1), (None, 200, 333, 6, 2),
    (2, 16, 144, 8, 2), (None, 257, 1000, 7, 1), (None, 777, 777, 4, 2), (2, 100, 2148, 4, 2), (None, 1500, 1500, 8, 1),
    # rows that see nothing: some, those of whole tiles, all but one
    (None, 70, 50, 2, 1), (2, 300, 100, 4, 2), (None, 513, 1, 2, 2),
]


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("batch,Tq,Tk,Hq,Hkv", SHAPES)
def test_gradients(batch, Tq, Tk, Hq, Hkv, d):
    q, k, v, dout = inputs(batch, Tq, Tk, Hq, Hkv, d)
    out, lse, (dq, dk, dv) = check(q, k, v, dout)
    if Tq > Tk:
        rows = Tq - Tk
        assert not out[..., :rows, :, :].any() and not dq[..., :rows, :, :].any()
        assert bool((lse[..., :rows] == NONE).all())
    # a row of one key: its weight is 1 whatever the scores are
    first = Tq - Tk
    if first >= 0:
        assert not dq[..., first, :, :].any()
    if Tk == 1:
        assert not dk.any() and not dq.any()


@pytest.mark.parametrize("scale", [0.0, -0.3, 1.0])
def test_scales(scale):
    check(*inputs(None, 150, 180, 4, 2, 64, seed=3), scale=scale)


@pytest.mark.parametrize("Tq,Tk,Hq,Hkv,d", [(1024, 1024, 8, 2, 128), (96, 3000, 16, 2, 128), (640, 640, 4, 4, 64), (300, 1300, 4, 1, 256)])
def test_same_bits(Tq, Tk, Hq, Hkv, d):
    q, k, v, dout = inputs(1, Tq, Tk, Hq, Hkv, d)
    out, lse = A.attention_forward(q, k, v)
    a, b = (A.attention_backward(dout, q, k, v, out, lse) for _ in range(2))
    assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_forward_is_the_prefills():
    q, k, v, _ = inputs(None, 300, 300, 8, 2, 128)
    out, _ = A.attention_forward(q, k, v, 0.09)
    want, off = definition(q, k, v, q, 0.09)
    near("causal", K.causal(q, k, v, 0.09), want["out"], off["out"])
    near("out", out, want["out"], off["out"])


def test_strides():
    q, k, v, dout = inputs(2, 150, 170, 4, 2, 64, seed=5)
    want = check(q, k, v, dout)
    flip = lambda t: t.transpose(-2, -3).contiguous().transpose(-2, -3)  # noqa: E731
    pad = lambda t: torch.cat([t, t], -1)[..., :t.shape[-1]]  # noqa: E731
    odd = lambda t: torch.cat([t, t[..., :1]], -1)[..., :-1]  # noqa: E731
    off = lambda t: torch.cat([t.flatten()[:1], t.flatten()])[1:].view(t.shape)  # noqa: E731
    last = lambda t: t.transpose(-1, -2).contiguous().transpose(-1, -2)  # noqa: E731
    for f in (flip, pad, odd, off, last):
        got = check(f(q), f(k), f(v), f(dout))
        assert torch.equal(got[0], want[0]) and all(torch.equal(a, b) for a, b in zip(got[2], want[2]))
    # one prompt's keys for a batch of continuations
    k1, v1 = k[:1].expand(2, -1, -1, -1), v[:1].expand(2, -1, -1, -1)
    check(q, k1, v1, dout)


def test_autograd():
    q, k, v, dout = inputs(None, 90, 300, 6, 3, 128, seed=6)
    out, lse = A.attention_forward(q, k, v)
    want = A.attention_backward(dout, q, k, v, out, lse)
    leaves = [t.clone().requires_grad_() for t in (q, k, v)]
    y = A.attention(*leaves)
    assert torch.equal(y.detach(), out)
    got = torch.autograd.grad(y, leaves, dout)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    # a gradient that is the same for every element comes as a view without strides
    A.attention(*leaves).float().sum().backward()
    ones = A.attention_backward(torch.ones_like(q), q, k, v, out, lse)
    assert all(torch.equal(t.grad, b) for t, b in zip(leaves, ones))
    # a span shared by a batch: its gradient is the batch's sum
    q4 = torch.stack([q, q.flip(0)])
    kl, vl = k.clone().requires_grad_(), v.clone().requires_grad_()
    y = A.attention(q4, kl.expand(2, -1, -1, -1), vl.expand(2, -1, -1, -1))
    y.backward(torch.stack([dout, dout]))
    each = [A.attention_backward(dout, x, k, v, *A.attention_forward(x, k, v)) for x in q4]
    assert torch.allclose(kl.grad.float(), (each[0][1].float() + each[1][1].float()), rtol=2 ** -7, atol=1e-3)


def test_by_differences():
    """The kernels' gradients against differences of the fp64 definition."""
    q, k, v, dout = inputs(None, 40, 70, 2, 1, 64, seed=7)
    scale = 0.125
    out, lse = A.attention_forward(q, k, v, scale)
    grads = A.attention_backward(dout, q, k, v, out, lse, scale)
    _, off = definition(q, k, v, dout, scale)
    h = 1e-5
    for i, (t, g, n) in enumerate(zip((q, k, v), grads, ("dq", "dk", "dv"))):
        by = torch.randn(t.shape, generator=gen(i), device="cuda", dtype=torch.double)
        loss = []
        for s in (h, -h):
            moved = [x.double() for x in (q, k, v)]
            moved[i] = moved[i] + s * by
            loss.append((definition(*moved, dout, scale)[0]["out"] * dout.double()).sum())
        slope = (loss[0] - loss[1]) / (2 * h)
        bound = (off[n].reshape(t.shape) * by.abs()).sum()
        assert float((slope - (g.double() * by).sum()).abs()) <= float(bound) + 1e-4


def test_inputs_that_are_not_finite():
    """A key's infinity or NaN stays with the rows that see it or share a tile
    with those that do."""
    q, k, v, dout = inputs(None, 400, 400, 2, 1, 64, seed=8)
    k[0, 390, 3] = float("nan")
    out, lse = A.attention_forward(q, k, v)
    dq, dk, dv = A.attention_backward(dout, q, k, v, out, lse)
    assert bool(lse[:, 390:].isnan().all()) and bool(lse[:, :390].isfinite().all())
    assert bool(out[:256].isfinite().all()) and bool(dq[:256].isfinite().all())
    assert bool(dq[390:].isnan().any(-1).all()) and bool(dk[0, 390].isnan().any())


def test_streams_and_graph():
    q, k, v, dout = inputs(None, 256, 512, 4, 1, 128, seed=9)
    want = check(q, k, v, dout)[2]
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            for _ in range(3):
                out, lse = A.attention_forward(q, k, v)
                got.append(A.attention_backward(dout, q, k, v, out, lse))
    for s in streams:
        torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, lse = A.attention_forward(q, k, v)
        got.append(A.attention_backward(dout, q, k, v, out, lse))
    graph.replay()
    for g in got:
        assert all(torch.equal(a, b) for a, b in zip(g, want))


def test_lengths_of_zero():
    q, k, v, dout = inputs(2, 3, 5, 4, 2, 64)
    out, lse = A.attention_forward(q, k[:, :, :0], v[:, :, :0])
    assert not out.any() and bool((lse == NONE).all())
    dq, dk, dv = A.attention_backward(dout, q, k[:, :, :0], v[:, :, :0], out, lse)
    assert not dq.any() and dk.shape == dv.shape == (2, 2, 0, 64)
    out, lse = A.attention_forward(q[:, :0], k, v)
    dq, dk, dv = A.attention_backward(dout[:, :0], q[:, :0], k, v, out, lse)
    assert out.shape == (2, 0, 4, 64) and not dk.any() and not dv.any()
    assert A.attention_forward(q[:0], k[:0], v[:0])[0].shape == (0, 3, 4, 64)


def test_refusals():
    q, k, v, dout = inputs(None, 4, 6, 4, 2, 64)
    out, lse = A.attention_forward(q, k, v)
    for error, call in [
            (TypeError, lambda: A.attention(q.float(), k, v)),
            (TypeError, lambda: A.attention(q, k.half(), v)),
            (ValueError, lambda: A.attention(q.cpu(), k.cpu(), v.cpu())),
            (ValueError, lambda: A.attention(q, k.cpu(), v)),
            (ValueError, lambda: A.attention(q, k, v[:, :5])),
            (ValueError, lambda: A.attention(q[:, :3], k, v)),
            (ValueError, lambda: A.attention(q[None], k, v)),
            (ValueError, lambda: A.attention(q[..., :32], k[..., :32], v[..., :32])),
            (ValueError, lambda: A.attention(q[None], k.expand(2, -1, -1, -1), v.expand(2, -1, -1, -1))),
            (ValueError, lambda: A.attention(q, k[:0], v[:0])),
            (TypeError, lambda: A.attention_backward(dout.float(), q, k, v, out, lse)),
            (ValueError, lambda: A.attention_backward(dout[:3], q, k, v, out, lse)),
            (ValueError, lambda: A.attention_backward(dout, q, k, v, out[:3], lse)),
            (TypeError, lambda: A.attention_backward(dout, q, k, v, out, lse.double())),
            (ValueError, lambda: A.attention_backward(dout, q, k, v, out, lse[:1]))]:
        with pytest.raises(error):
            call()
    assert K.lib().decoder_attention_scratch(2, 130, 4) == 2 * 4 * 256 * 40
    # a shape past the kernels' index range comes back as an error
    big = torch.empty(1, 1, 64, dtype=BF, device="cuda").expand((1 << 20) + 1, 1, 64)
    with pytest.raises(RuntimeError):
        K._launch("decoder_attention", big.data_ptr(), k.data_ptr(), v.data_ptr(), (__import__("ctypes").c_long * 9)(*[64] * 9), out.data_ptr(),
                  lse.data_ptr(), 1, big.shape[0], 6, 1, 1, 64, 1.0)
