"""Causal attention with its gradients, for one sequence or a batch.

``attention`` is differentiable; ``attention_forward`` and
``attention_backward`` are its halves for callers without autograd.  The
queries are the last Tq positions of the Tk that keys and values cover: a whole
prompt (Tq = Tk), a continuation of a cached span (Tq < Tk), one token
(Tq = 1).  With Tq above Tk the first Tq - Tk rows see no key: their outputs
and gradients are 0.

q is [Tq, Hq, d] and k, v are [Hkv, Tk, d] (as the decoder's stores lay a layer
out), or all with a batch in front; bf16, d 64, 128 or 256, Hq a multiple of
Hkv, any strides (those that the kernels cannot read are copied); lengths, and
batch times heads, of up to 2^20.  Scores, sums
and gradients are accumulated in fp32; probabilities and the gradients of scores
are rounded to bf16 for their products.  The same inputs give the same bits.

Kernels go to torch's current stream; a bounded wait that ran out shows in
``decoder.check_device_error``.  Tracers, which would not record them, are refused.
"""
from __future__ import annotations

import ctypes
import math
from typing import Optional, Tuple

import torch

from . import BF16, F32, _current_device, _launch, lib, there, untraced


def _fits(q, k, v):
    """Whether the arguments are as they have to be."""
    try:
        (Hq, d), (Hkv, _, dk), device = q.shape[-2:], k.shape[-3:], q.device
        return (q.dtype is k.dtype is v.dtype is BF16 and device.type == "cuda" and device == k.device == v.device
                and k.shape == v.shape and q.dim() == k.dim() and (q.dim() == 3 or q.dim() == 4 and q.shape[0] == k.shape[0])
                and d == dk and d in (64, 128, 256) and Hkv > 0 and Hq > 0 and Hq % Hkv == 0)
    except (AttributeError, ValueError):
        return False


def _check(what, q, k, v):
    if _fits(q, k, v):
        return
    for name, t in (("q", q), ("k", k), ("v", v)):
        if not isinstance(t, torch.Tensor) or t.dtype is not BF16:
            raise TypeError(f"{what}: {name} must be a bf16 tensor")
        if t.device.type != "cuda" or t.device != q.device:
            raise ValueError(f"{what}: q, k and v must be on one CUDA device")
    if q.dim() not in (3, 4) or k.dim() != q.dim() or k.shape != v.shape:
        raise ValueError(f"{what}: q must be [Tq, Hq, d] and k, v [Hkv, Tk, d], or all with a batch in front")
    if k.shape[-1] != q.shape[-1] or q.shape[-1] not in (64, 128, 256) or (q.dim() == 4 and k.shape[0] != q.shape[0]):
        raise ValueError(f"{what}: heads of 64, 128 or 256, the same for q, k and v, and one batch")
    raise ValueError(f"{what}: the query heads must be a multiple of the kv heads")


_STRIDES = {n: ctypes.c_long * n for n in (9, 15)}


def _readable(t, heads_first):
    """A copy of the tensor that the kernels can read, or the tensor, and its
    (row, head, batch) strides."""
    def strides(t):
        s = t.stride()
        return (s[-2], s[-3], s[0]) if heads_first else (s[-3], s[-2], s[0])

    sizes = (t.shape[-2], t.shape[-3]) if heads_first else (t.shape[-3], t.shape[-2])
    sizes += (t.shape[0] if t.dim() == 4 else 1,)
    st = strides(t)
    if t.stride(-1) != 1 or t.data_ptr() & 15 or t.is_neg() \
            or any(n > 1 and (s <= 0 or s & 7 or s >= 1 << 38) for n, s in zip(sizes, st)):
        t = t.resolve_neg().clone(memory_format=torch.contiguous_format)
        st = strides(t)
    return t, st


def _operands(*ts):
    """The tensors as the kernels can read them (the last two, k and v, have
    their heads first), their addresses, and their strides as a C array (None:
    all contiguous)."""
    ptrs, low, plain = [], 0, True
    for t in ts:
        p = t.data_ptr()
        if not p:
            raise ValueError("attention: an operand has no memory")
        ptrs.append(p)
        if t.is_neg():
            low = 1
        low |= p
        plain = plain and t.is_contiguous()
    if not low & 15:
        if plain:
            return ts, ptrs, None
        flat, last = [], len(ts) - 2
        for i, t in enumerate(ts):
            s = t.stride()
            b, (x, y, one) = s[0], s[-3:]
            if one != 1 or (b | x | y) & 7 or not 0 < min(s) or max(s) >= 1 << 38:
                break
            flat += (y, x, b) if i >= last else (x, y, b)
        else:
            return ts, ptrs, _STRIDES[len(flat)](*flat)
    got = [_readable(t, i >= len(ts) - 2) for i, t in enumerate(ts)]
    return [t for t, _ in got], [t.data_ptr() for t, _ in got], _STRIDES[3 * len(ts)](*[s for _, st in got for s in st])


def _scale(scale, d):
    return 1.0 / math.sqrt(d) if scale is None else float(scale)


def attention_forward(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                      scale: Optional[float] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Attention's output, like q and contiguous, and the rows' log sums of
    e^(scale q . k), fp32 [Hq, Tq] ([B, Hq, Tq]); -inf for a row that sees no
    key.  ``scale`` is 1 / sqrt(d) by default."""
    return _forward(q, k, v, scale, False)


def _forward(q, k, v, scale, function):
    untraced("attention_forward", function)
    _check("attention_forward", q, k, v)
    device = q.device
    if device.index != _current_device():
        with torch.cuda.device(device):
            return _forward(q, k, v, scale, function)
    *B, Tq, Hq, d = q.shape
    Hkv, Tk, _ = k.shape[-3:]
    out = torch.empty(q.shape, dtype=BF16, device=device)
    lse = torch.empty((*B, Hq, Tq), dtype=F32, device=device)
    B = B[0] if B else 1
    if B * Tq * Tk == 0:
        return out.zero_(), lse.fill_(-math.inf)
    ts, ptrs, strides = _operands(q, k, v)      # (ts: copies live until the launch)
    _launch("decoder_attention", *ptrs, strides, out.data_ptr(), lse.data_ptr(), B, Tq, Tk, Hq, Hkv, d, _scale(scale, d))
    return out, lse


def attention_backward(dout: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor,
                       lse: torch.Tensor, scale: Optional[float] = None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """Gradients with respect to q, k and v (bf16, contiguous), given the
    output's, and output and log sums as ``attention_forward`` gave them."""
    what = "attention_backward"
    untraced(what)
    _check(what, q, k, v)
    shape, device = q.shape, q.device
    *B, Tq, Hq, d = shape
    for name, t in (("dout", dout), ("out", out)):
        if not isinstance(t, torch.Tensor) or t.dtype is not BF16:
            raise TypeError(f"{what}: {name} must be a bf16 tensor")
        if t.shape != shape or t.device != device:
            raise ValueError(f"{what}: {name} must be like q")
    if not isinstance(lse, torch.Tensor) or lse.dtype is not F32:
        raise TypeError(f"{what}: lse must be an fp32 tensor")
    if lse.shape != (*B, Hq, Tq) or lse.device != device:
        raise ValueError(f"{what}: lse must be [Hq, Tq], or [B, Hq, Tq]")
    if device.index != _current_device():
        with torch.cuda.device(device):
            return attention_backward(dout, q, k, v, out, lse, scale)
    B, (Hkv, Tk, _) = B[0] if B else 1, k.shape[-3:]
    if B * Tq * Tk == 0:
        return torch.zeros(shape, dtype=BF16, device=device), torch.zeros(k.shape, dtype=BF16, device=device), \
            torch.zeros(k.shape, dtype=BF16, device=device)
    ts, ptrs, strides = _operands(dout, q, out, k, v)      # (ts: copies live until the launch)
    if not lse.is_contiguous() or lse.is_neg():
        lse = lse.resolve_neg().contiguous()
    there(what, "lse", lse)
    dq = torch.empty(shape, dtype=BF16, device=device)
    dk = torch.empty(k.shape, dtype=BF16, device=device)
    dv = torch.empty(k.shape, dtype=BF16, device=device)
    scratch = torch.empty(lib().decoder_attention_scratch(B, Tq, Hq), dtype=torch.uint8, device=device)
    _launch("decoder_attention_backward", *ptrs, lse.data_ptr(), strides, scratch.data_ptr(), dq.data_ptr(), dk.data_ptr(),
            dv.data_ptr(), B, Tq, Tk, Hq, Hkv, d, _scale(scale, d))
    return dq, dk, dv


class _Attention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, scale):
        out, lse = _forward(q, k, v, scale, True)
        ctx.save_for_backward(q, k, v, out, lse)
        ctx.scale = scale
        return out

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dout):
        q, k, v, out, lse = ctx.saved_tensors
        return (*attention_backward(dout, q, k, v, out, lse, ctx.scale), None)


def attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, scale: Optional[float] = None) -> torch.Tensor:
    """Causal attention of q over k and v, differentiable with respect to all
    three; see the module for the layouts."""
    return _Attention.apply(q, k, v, scale)
