"""What logits say of tokens, and how far they are from a teacher's.

``token_logprobs`` scores a row of logits: the log probability of a given
token, the entropy, and the most likely tokens.  ``distill_loss`` is the
divergence of a row's distribution from a teacher's top alternatives (such as
``token_logprobs`` of another run gives), differentiable with respect to the
logits; ``distill_loss_and_grad`` gives loss and gradient in one pass over the
logits where the rows' weights are known beforehand.

Logits are CUDA tensors [..., V] of fp32, bf16 or fp16 whose rows may lie apart
(a slice of a padded vocabulary); tokens of other strides or int32 are copied.
Kernels go to torch's current stream and read and write on the device only; a
bounded wait of a distillation that ran out shows in
``decoder.check_device_error``.  Tracers, which would not record the launches, are
refused.
Sums are in fp32 in a fixed order: the same inputs give the same bits.
"""
from __future__ import annotations

from typing import NamedTuple, Optional, Tuple

import torch

from . import _current_device, _launch, lib, there, untraced

TOP_MAX = 128
_TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}


class TokenScores(NamedTuple):
    """Per row: the token's log probability (None without tokens) and the
    entropy, in nats, and the ``top`` largest log probabilities with their
    tokens, in order (None for ``top`` 0).  fp32 and int64."""
    logprobs: Optional[torch.Tensor]
    entropy: torch.Tensor
    top_logprobs: Optional[torch.Tensor]
    top_ids: Optional[torch.Tensor]


def _rows_of(logits: torch.Tensor, what: str) -> torch.Tensor:
    """The logits as [rows][V], V contiguous, without a copy where they can be."""
    if not isinstance(logits, torch.Tensor) or logits.dtype not in _TYPES:
        raise TypeError(f"{what}: logits must be a tensor of fp32, bf16 or fp16")
    if not logits.is_cuda:
        raise ValueError(f"{what}: logits must be on a CUDA device")
    if logits.dim() == 0 or logits.shape[-1] == 0:
        raise ValueError(f"{what}: logits must be [..., V] with V > 0")
    if logits.is_neg():
        logits = logits.resolve_neg()
    if logits.dim() != 2:
        logits = logits.reshape(-1, logits.shape[-1])
    if logits.stride(1) != 1 and logits.shape[1] > 1:
        logits = logits.contiguous()
    return there(what, "logits", logits)


def _same_device(what: str, logits: torch.Tensor, **others) -> None:
    for name, t in others.items():
        if t is not None and t.device != logits.device:
            raise ValueError(f"{what}: {name} must be on the logits' device")


def _tokens(what: str, name: str, t: torch.Tensor, shape) -> torch.Tensor:
    if not isinstance(t, torch.Tensor) or t.dtype not in (torch.int64, torch.int32):
        raise TypeError(f"{what}: {name} must be a tensor of int64 or int32")
    if t.shape != shape:
        raise ValueError(f"{what}: {name} must have the shape {tuple(shape)}")
    if t.dtype is not torch.int64 or not t.is_contiguous() or t.is_neg():
        t = t.long().resolve_neg().contiguous()
    return there(what, name, t)


def _inverse(what: str, temperature: float) -> float:
    # (finite in fp32: 1 / T, log2(e) / T, and 111 T, from where on below the
    # maximum a weight counts as 2^-160)
    if not 2.0 ** -127 <= temperature <= 2.0 ** 120:
        raise ValueError(f"{what}: the temperature must be positive and finite, between 2^-127 and 2^120")
    return 1.0 / temperature


def token_logprobs(logits: torch.Tensor, tokens: Optional[torch.Tensor] = None, top: int = 0,
                   temperature: float = 1.0) -> TokenScores:
    """Scores rows of logits [..., V] under softmax(logits / temperature):
    log probabilities of ``tokens`` [...] (int64 or int32), entropies, and the
    ``top`` (at most 128) most likely tokens.

    Among equal logits the lowest token comes first.  A token below 0 asks for
    nothing (0 comes back); one past the vocabulary gives NaN.  Tokens with a
    logit of -inf have no probability; where all have, log probabilities are
    -inf and the entropy is 0.  A NaN or +inf among a row's logits makes its
    numbers NaN; NaN comes last in the order of tokens, with -inf.  No gradient
    (``distill_loss`` of one alternative has it)."""
    what = "token_logprobs"
    untraced(what)
    x = _rows_of(logits, what)
    rows, V = x.shape
    lead = logits.shape[:-1]
    if not isinstance(top, int) or top < 0 or top > min(TOP_MAX, V):
        raise ValueError(f"{what}: top must be between 0 and {min(TOP_MAX, V)}")
    inv_T = _inverse(what, temperature)
    if tokens is not None:
        tokens = _tokens(what, "tokens", tokens, lead)
        _same_device(what, x, tokens=tokens)
    if x.device.index != _current_device():
        with torch.cuda.device(x.device):
            return token_logprobs(logits, tokens, top, temperature)
    f32 = dict(dtype=torch.float32, device=x.device)
    logprobs = torch.empty(lead, **f32) if tokens is not None else None
    entropy = torch.empty(lead, **f32)
    best = torch.empty((*lead, top), **f32) if top else None
    ids = torch.empty((*lead, top), dtype=torch.int64, device=x.device) if top else None
    if rows:
        _launch("decoder_token_scores", x.data_ptr(), _TYPES[x.dtype], x.stride(0), rows, V,
                tokens.data_ptr() if tokens is not None else None, top, inv_T,
                logprobs.data_ptr() if tokens is not None else None, entropy.data_ptr(),
                best.data_ptr() if top else None, ids.data_ptr() if top else None)
    return TokenScores(logprobs, entropy, best, ids)


def _distill_args(what, logits, ids, teacher, weight, temperature):
    x = _rows_of(logits, what)
    V, lead = x.shape[1], logits.shape[:-1]
    if V > lib().decoder_distill_vocab(_TYPES[x.dtype]):
        raise ValueError(f"{what}: at most {lib().decoder_distill_vocab(_TYPES[x.dtype])} logits of {x.dtype} to a row")
    if not isinstance(ids, torch.Tensor) or ids.dim() != len(lead) + 1 or not 1 <= ids.shape[-1] <= TOP_MAX:
        raise ValueError(f"{what}: ids must be [..., K] with K between 1 and {TOP_MAX}")
    K = ids.shape[-1]
    ids = _tokens(what, "ids", ids, (*lead, K))
    if not isinstance(teacher, torch.Tensor) or not teacher.is_floating_point():
        raise TypeError(f"{what}: teacher must be a floating tensor")
    if teacher.shape != ids.shape:
        raise ValueError(f"{what}: teacher must have the ids' shape")
    if weight is not None:
        if not isinstance(weight, torch.Tensor) or not weight.is_floating_point():
            raise TypeError(f"{what}: weight must be a floating tensor")
        if weight.shape != lead:
            raise ValueError(f"{what}: weight must have the shape {tuple(lead)}")
    _same_device(what, x, ids=ids, teacher=teacher, weight=weight)
    return x, ids, _f32(what, "teacher", teacher), None if weight is None else _f32(what, "weight", weight), _inverse(what, temperature)


def _f32(what, name, t):
    if t.dtype is not torch.float32 or not t.is_contiguous() or t.is_neg():
        t = t.detach().to(torch.float32).resolve_neg().contiguous()
    return there(what, name, t)


def _distill(x, ids, teacher, weight, rest, inv_T, grad, function=True):
    """Loss [rows] and, if asked for, the gradient [rows][V]."""
    untraced("distillation", function)
    if x.device.index != _current_device():
        with torch.cuda.device(x.device):
            return _distill(x, ids, teacher, weight, rest, inv_T, grad, function)
    rows, V = x.shape
    loss = torch.empty(rows, dtype=torch.float32, device=x.device)
    dx = torch.empty((rows, V), dtype=x.dtype, device=x.device) if grad else None
    if rows:
        _launch("decoder_distill", x.data_ptr(), _TYPES[x.dtype], x.stride(0), rows, V, ids.data_ptr(),
                teacher.data_ptr(), ids.shape[-1], None if weight is None else weight.data_ptr(), 1 if rest else 0, inv_T,
                loss.data_ptr(), dx.data_ptr() if grad else None)
    return loss, dx


class _DistillLoss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, ids, teacher, weight, rest, inv_T):
        ctx.save_for_backward(x, ids, teacher, weight)
        ctx.rest, ctx.inv_T = rest, inv_T
        return _distill(x, ids, teacher, weight, rest, inv_T, False)[0]

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad_loss):
        # (the row's sums again, from the read that the gradient needs anyway)
        x, ids, teacher, weight = ctx.saved_tensors
        w = grad_loss if weight is None else grad_loss * weight
        return (_distill(x, ids, teacher, _f32("distill_loss", "the loss' gradient", w), ctx.rest, ctx.inv_T, True)[1],) + (None,) * 5


def distill_loss(logits: torch.Tensor, ids: torch.Tensor, teacher: torch.Tensor, *,
                 weight: Optional[torch.Tensor] = None, rest: bool = False, temperature: float = 1.0) -> torch.Tensor:
    """Divergence of p = softmax(logits / temperature) [..., V] from a teacher
    known by K alternatives (at most 128): ``ids`` [..., K] and their
    log probabilities ``teacher`` [..., K] at that temperature.  Per row, times
    ``weight`` [...] if given:

    * ``rest`` False: sum_k q_k (log q_k - log p(id_k)), q the teacher's
      probabilities made to sum to 1 over the K (so logits over temperature
      serve as well);
    * ``rest`` True: q as they are, and all other tokens together as one more
      outcome, with what is left of 1: with nothing, where that is no more than
      the rounding of log probabilities that are all there are, 2^-21 sum_k q_k (1
      + |log q_k|).

    An id below 0 is no alternative; a row with none has the loss 0 and no
    gradient, and so has a row of weight 0, whatever else they hold.  An id that comes twice counts
    twice; one past the vocabulary makes its row NaN.  Where the teacher has
    weight on a logit of -inf the loss is +inf, and where it has some on the rest
    and all other logits are -inf; a NaN or +inf among a row's logits makes it NaN.
    Differentiable with respect to the logits; the teacher and the weights get no
    gradient."""
    x, ids, teacher, weight, inv_T = _distill_args("distill_loss", logits, ids, teacher, weight, temperature)
    if weight is not None:
        weight = weight.reshape(-1)
    return _DistillLoss.apply(x, ids, teacher.detach(), None if weight is None else weight.detach(), bool(rest),
                              inv_T).reshape(logits.shape[:-1])


def distill_loss_and_grad(logits: torch.Tensor, ids: torch.Tensor, teacher: torch.Tensor, *,
                          weight: Optional[torch.Tensor] = None, rest: bool = False,
                          temperature: float = 1.0) -> Tuple[torch.Tensor, torch.Tensor]:
    """``distill_loss`` and its sum's gradient with respect to the logits (of
    their type, contiguous), in one pass."""
    x, ids, teacher, weight, inv_T = _distill_args("distill_loss_and_grad", logits, ids, teacher, weight, temperature)
    with torch.no_grad():
        loss, dx = _distill(x, ids, teacher, weight, rest, inv_T, True, False)
    if logits.dim() != 2:
        loss, dx = loss.view(logits.shape[:-1]), dx.view(logits.shape)
    return loss, dx
