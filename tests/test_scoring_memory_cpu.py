"""Tensors without memory (torch's zeros that have none, storage given back) are
refused before a kernel could read address 0; negated views are read as such."""
import pytest
import torch

from paper_2605_30574_gb300.decoder import attention as A
from paper_2605_30574_gb300.decoder import scoring

BF = torch.bfloat16


def zeros(*shape, dtype):
    return torch._efficientzerotensor(shape, dtype=dtype)


def freed(*shape, dtype):
    t = torch.zeros(shape, dtype=dtype)
    t.untyped_storage().resize_(0)
    return t


@pytest.mark.parametrize("nothing", [zeros, freed])
def test_operands_without_memory(nothing):
    q, k = torch.zeros(3, 4, 64, dtype=BF), torch.zeros(2, 5, 64, dtype=BF)
    no_q, no_k = nothing(3, 4, 64, dtype=BF), nothing(2, 5, 64, dtype=BF)
    for ts in ((no_q, k, k), (q, no_k, k), (q, k, no_k), (no_q, q, q, k, k), (q, no_q, q, k, k), (q, q, no_q, k, k)):
        with pytest.raises(ValueError, match="no memory"):
            A._operands(*ts)
    with pytest.raises(ValueError, match="tokens has no memory"):
        scoring._tokens("a call", "tokens", nothing(4, dtype=torch.int64), (4,))
    with pytest.raises(ValueError, match="teacher has no memory"):
        scoring._f32("a call", "teacher", nothing(4, 3, dtype=torch.float32))
    # (none is needed)
    empty = torch.zeros(0, dtype=torch.int64)
    assert scoring._tokens("a call", "tokens", empty, (0,)).shape == (0,)


@pytest.mark.parametrize("dtype", [torch.int64, torch.int32])
def test_tokens_that_are_a_negated_view(dtype):
    t = torch._neg_view(torch.tensor([1, -2, 3], dtype=dtype))
    got = scoring._tokens("a call", "tokens", t, (3,))
    assert not got.is_neg() and got.is_contiguous() and got.tolist() == [-1, 2, -3]
