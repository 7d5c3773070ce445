"""The paged cache's calls have no gradients, and lose none: tensors that have some, or
tangents, are refused."""
import pytest
import torch
import torch.autograd.forward_ad as fwad

from paper_2605_30574_gb300.decoder import pages as P

from page_util import BF
from test_pages_cpu import OnCpu, _built, launched, where  # noqa: F401


def zeros(heads):
    return torch.zeros(2, heads, 64, dtype=BF)


def calls(cache, k, v, q, out=None):
    w = where()
    return {"store k": lambda: P.store_pages(cache, 0, k, zeros(2), *w), "store v": lambda: P.store_pages(cache, 0, zeros(2), v, *w),
            "load k": lambda: P.load_pages(cache, 0, k, zeros(2), *w), "load v": lambda: P.load_pages(cache, 0, zeros(2), v, *w),
            "q": lambda: P.page_attention(cache, 0, q, *w), "out": lambda: P.page_attention(cache, 0, zeros(4), *w, out=out)}


@pytest.mark.parametrize("which", ["store k", "store v", "load k", "load v", "q", "out"])
def test_gradients_are_not_lost(launched, which):  # noqa: F811
    cache = OnCpu()
    leaf = lambda heads: zeros(heads).requires_grad_()  # noqa: E731
    with pytest.raises(ValueError, match="requires a gradient"):
        calls(cache, leaf(2), leaf(2), leaf(4), leaf(4))[which]()
    # what a leaf makes, and as copies are made of
    some = [(leaf(h) * 2).transpose(0, 1).contiguous().transpose(0, 1) for h in (2, 2, 4)]
    some += [leaf(4) * 2]
    with pytest.raises(ValueError, match="requires a gradient"):
        calls(cache, *some)[which]()
    assert not launched
    with torch.no_grad():
        calls(cache, leaf(2), leaf(2), leaf(4), leaf(4))[which]()
    calls(cache, *(x.detach() for x in some))[which]()
    assert len(launched) == 2


@pytest.mark.parametrize("which", ["store k", "store v", "load k", "load v", "q", "out"])
def test_tangents_are_not_lost(launched, which):  # noqa: F811
    cache = OnCpu()
    with fwad.dual_level():
        dual = lambda heads: fwad.make_dual(zeros(heads), torch.ones(2, heads, 64, dtype=BF))  # noqa: E731
        for mode in (torch.enable_grad, torch.no_grad):
            with mode(), pytest.raises(ValueError, match="tangent"):
                calls(cache, dual(2), dual(2), dual(4), dual(4))[which]()
        assert not launched
        calls(cache, zeros(2), zeros(2), zeros(4), zeros(4))[which]()
    assert len(launched) == 1
