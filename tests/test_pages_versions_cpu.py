"""What is stored and copied makes the cache's tensors other versions, as what is loaded does
to where it goes."""
import pytest
import torch

from paper_2605_30574_gb300.decoder import pages as P

from page_util import BF
from test_pages_cpu import OnCpu, _built, launched, where  # noqa: F401


def versions(cache):
    return [t._version for t in (cache.codes, cache.ratios, cache.exponents)]


def test_the_caches_tensors_are_other_versions(launched):  # noqa: F811
    cache, w = OnCpu(), where()
    k, q = torch.zeros(2, 2, 64, dtype=BF), torch.zeros(2, 4, 64, dtype=BF)
    was = versions(cache)
    P.store_pages(cache, 0, k, k, *w)
    stored = versions(cache)
    assert all(b > a for a, b in zip(was, stored))
    P.copy_pages(cache, [0], [1])
    copied = versions(cache)
    assert all(b > a for a, b in zip(stored, copied))
    # what only reads them, and what does nothing
    P.load_pages(cache, 0, k, torch.zeros_like(k), *w)
    P.page_attention(cache, 0, q, *w)
    P.store_pages(cache, 0, k[:0], k[:0], *w)
    P.copy_pages(cache, [], [])
    assert versions(cache) == copied
    assert len(launched) == 4


def test_a_gradient_that_has_kept_them_is_refused(launched):  # noqa: F811
    cache = OnCpu()
    x = torch.ones(cache.codes.shape, requires_grad=True)
    y = (x * cache.codes).sum()                          # (keeps the codes for x's gradient)
    P.store_pages(cache, 0, *(torch.zeros(2, 2, 64, dtype=BF) for _ in range(2)), *where())
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()


def test_caches_made_for_inference(launched):  # noqa: F811
    """Inference tensors have no versions, and may be written to at any time."""
    with torch.inference_mode():
        cache = OnCpu()
    k = torch.zeros(2, 2, 64, dtype=BF)
    P.store_pages(cache, 0, k, k, *where())
    P.copy_pages(cache, [0], [1])
    with torch.inference_mode():
        P.store_pages(cache, 0, k, k, *where())
        P.copy_pages(OnCpu(), [0], [1])
    assert len(launched) == 4
