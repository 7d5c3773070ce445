"""Attention over pages where the sums of weights and the values' sizes are far apart: rows
of zeros, or of the least values, that many keys have, next to large values.  Against the
definition, within the bounds of the other tests (their derivation is there)."""
import math

import pytest
import torch

from paper_2605_30574_gb300 import build as B
from paper_2605_30574_gb300.decoder import pages as P

from page_util import BF, ints, tables
from test_gpu_page_attention import check

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    B.build()


@pytest.mark.parametrize("d,heads,G", [(64, 2, 4), (128, 1, 2), (256, 1, 8), (128, 1, 12)])
@pytest.mark.parametrize("length", [40, 300, 20000])
@pytest.mark.parametrize("at", ["first", "middle", "last"])
@pytest.mark.parametrize("size,bits", [(0, 40), (10, 20), (20, 12), (20, 30), (60, 5), (60, -20), (99, 3), (99, -60), (99, -90)])
def test_zeros_that_outweigh_large_values(d, heads, G, length, at, size, bits):
    """Keys of zeros with values of zeros, and one key whose weight is 2^bits of one of theirs,
    with values of 2^size: as weights go by score and value together, its is up to 2^199 of
    theirs."""
    page = 16
    pages = -(-length // page)
    cache = P.PageCache.empty(1, pages, heads, d, page)
    where = tables([length], [1], page, pages)
    k, v = torch.zeros(length, heads, d), torch.zeros(length, heads, d)
    # (the newest token sees it wherever it is)
    i = {"first": 0, "middle": length // 2, "last": length - 1}[at]
    g = torch.Generator().manual_seed(length + d)
    k[i, :, 0] = 1.75 if bits > 0 else -1.75                            # (7 eighths of 2: exact in the cache)
    v[i] = 2.0 ** size * (0.5 + 0.49 * torch.rand(heads, d, generator=g)) * torch.randn(heads, d, generator=g).sign()
    q = torch.zeros(1, heads * G, d)
    q[..., 0] = 1.0
    scale = abs(bits) * math.log(2) / 1.75
    P.store_pages(cache, 0, k.to(BF).cuda(), v.to(BF).cuda(), where[0], ints(0, length), ints(length))
    check(cache, q.to(BF).cuda(), where, scale=scale)


def test_two_thousand_million_keys_of_the_least_values():
    """A sum of 2^31 weights, each 2^100 and more as weights go by score and value together.
    The most tokens that a sequence has, in one page that comes again and again: all their
    values are 2^-100, and so is the output.  A warp's share of 2^20 keys is added up in 2^16
    steps, in each of which 17 numbers are cut at 2^-23 of the sum: 17 2^-7, below 2^-2, of an
    element that is the upper nibble of a byte.  (The lower one's is a difference of sums that are
    17 and 16 times as large: of that no more is asked than that it is a number.)"""
    page, d = 256, 64
    cache = P.PageCache.empty(1, 1, 1, d, page)
    k, v = torch.zeros(page, 1, d, device="cuda"), torch.full((page, 1, d), 2.0 ** -100, device="cuda")
    k[32:, 0, 0] = 1.75
    P.store_pages(cache, 0, k.to(BF), v.to(BF), ints([0]), ints(0, page), ints(page))
    kk, vv = (torch.empty(page, 1, d, dtype=BF, device="cuda") for _ in range(2))
    P.load_pages(cache, 0, kk, vv, ints([0]), ints(0, page), ints(page))
    q = torch.zeros(1, 1, d, dtype=BF, device="cuda")
    q[..., 0] = 1.0
    table = torch.zeros(1, 1 << 23, dtype=torch.int32, device="cuda")
    # (the first 32 of a page have weights of 2^-7.5 of the others': what a warp begins with may be the lesser)
    got = P.page_attention(cache, 0, q, table, ints(0, 1), ints((1 << 31) - 1), scale=7.5 * math.log(2) / 1.75)
    got, want = got.double(), vv[:1].double()
    assert bool(got.isfinite().all())
    assert bool(((got - want).abs() <= 2.0 ** -2 * want.abs())[..., 1::2].all()), (got.flatten()[:4], want.flatten()[:4])
