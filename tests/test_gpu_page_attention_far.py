"""Attention over pages where scores are large and the values' sizes far apart: a score that
is past 2^24 has no bits left for a size beside it.

Scores are such that what is expected is known, as in the tests of the ends of fp32."""

import pytest
import torch

from paper_2605_30574_gb300 import build as B
from paper_2605_30574_gb300.decoder import pages as P

from page_util import BF, ints, values

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    B.build()


@pytest.mark.parametrize("bits", [10, 16, 20, 23, 25, 28, 35, 60, 120])
@pytest.mark.parametrize("least,most", [(-90, -90), (-35, -35), (30, 30), (90, 90), (-90, 90), (0, 20)])
@pytest.mark.parametrize("d,heads,G,length,new", [(64, 2, 4, 40, 1), (64, 1, 2, 40, 3), (128, 2, 2, 300, 1), (128, 1, 12, 3000, 2), (256, 1, 8, 100, 1),
                                                  (128, 8, 4, 200, 1), (64, 1, 1, 40000, 1)])
@pytest.mark.parametrize("sign", [1, -1])
def test_large_scores_and_sizes_far_apart(bits, least, most, d, heads, G, length, new, sign):
    """Keys have one element, f 2^(bits / 2) with f = 4/16 to 16/16 as the cache holds it, q one of
    2^(bits / 2) times 1 or -1, by the head: scores are f 2^bits.  No two such f are within a
    sixteenth of each other, so that from 2^15 on the largest, and what equals it, takes all."""
    page = 16
    cache = P.PageCache.empty(1, -(-length // page), heads, d, page)
    g = torch.Generator().manual_seed(length)
    f = torch.randint(4, 17, (length, heads, 1), generator=g).float() / 16
    f[:new] = 5 / 16
    k, v = torch.zeros(length, heads, d), torch.randn(length, heads, d, generator=g)
    k[..., 5:6] = sign * f * 2.0 ** (bits // 2)
    v = v * 2.0 ** torch.randint(least, most + 1, (length, heads, 1), generator=g).double()
    q = torch.zeros(new, heads * G, d)
    q[..., 5] = 2.0 ** (bits - bits // 2) * torch.tensor([1.0, -1.0]).repeat(heads * G)[:heads * G]
    table = torch.arange(-(-length // page), dtype=torch.int32)[None].cuda()
    P.store_pages(cache, 0, k.to(BF).cuda(), v.to(BF).cuda(), table, ints(0, length), ints(length))
    got = P.page_attention(cache, 0, q.to(BF).cuda(), table, ints(0, new), ints(length), scale=1.0).cpu().double()
    kk, vv = values(cache, 0).permute(1, 2, 0, 3, 4).flatten(2, 3)[:, :, :length]
    for i in range(new):
        keys, vals = (x[:, :length - new + 1 + i].repeat_interleave(G, 0) for x in (kk, vv))
        s = (keys @ q[i].double()[:, :, None])[..., 0]
        # what is off: see the tests of the ends of fp32
        e = float(s.abs().max()) * 2.0 ** -21
        if e < 2.0 ** -6:
            p = torch.softmax(s, -1)
        else:
            p = (s == s.amax(-1, keepdim=True)).double()
            p, e = p / p.sum(-1, keepdim=True), 0.0
        want = torch.einsum("hn,hnd->hd", p, vals)
        pv = p[..., None] * vals.abs()
        bound = (2.0 ** -8 + 2.0 ** -10 + 2.0 ** -16 + 2 * e) * pv.sum(1) + 2.0 ** -13 * pv.amax(-1).sum(-1)[:, None] \
            + 2.0 ** -28 * length * pv.amax((1, 2))[:, None]
        err = (got[i] - want).abs()
        assert bool((err <= bound).all()), (i, float((err / bound).max()))


def test_scores_that_become_large():
    """A row whose first keys have small scores and whose last have large ones, and the other
    way round; values' sizes by turns."""
    page, d, n = 16, 64, 4000
    cache = P.PageCache.empty(1, n // page, 1, d, page)
    k, v = torch.zeros(n, 1, d), torch.randn(n, 1, d, generator=torch.Generator().manual_seed(3))
    size = torch.arange(n) % 7
    v *= (2.0 ** (30.0 * size - 90))[:, None, None]
    for order in (1, -1):
        at = torch.arange(n)[::order] if order == 1 else torch.arange(n - 1, -1, -1)
        k[at, 0, 0] = torch.where(torch.arange(n) < n // 2, torch.zeros(n), 2.0 ** (torch.arange(n) // (n // 50)).clamp(min=25).double() - 20).float()
        table = torch.arange(n // page, dtype=torch.int32)[None].cuda()
        P.store_pages(cache, 0, k.to(BF).cuda(), v.to(BF).cuda(), table, ints(0, n), ints(n))
        q = torch.zeros(1, 2, d)
        q[..., 0] = torch.tensor([2.0 ** 8, -2.0 ** 8])
        got = P.page_attention(cache, 0, q.to(BF).cuda(), table, ints(0, 1), ints(n), scale=1.0).cpu().double()
        kk, vv = values(cache, 0).permute(1, 2, 0, 3, 4).flatten(2, 3)[:, 0, :n]
        for h in (0, 1):
            s = kk[:, 0] * float(q[0, h, 0])
            p = (s == s.max()).double()
            p /= p.sum()
            pv = p[:, None] * vv.abs()
            bound = (2.0 ** -8 + 2.0 ** -10 + 2.0 ** -16) * pv.sum(0) + 2.0 ** -13 * pv.amax(-1).sum() + 2.0 ** -28 * n * pv.max()
            err = (got[0, h] - p @ vv).abs()
            assert bool((err <= bound).all()), (order, h, float((err / bound).max()))
