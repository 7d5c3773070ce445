"""Attention over pages where q, keys, scale and scores come near the ends of fp32.

The rows look at few keys, so that what is expected is known: of scores that are far apart
the largest takes all, of ones that are equal each the same."""
import pytest
import torch

from paper_2605_30574_gb300 import build as B
from paper_2605_30574_gb300.decoder import pages as P

from page_util import BF, ints, values

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    B.build()


# exponents of q, of keys and of the scale: scores, and scale times q, are below 2^127
SIZES = [(127, -100, -3), (127, -20, -3), (126, 0, -4), (120, 3, -4), (119, 4, 0), (60, 64, -4), (28, 99, -4), (90, 99, -70), (127, -100, 0),
         (-100, 99, 0), (-90, 90, 3), (-126, 99, 100), (10, -30, 60),
         (-130, 90, 40), (-130, 99, 100)]


@pytest.mark.parametrize("eq,ek,es", SIZES)
@pytest.mark.parametrize("d,heads,G,length", [(64, 2, 4, 40), (64, 1, 2, 40), (128, 2, 2, 300), (128, 1, 12, 3000), (256, 1, 8, 100)])
@pytest.mark.parametrize("sign", [1, -1])
def test_scores_near_the_ends(eq, ek, es, d, heads, G, length, sign):
    """q and the keys have one element that is not 0: q's is 2^eq, a key's f 2^ek with f = 4/16
    to 16/16 (as the cache holds it), so that scores are f 2^(eq + ek + es).  No two such f are
    within a sixteenth of each other: scores past 2^15 leave the weight to the largest, and to
    those that equal it."""
    page = 16
    cache = P.PageCache.empty(1, -(-length // page), heads, d, page)
    g = torch.Generator().manual_seed(length)
    f = torch.randint(4, 17, (length, heads, 1), generator=g).float() / 16
    k, v = torch.zeros(length, heads, d), torch.randn(length, heads, d, generator=g).to(BF)
    k[..., 5:6] = f
    k = sign * k * 2.0 ** ek
    q = torch.zeros(1, heads * G, d)
    q[..., 5] = 2.0 ** eq
    table = torch.arange(-(-length // page), dtype=torch.int32)[None].cuda()
    P.store_pages(cache, 0, k.to(BF).cuda(), v.cuda(), table, ints(0, length), ints(length))
    got = P.page_attention(cache, 0, q.to(BF).cuda(), table, ints(0, 1), ints(length), scale=2.0 ** es).cpu().double()
    kk, vv = values(cache, 0).permute(1, 2, 0, 3, 4).flatten(2, 3)[:, :, :length]
    s = kk[..., 5] * 2.0 ** (eq + es)
    # What is off, relatively: a score, which is exact but for the factor that makes it bits and
    # four roundings, 2^-21; weights 2^-10; sums 2^-16; the output 2^-8.  The values' codes add
    # 2^-11 of their scales, a quarter of a row's largest at most; weights below fp16's normal
    # range 2^-28 of the largest.
    assert float(s.abs().max()) < 2.0 ** 127
    e = float(s.abs().max()) * 2.0 ** -21
    if e < 2.0 ** -6:
        p = torch.softmax(s, -1)
    else:
        p = (s == s.amax(-1, keepdim=True)).double()
        p, e = p / p.sum(-1, keepdim=True), 0.0
    want = torch.einsum("hn,hnd->hd", p, vv)
    size = torch.einsum("hn,hnd->hd", p, vv.abs())
    bound = (2.0 ** -8 + 2.0 ** -10 + 2.0 ** -16 + 2 * e) * size + 2.0 ** -13 * torch.einsum("hn,hn->h", p, vv.abs().amax(-1))[:, None] \
        + 2.0 ** -28 * length * vv.abs().max()
    err = (got[0].unflatten(0, (heads, G)) - want[:, None]).abs()
    assert bool((err <= bound[:, None]).all()), float((err / bound[:, None]).max())
