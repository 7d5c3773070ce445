"""Rows into the pages of a 4-bit cache and out of them, and pages copied: all exact.

What a row is held as is decided in 32 bits without error: a quotient of an 8-bit by a
4-bit number that is halfway between two codes is found as such, any other is 2^-10
away, and a value has seven bits, which bf16 holds."""
import pytest
import torch

from paper_2605_30574_gb300 import build as B
from paper_2605_30574_gb300.decoder import pages as P

from page_util import BF, held, ints, tables, values

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    B.build()


def rows(n, heads, d, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(2, n, heads, d, generator=g, device="cuda") * torch.exp(torch.randn(2, n, heads, d // 32, 1, generator=g, device="cuda")).expand(
        2, n, heads, d // 32, 32).flatten(-2)
    return x.to(BF).unbind(0)


def expected(x):
    # (on the CPU, whose powers of two are exact)
    return held(x.cpu())[0].to(BF).to(x.device)


def same(a, b):
    return torch.equal(a.isnan(), b.isnan()) and torch.equal(a.nan_to_num(9.0), b.nan_to_num(9.0))


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("heads,page", [(1, 16), (3, 32), (8, 64), (2, 256), (17, 16), (5, 32)])
@pytest.mark.parametrize("new,old", [([1], [0]), ([1] * 9, [0, 15, 16, 17, 63, 64, 300, 1, 2]),
                                     ([5, 0, 100, 33, 1, 0], [3, 9, 0, 31, 64, 0])])
def test_rows_come_back_as_they_are_held(d, heads, page, new, old):
    lengths = [a + b for a, b in zip(new, old)]
    pages = sum(-(-n // page) for n in lengths) + 3
    cache = P.PageCache.empty(2, pages, heads, d, page)
    for t in (cache.codes, cache.ratios, cache.exponents):
        t.random_(0, 255)
    before = [t.clone() for t in (cache.codes, cache.ratios, cache.exponents)]
    table, starts, n = tables(lengths, new, page, pages, seed=d + page)
    k, v = rows(sum(new), heads, d, seed=1)
    P.store_pages(cache, 1, k, v, table, starts, n)
    to = [torch.full_like(k, 3.0) for _ in range(2)]
    P.load_pages(cache, 1, *to, table, starts, n)
    for x, y in zip((k, v), to):
        assert same(y, expected(x))
    # by place, and nothing else was written
    written = torch.zeros((pages, page), dtype=torch.bool)
    at, got = 0, values(cache, 1)
    for b, (m, L) in enumerate(zip(new, lengths)):
        for i in range(m):
            pos = L - m + i
            p, s = int(table[b, pos // page]), pos % page
            written[p, s] = True
            for kv, x in enumerate((k, v)):
                assert same(got[p, kv, :, s], held(x[at].cpu())[0])
            at += 1
    for t, was in zip((cache.codes, cache.ratios, cache.exponents), before):
        assert torch.equal(t[0], was[0])
        keep = ~written.cuda()
        now, was = (x[1].movedim(-2, 1) for x in (t, was))
        assert torch.equal(now[keep], was[keep])


@pytest.mark.parametrize("d", [64, 128, 256])
def test_every_row_size_and_every_tie(d):
    g = torch.Generator().manual_seed(d)
    n = 4096
    x = torch.randn(n, 1, d, generator=g) * 2.0 ** torch.randint(-132, 127, (n, 1, 1), generator=g).double()
    x = (x * 2.0 ** (-20 * torch.rand(n, 1, d, generator=g).double())).to(BF)
    # halfway between codes, and scales halfway between two of four bits
    x[:2000] = (torch.randint(-255, 256, (2000, 1, d), generator=g) / 16).to(BF)
    x[2000:2100] = 119.0 / 64
    x[2100] = 0
    x[2101] = -0.0
    x[2102, 0, 5] = float("inf")
    x[2103, 0, 7] = float("-inf")
    x[2104, 0, 9] = float("nan")
    x[2105, 0, 3] = 2.0 ** 100
    x[2106] = 2.0 ** -100
    x[2107] = 2.0 ** -101
    x[2108] = torch.finfo(BF).smallest_normal / 64
    x[2109, 0, :32] = 0
    x[2110] = 2.0 ** -30
    x[2110, 0, 40] = 2.0 ** 99
    x = x.cuda()
    cache = P.PageCache.empty(1, n // 16, 1, d, 16)
    table, starts, lengths = tables([n], [n], 16, n // 16)
    P.store_pages(cache, 0, x, x.flip(0), table, starts, lengths)
    k, v = torch.empty_like(x), torch.empty_like(x)
    P.load_pages(cache, 0, k, v, table, starts, lengths)
    assert same(k, expected(x)) and same(v, expected(x.flip(0)))
    # (off by half a scale at most, where the scale is not the least that a row has)
    want, s = held(x.cpu())
    worst = (want - x.cpu().double()).abs().unflatten(-1, (-1, 32)).amax(-1)
    assert bool((worst <= s / 2)[:2000].all())


@pytest.mark.parametrize("how", ["joined", "transposed", "unaligned", "negated", "reversed heads"])
def test_strides(how):
    d, heads, n = 128, 4, 37
    k, v = rows(n, heads, d, 5)
    if how == "joined":
        y = torch.cat([k, v], 1)
        k, v = y[:, :heads], y[:, heads:]
    elif how == "transposed":
        k, v = (x.transpose(0, 1).contiguous().transpose(0, 1) for x in (k, v))
    elif how == "unaligned":
        k, v = (torch.cat([x, x], -1)[..., 1:d + 1] for x in (k, v))
    elif how == "negated":
        k, v = torch._neg_view(k), torch._neg_view(v)
    else:
        k, v = (x.transpose(1, 2).contiguous().transpose(1, 2) for x in (k, v))
    cache = P.PageCache.empty(1, 9, heads, d, 16)
    where = tables([40, 20], [30, 7], 16, 9)
    P.store_pages(cache, 0, k, v, *where)
    to = [torch.zeros_like(x) if how != "unaligned" else torch.zeros(n, heads, d + 8, dtype=BF, device="cuda")[..., 1:d + 1] for x in (k, v)]
    if how == "negated":
        to = [torch._neg_view(x) for x in to]
    P.load_pages(cache, 0, *to, *where)
    for x, y in zip((k, v), to):
        assert same(y.resolve_neg(), expected(x.resolve_neg()))


@pytest.mark.parametrize("heads,d", [(2, 64), (8, 128), (17, 64), (4, 256)])
@pytest.mark.parametrize("garbage", [False, True])
def test_rows_outside_of_all_sequences_and_places_that_are_none(heads, d, garbage):
    cache = P.PageCache.empty(1, 4, heads, d, 16)
    for t in (cache.codes, cache.ratios, cache.exponents):
        t.random_(0, 256) if garbage else t.zero_()
    before = cache.exponents.clone()
    k, v = rows(12, heads, d, 3)
    # rows 0, 1 and 10, 11 are nobody's; the first sequence has two tokens before
    # position 0, the second a page that is none, the third one behind its table
    table, starts, lengths = ints([2, 0], [9, 1], [3, -1]), ints(2, 5, 8, 10), ints(1, 17, 33)
    P.store_pages(cache, 0, k, v, table, starts, lengths)
    to = [torch.full_like(k, 5.0) for _ in range(2)]
    P.load_pages(cache, 0, *to, table, starts, lengths)
    for x, y in zip((k, v), to):
        assert bool((y[:2] == 5).all()) and bool((y[10:] == 5).all())
        assert bool((y[2:4] == 0).all()) and same(y[4], expected(x[4]))
        assert bool(y[5:7].isnan().all()) and same(y[7], expected(x[7]))
        assert bool(y[8:10].isnan().all())
    if not garbage:
        assert int((cache.exponents != before).sum()) == 2 * heads * 2      # (two tokens, keys and values)


def test_offsets_past_32_bits():
    # 2.2 GB of codes of one head: the last pages lie behind 2^31
    pages = (1 << 31) // (2 * 256 * 128) + 100
    cache = P.PageCache.empty(1, pages, 1, 256, 256)
    k, v = rows(70, 1, 256, 2)
    where = ints([pages - 1], [0]), ints(0, 40, 70), ints(256, 30)
    P.store_pages(cache, 0, k, v, *where)
    to = [torch.empty_like(k) for _ in range(2)]
    P.load_pages(cache, 0, *to, *where)
    assert same(to[0], expected(k)) and same(to[1], expected(v))
    P.store_pages(cache, 0, *rows(256, 1, 256, 4), ints([pages - 1]), ints(0, 256), ints(256))
    P.copy_pages(cache, [pages - 1], [pages - 2])
    assert torch.equal(cache.codes[0, -1], cache.codes[0, -2])
    # the copy as the last page of a cache of its own, which small offsets reach
    small = P.PageCache(*(t[:, -2:].contiguous() for t in (cache.codes, cache.ratios, cache.exponents)))
    q = rows(2, 4, 256, 5)[0]
    for window in (0, 50):
        got, want = (P.page_attention(c, 0, q, ints([i]), ints(0, 2), ints(256), window=window) for c, i in ((cache, pages - 1), (small, 0)))
        assert torch.equal(got, want) and not bool(want.isnan().any())


@pytest.mark.parametrize("layers,heads,d,page,n", [(1, 1, 64, 16, 1), (3, 2, 128, 32, 5), (2, 3, 256, 16, 1000), (36, 8, 128, 64, 3)])
def test_pages_copied(layers, heads, d, page, n):
    pages = 2 * n + 3
    cache = P.PageCache.empty(layers, pages, heads, d, page)
    tensors = (cache.codes, cache.ratios, cache.exponents)
    for t in tensors:
        t.random_(0, 256)
    g = torch.Generator().manual_seed(n)
    order = torch.randperm(pages, generator=g).tolist()
    src, dst = [order[i // 2 if i % 5 == 0 else i] for i in range(n)], order[n:2 * n]      # (some come twice)
    want = [t.clone() for t in tensors]
    for t in want:
        t[:, torch.tensor(dst)] = t[:, torch.tensor(src)]
    P.copy_pages(cache, src, dst)
    for t, w in zip(tensors, want):
        assert torch.equal(t, w)
    P.copy_pages(cache, [], [])


def test_captured_with_other_lengths_at_replay():
    cache = P.PageCache.empty(1, 8, 2, 64, 16)
    k, v = rows(3, 2, 64, 9)
    table, starts, lengths = ints([0, 1], [2, 3], [4, 5]), ints(0, 1, 2, 3), ints(1, 1, 1)
    to = [torch.zeros_like(k) for _ in range(2)]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        P.store_pages(cache, 0, k, v, table, starts, lengths)
        P.copy_pages(cache, [1], [6])
        P.load_pages(cache, 0, *to, table, starts, lengths)
    for step in range(3):
        a, b = rows(3, 2, 64, step)
        k.copy_(a)
        v.copy_(b)
        lengths.copy_(ints(17 + step, 5, 16 + step))
        graph.replay()
        torch.cuda.synchronize()
        assert same(to[0], expected(a)) and same(to[1], expected(b))
        assert torch.equal(cache.codes[0, 6], cache.codes[0, 1])
