"""Attention over the pages of a 4-bit cache against its definition in fp64.

Tolerances.  The keys and values are what the cache holds, exactly.  A row of q is
rounded to fp16 relative to its largest, to 2^-38 of that.  A tensor core adds 16 products
to a sum, each of the 17 cut at 2^-23 of the largest.

Scores: products are taken with codes of 1 to 15, and 8 times what they were taken with
off again: two products of a group and one of what is taken off, of up to 15 s |q|, s the
group's scale: 2 17 15 2^-23 < 2^-14 of s |q|, so e = 2^-14 scale sum of s |q| with all
groups' and the third product's; a weight is off by e relatively, and so is the row's
sum.  Weights are rounded to fp16 before and after the group's scale, 2^-11 each (below
fp16's normal range by 2^-25, against the largest of 2^6 and more: 2^-31 of it, for each
key); fp32 sums leave 2^-16.  Output: the codes of two elements in one, of up to 119 s, and
what the second adds to them, for 16 keys at once: 2 17 119 2^-23 < 2^-11 of the largest
p s among them, s the value's scale.  Together, with S the sum of p |v| and N keys,

  (2^-10 + 2^-16 + 2 max e) S + 2^-11 sum p s + 2^-28 N max p |v|,

and the output's rounding, 2^-8 |o|.
"""
import math

import pytest
import torch

from paper_2605_30574_gb300 import build as B
from paper_2605_30574_gb300.decoder import pages as P

from page_util import BF, held, ints, tables, values

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    B.build()


def filled(lengths, new, heads, d, page, seed=0, spread=0.5, width=None):
    """A cache that holds rows for the sequences, and garbage elsewhere."""
    pages = sum(-(-max(0, n) // page) for n in lengths) + 2
    cache = P.PageCache.empty(1, pages, heads, d, page)
    for t in (cache.codes, cache.ratios, cache.exponents):
        t.random_(0, 256)
    cache.exponents[0, :, :, ::3] = 255
    where = tables(lengths, new, page, pages, seed, width)
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = sum(max(0, x) for x in lengths)
    k, v = torch.randn(2, n, heads, d, generator=g, device="cuda").unbind(0)
    k = (k * torch.exp(spread * torch.randn(1, heads, d, generator=g, device="cuda"))).to(BF)
    v = (v * torch.exp(spread * torch.randn(n, heads, 1, generator=g, device="cuda"))).to(BF)
    starts = [0]
    for x in lengths:
        starts.append(starts[-1] + max(0, x))
    if n:
        P.store_pages(cache, 0, k, v, where[0], ints(*starts), ints(*[max(0, x) for x in lengths]))
    return cache, where


def queries(n, heads, d, seed=0, size=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed + 77)
    return (size * torch.randn(n, heads, d, generator=g, device="cuda")).to(BF)


def definition(cache, q, table, starts, lengths, scale, window):
    """fp64 outputs and the bound of their errors (see above)."""
    all_, page, heads, d = values(cache, 0), cache.page, cache.kv_heads, cache.head_dim
    s_all = 2.0 ** (cache.exponents[0].cpu().double() - 129.0).movedim(-1, 1)[..., None] * (
        (1 + (cache.ratios[0].cpu() & 7).double() / 8) * 2.0 ** ((cache.ratios[0].cpu().long() >> 3) - 15).double())
    q = q.cpu().double()
    G = q.shape[1] // heads
    out, bound = torch.zeros_like(q), torch.zeros_like(q)
    for b in range(len(lengths)):
        L = max(0, int(lengths[b]))
        ids = [int(table[b, i]) for i in range(-(-L // page))]
        n = int(starts[b + 1]) - int(starts[b])
        for h in range(heads):
            k, v, ks, vs = ((torch.cat([x[i, j, h] for i in ids])[:L] if ids else x[:0, j, h].flatten(0, 1))
                            for x, j in ((all_, 0), (all_, 1), (s_all, 0), (s_all, 1)))
            for i in range(n):
                pos = int(lengths[b]) - n + i
                lo = max(0, pos - window + 1) if window else 0
                if pos < lo:
                    continue
                kk, vv, kss = k[lo:pos + 1], v[lo:pos + 1], ks[lo:pos + 1]
                row = int(starts[b]) + i
                for x in range(h * G, h * G + G):
                    s = scale * (kk @ q[row, x])
                    p = torch.softmax(s, 0)
                    e = abs(scale) * float((kss @ q[row, x].abs().view(-1, 32).sum(-1)).max()) * 2.0 ** -14
                    out[row, x] = p @ vv
                    pv = p[:, None] * vv.abs()
                    ps = (p @ vs[lo:pos + 1]).repeat_interleave(32)
                    bound[row, x] = ((2.0 ** -10 + 2.0 ** -16 + 2 * e) * pv.sum(0) + 2.0 ** -11 * ps + 2.0 ** -28 * len(s) * pv.max()
                                     + 2.0 ** -8 * out[row, x].abs())
    return out, bound


def check(cache, q, where, scale=None, window=0, rows=None):
    got = P.page_attention(cache, 0, q, *where, scale=scale, window=window)
    want, bound = definition(cache, q, *where, 1 / math.sqrt(q.shape[-1]) if scale is None else scale, window)
    rows = slice(0, int(where[1][-1])) if rows is None else rows
    err = (got.cpu().double() - want).abs()[rows]
    assert bool((err <= bound[rows]).all()), float((err / bound[rows].clamp(min=1e-300)).max())
    return got


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("heads,G,page", [(1, 1, 16), (2, 4, 64), (3, 7, 32), (2, 8, 128), (1, 12, 16), (1, 33, 256)])
def test_single_tokens(d, heads, G, page):
    lengths = [1, 2, 15, 16, 17, 64, 100, 255]
    cache, where = filled(lengths, [1] * 8, heads, d, page, seed=d + G)
    check(cache, queries(8, heads * G, d), where)


@pytest.mark.parametrize("d,heads,G,page", [(64, 2, 4, 16), (128, 2, 4, 64), (256, 1, 2, 32), (128, 1, 3, 16)])
@pytest.mark.parametrize("new,lengths", [([3, 1, 0, 8], [3, 40, 9, 130]), ([17], [500]), ([5, 2], [5, 2]), ([1, 20, 1], [1, 20, 300])])
@pytest.mark.parametrize("window", [0, 1, 21])
def test_several_tokens_and_windows(d, heads, G, page, new, lengths, window):
    cache, where = filled(lengths, new, heads, d, page, seed=window)
    check(cache, queries(sum(new), heads * G, d), where, window=window)


@pytest.mark.parametrize("d,heads,G", [(64, 1, 4), (128, 2, 8), (256, 1, 1)])
@pytest.mark.parametrize("length", [1000, 4099, 20000])
def test_keys_that_are_split(d, heads, G, length):
    cache, where = filled([length], [1], heads, d, 64, seed=length)
    check(cache, queries(1, heads * G, d), where)


def test_many_sequences_of_all_lengths():
    g = torch.Generator().manual_seed(1)
    lengths = [int(x) for x in (2 ** (11 * torch.rand(700, generator=g))).long()]
    cache, where = filled(lengths, [1] * 700, 1, 64, 16, seed=4)
    check(cache, queries(700, 2, 64), where)


@pytest.mark.parametrize("d,heads,G,page", [(64, 2, 4, 16), (128, 2, 4, 64), (256, 1, 2, 32), (128, 1, 3, 16), (128, 1, 12, 16), (64, 1, 33, 32)])
@pytest.mark.parametrize("new,lengths", [([3, 1, 0, 8], [3, 40, 9, 130]), ([17], [500]), ([1, 20, 1], [1, 20, 300]), ([1], [1]), ([1] * 6, [60] * 6)])
@pytest.mark.parametrize("window", [0, 21])
def test_tables_far_wider_than_lengths(d, heads, G, page, new, lengths, window):
    """Work that is shared by the stage, of sequences that are short."""
    cache, where = filled(lengths, new, heads, d, page, seed=window, width=40000 // page)
    check(cache, queries(sum(new), heads * G, d), where, window=window)


@pytest.mark.parametrize("d,heads,G,batch,page", [(64, 3, 1, 900, 16), (128, 2, 4, 2000, 16), (256, 1, 3, 1300, 32), (128, 1, 2, 300, 64), (64, 1, 40, 500, 16)])
def test_many_short_sequences(d, heads, G, batch, page):
    """More tiles than warps, and fewer; sequences without tokens among them."""
    lengths = [(7 * i) % 41 for i in range(batch)]
    new = [min(n, 1 + (i % 50 == 0)) for i, n in enumerate(lengths)]
    cache, where = filled(lengths, new, heads, d, page, seed=batch)
    check(cache, queries(sum(new), heads * G, d), where)


@pytest.mark.parametrize("d,heads,G", [(64, 2, 4), (128, 8, 4), (128, 1, 16), (256, 4, 2)])
@pytest.mark.parametrize("batch,length", [(1, 100), (1, 300), (5, 300), (20, 200)])
def test_warps_that_share_a_tile(d, heads, G, batch, length):
    lengths = [max(0, length - 13 * i) for i in range(batch)]
    new = [min(1, n) for n in lengths]
    cache, where = filled(lengths, new, heads, d, 16, seed=batch)
    check(cache, queries(sum(new), heads * G, d), where)
    check(cache, queries(sum(new), heads * G, d), where, window=70)


def test_rows_that_see_nothing():
    # no tokens at all, more new tokens than the sequence has, none new
    cache, where = filled([0, 2, 5, -3], [1, 4, 0, 1], 2, 64, 16)
    got = check(cache, queries(6, 4, 64), where)
    assert bool((got[0] == 0).all()) and bool((got[1:3] == 0).all()) and bool((got[5] == 0).all())


def test_rows_outside_of_all_sequences():
    cache, (table, starts, lengths) = filled([30, 9], [2, 1], 2, 64, 16)
    q = queries(8, 4, 64)
    out = torch.full_like(q, 7.0)
    got = P.page_attention(cache, 0, q, table, starts + 2, lengths, out=out)
    assert got is out and bool((out[:2] == 7).all()) and bool((out[5:] == 7).all())
    check(cache, q, (table, starts + 2, lengths), rows=slice(2, 5))


@pytest.mark.parametrize("size", [0.0, 1e-3, 30.0, -4.0, 1e4])
@pytest.mark.parametrize("spread", [0.0, 3.0])
def test_sharp_and_flat_rows(size, spread):
    cache, where = filled([300, 77], [1, 1], 2, 128, 32, spread=spread)
    check(cache, queries(2, 8, 128, size=abs(size)), where, scale=math.copysign(1 / math.sqrt(128), size or 1))


@pytest.mark.parametrize("kind", ["values far apart", "keys far apart", "elements far apart"])
def test_sizes_far_apart(kind):
    """Weights relative to the row's largest product of weight and size: large values
    that no row looks at leave the others theirs."""
    cache, where = filled([200], [1], 1, 64, 16)
    n = 200
    k, v = queries(n, 1, 64, 5).float(), queries(n, 1, 64, 6).float()
    q = queries(1, 4, 64)
    if kind == "values far apart":
        v *= 2.0 ** torch.linspace(-90, 90, n, device="cuda")[:, None, None]
        k[:, :, :] = q[:, :1].float() * torch.linspace(40, -40, n, device="cuda")[:, None, None]
    elif kind == "keys far apart":
        k *= 2.0 ** torch.linspace(-60, 4, n, device="cuda")[:, None, None]
    else:
        q = (q.float() * 2.0 ** torch.linspace(-25, 0, 64, device="cuda")).to(BF)
    P.store_pages(cache, 0, k.to(BF), v.to(BF), where[0], ints(0, n), ints(n))
    check(cache, q, where)


def test_what_no_row_sees_may_be_nan():
    cache, where = filled([40], [1], 2, 64, 64)
    n = 64
    k, v = queries(n, 2, 64, 5), queries(n, 2, 64, 6)
    k[40:] = float("nan")
    v[40:] = float("inf")
    P.store_pages(cache, 0, k, v, where[0], ints(0, n), ints(n))
    check(cache, queries(1, 4, 64), where)
    # before the window
    k[:8], v[:8] = float("inf"), float("nan")
    P.store_pages(cache, 0, k, v, where[0], ints(0, n), ints(n))
    check(cache, queries(1, 4, 64), where, window=32)


@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_scores_of_any_size(sign):
    """One key's score is far above the others', all of them far below (or above) 0."""
    cache, where = filled([100], [1], 1, 64, 64)
    k, v = torch.zeros(100, 1, 64, device="cuda"), queries(100, 1, 64, 6)
    k[:, 0, 0] = sign * 2.0 ** 60 * torch.linspace(1, 2, 100, device="cuda")
    q = torch.zeros(1, 2, 64, dtype=BF, device="cuda")
    q[..., 0] = 2.0 ** 50
    P.store_pages(cache, 0, k.to(BF), v, where[0], ints(0, 100), ints(100))
    got = P.page_attention(cache, 0, q, *where, scale=1.0)
    held_k, held_v = values(cache, 0)[int(where[0][0, 0]), :, 0, :, :], values(cache, 0)[int(where[0][0, 1]), :, 0, :36, :]
    kk, vv = (torch.cat([held_k[i], held_v[i]]) for i in (0, 1))
    best = kk[:, 0] == kk[:, 0].max()                  # (equal scores share)
    want = vv[best].mean(0)
    assert bool(((got[0].cpu().double() - want).abs() <= 2.0 ** -7 * vv[best].abs().mean(0) + 2.0 ** -10).all())


@pytest.mark.parametrize("which", ["k", "v", "q"])
def test_nan_that_is_seen(which):
    cache, where = filled([40, 40], [2, 2], 2, 64, 64)
    n = 40
    k, v, q = queries(2 * n, 2, 64, 5), queries(2 * n, 2, 64, 6), queries(4, 4, 64)
    if which == "q":
        q[1, 2, 3] = float("nan")
        q[2, 1, 5] = float("inf")
    else:
        (k if which == "k" else v)[39, 1, 9] = float("nan")       # (seen by the first sequence's last token)
    P.store_pages(cache, 0, k, v, where[0], ints(0, n, 2 * n), ints(n, n))
    got = P.page_attention(cache, 0, q, *where)
    nan = got.isnan().all(-1)
    assert torch.equal(nan, got.isnan().any(-1))
    want = torch.zeros_like(nan)
    if which == "q":
        want[1, 2] = want[2, 1] = True
    else:
        want[1, 2:] = True
    assert torch.equal(nan, want)


def test_pages_that_are_none_make_their_rows_nan():
    cache, (table, starts, lengths) = filled([40, 40, 40], [1, 2, 1], 2, 64, 16)
    want, bound = definition(cache, queries(4, 4, 64), table, starts, lengths, 1 / 8, 0)
    table[1, 1] = cache.pages
    lengths[2] = 16 * table.shape[1] + 1
    got = P.page_attention(cache, 0, queries(4, 4, 64), table, starts, lengths)
    assert bool(((got[0].cpu().double() - want[0]).abs() <= bound[0]).all()) and bool(got[1:].isnan().all())


def test_lengths_and_starts_that_say_too_much():
    """A length past the table's pages: its rows are NaN, and no more keys are gone through
    than the table has.  Starts past the rows that there are: those that there are."""
    cache, (table, starts, lengths) = filled([40, 40], [1, 3], 2, 64, 16)
    want, bound = definition(cache, queries(4, 4, 64), table, starts, lengths, 1 / 8, 0)
    long_ = lengths.clone()
    for n in (16 * table.shape[1] + 1, 1 << 20, (1 << 31) - 1):
        long_[0] = n
        got = P.page_attention(cache, 0, queries(4, 4, 64), table, starts, long_)
        assert bool(got[0].isnan().all()) and bool(((got[1:].cpu().double() - want[1:]).abs() <= bound[1:]).all())
    got = P.page_attention(cache, 0, queries(4, 4, 64)[:3].contiguous(), table, starts, lengths)
    assert bool(((got.cpu().double() - want[:3]).abs() <= bound[:3]).all())


@pytest.mark.parametrize("d,heads,G", [(64, 2, 4), (128, 1, 8), (64, 1, 12)])
@pytest.mark.parametrize("window", [(1 << 31) - 1, (1 << 31) - 8, 1 << 30])
def test_windows_wider_than_all(d, heads, G, window):
    """Rows before position 0 next to rows that see keys."""
    cache, where = filled([5, 40], [8, 3], heads, d, 16)
    check(cache, queries(11, heads * G, d), where, window=window)


@pytest.mark.parametrize("d,heads,G", [(64, 2, 4), (128, 1, 8), (64, 1, 12)])
def test_lengths_to_the_last(d, heads, G):
    """2^31 - 1 tokens, in pages that come again and again, of which a window sees the last."""
    page, W, tail = 256, 1 << 23, 5
    cache, (table, starts, _) = filled([page * tail], [2], heads, d, page)
    table = table[:, torch.arange(W, device="cuda") % tail].contiguous()
    lengths, last = ints((1 << 31) - 1), table[:, -tail:].contiguous()
    q, scale = queries(2, heads * G, d), d ** -0.5
    got = P.page_attention(cache, 0, q, table, starts, lengths, window=1000)
    want, bound = definition(cache, q, last, starts, [page * tail - 1], scale, 1000)
    assert bool(((got.cpu().double() - want).abs() <= bound).all())
    k, v, kk, vv = (torch.empty(2, heads, d, dtype=BF, device="cuda") for _ in range(4))
    P.load_pages(cache, 0, k, v, table, starts, lengths)
    P.load_pages(cache, 0, kk, vv, last, starts, ints(page * tail - 1))
    assert torch.equal(k, kk) and torch.equal(v, vv)


@pytest.mark.parametrize("how", ["joined", "transposed", "unaligned", "negated"])
def test_strides_of_q(how):
    cache, where = filled([40, 9], [1, 3], 2, 128, 16)
    q = queries(4, 8, 128)
    want = P.page_attention(cache, 0, q, *where)
    if how == "joined":
        y = torch.cat([q, q], 1)[:, :8]
    elif how == "transposed":
        y = q.transpose(0, 1).contiguous().transpose(0, 1)
    elif how == "unaligned":
        y = torch.zeros(4, 8, 136, dtype=BF, device="cuda")[..., 3:131].copy_(q)
    else:
        y = torch._neg_view(-q)
    assert torch.equal(P.page_attention(cache, 0, y, *where), want)


def test_the_same_bits_again_and_in_graphs():
    lengths = [3000, 17, 900, 1, 64]
    cache, where = filled(lengths, [1, 2, 1, 1, 3], 2, 128, 32)
    q = queries(8, 16, 128)
    want = P.page_attention(cache, 0, q, *where)
    streams, outs, graphs = [torch.cuda.Stream() for _ in range(2)], [torch.zeros_like(q) for _ in range(2)], []
    for s, o in zip(streams, outs):
        s.wait_stream(torch.cuda.current_stream())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            P.page_attention(cache, 0, q, *where, out=o)
        graphs.append(graph)
    for _ in range(5):
        for o in outs:
            o.zero_()
        torch.cuda.synchronize()
        for s, graph in zip(streams, graphs):
            with torch.cuda.stream(s):
                graph.replay()
        torch.cuda.synchronize()
        for o in outs:
            assert torch.equal(o, want)
    # replayed with other lengths
    where[2].copy_(ints(2000, 16, 900, 1, 60))
    graphs[0].replay()
    torch.cuda.synchronize()
    want, bound = definition(cache, q, *where, 1 / math.sqrt(128), 0)
    assert bool(((outs[0].cpu().double() - want).abs() <= bound).all())


def test_one_step_as_it_is_used():
    """A step's tokens stored, then attended to, over pages that two sequences share."""
    page, d, heads = 16, 64, 2
    cache = P.PageCache.empty(2, 8, heads, d, page)
    k, v = queries(40, heads, d, 1), queries(40, heads, d, 2)
    P.store_pages(cache, 1, k, v, ints([0, 1, 2]), ints(0, 40), ints(40))
    # the second goes its own way from token 32 on
    P.copy_pages(cache, [2], [5])
    table = ints([0, 1, 2], [0, 1, 5])
    for step in range(10):
        k1, v1, q = queries(2, heads, d, 10 + step), queries(2, heads, d, 30 + step), queries(2, 4, d, 50 + step)
        where = table, ints(0, 1, 2), ints(41 + step, 41 + step)
        if step == 8:
            table = where[0].new_tensor([[0, 1, 2, 3], [0, 1, 5, 6]])
        if step >= 8:
            where = table, *where[1:]
        P.store_pages(cache, 1, k1, v1, *where)
        got = P.page_attention(cache, 1, q, *where)
        sub = P.PageCache(cache.codes[1:], cache.ratios[1:], cache.exponents[1:])
        want, bound = definition(sub, q, *where, 1 / math.sqrt(d), 0)
        assert bool(((got.cpu().double() - want).abs() <= bound).all())
