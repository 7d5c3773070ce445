"""Calls of so many rows that a warp takes 8 or 16 of them, which other kernels do than
those of a token to a warp: what is loaded, and every byte of the cache, by the format's
definition.  All exact.

A warp takes 16 tokens where rows / 16 times the warps that a token's heads take, for keys
and values, comes to 32 for each of the card's 152 SMs, and 8 where rows / 8 times that
comes to 16; rows are stored with sixteen elements to a lane where a token's heads fill
warps so (heads d >= 1024), else with eight.  The sizes below are above and below both."""
import random

import pytest
import torch

from paper_2605_30574_gb300 import build as B
from paper_2605_30574_gb300.decoder import pages as P

from page_util import BF, held, nibble_place

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    B.build()


class Pool:
    """Some rows of d, what they are held as, and their bytes in a cache, by definition."""

    def __init__(self, d, seed, n=3000):
        g = torch.Generator().manual_seed(seed)
        x = torch.randn(n, d, generator=g) * torch.exp(torch.randn(n, d // 32, 1, generator=g)).expand(n, d // 32, 32).flatten(1)
        x = (x * 2.0 ** torch.randint(-60, 60, (n, 1), generator=g)).to(BF)
        x[:700] = (torch.randint(-255, 256, (700, d), generator=g) / 16).to(BF)          # (halfway between codes)
        x[0], x[1, 3], x[2, 5], x[3] = 0, float("nan"), float("inf"), 2.0 ** -110
        top = x.double().abs().amax(-1)
        self.bad, self.none = ~(top < 2.0 ** 100), top < 2.0 ** -100
        got, s = held(x)
        self.rows, self.held = x, got.to(BF)
        E = torch.frexp(torch.where(self.bad | self.none, torch.ones_like(top), top)).exponent.double() - 1
        self.exponents = torch.where(self.bad, 255, torch.where(self.none, 27, E + 127)).to(torch.uint8)
        s = torch.where((self.bad | self.none)[:, None], torch.ones_like(s), s)
        c = torch.round(got.unflatten(-1, (-1, 32)) / s[..., None]).flatten(-2).nan_to_num(0).long() + 8
        m, e = torch.frexp(s * 2.0 ** (2 - E)[:, None])                                  # (r = 2 m 2^(e - 1))
        self.ratios = ((e.long() + 14) * 8 + (m * 16 - 8).round().long()).to(torch.uint8)
        self.codes = []
        for value in (False, True):
            nibbles = torch.zeros_like(c)
            nibbles[:, nibble_place(d, value)] = c
            self.codes.append((nibbles[:, ::2] + 16 * nibbles[:, 1::2]).to(torch.uint8))


def ragged(n, page, seed):
    """Sequences of n new tokens in all: how many each has new, and of how many in all."""
    rng = random.Random(seed)
    # more than 32 begins within a warp's tokens; tokens before position 0; single ones
    got = [(0, 3)] * 40 + [(1, 1), (0, 9), (1, 16), (2, 16)] + [(0, 1)] * 45 + [(1, 1 + k) for k in range(20)] + [(5, 3), (1, 0), (3, 3)]
    left = n - sum(m for m, _ in got)
    while left:
        m = min(left, rng.choice((0, 1, 3, 7, page, 2 * page + 1, 300, 611)))
        got.append((m, m + rng.choice((0, 1, 5, page - 1, page, 2 * page + 3))))
        left -= m
    return got


@pytest.mark.parametrize("d,heads,page,n", [
    # narrow: eight rows to a warp, sixteen
    (64, 5, 16, 5003), (64, 5, 16, 19501), (128, 3, 64, 5003), (128, 3, 32, 19502), (256, 3, 32, 3301), (256, 3, 256, 13001),
    (64, 1, 16, 9801), (64, 2, 128, 38930),
    # a token's heads fill warps: eight, sixteen; stored by ones and loaded by eights
    (64, 16, 16, 4903), (64, 16, 32, 19502), (128, 8, 64, 4904), (128, 8, 16, 19501), (256, 4, 32, 4903), (256, 4, 16, 19509), (128, 9, 16, 3301),
    (128, 9, 32, 13002), (128, 8, 64, 2509), (256, 5, 16, 2509)])
@pytest.mark.parametrize("joined", [False, True])
def test_rows_and_bytes_of_many(d, heads, page, n, joined):
    seqs = ragged(n, page, seed=n + d)
    # a sequence's table may be too short for its last tokens, and hold a page that is none
    width = max(-(-L // page) for _, L in seqs) + 1
    seqs[-1] = (seqs[-1][0], width * page + min(3, seqs[-1][0]))
    pages = sum(min(width, -(-L // page)) for _, L in seqs) + 3
    order = list(range(pages))
    random.Random(d).shuffle(order)
    table = torch.full((len(seqs), width), -1, dtype=torch.int32)
    for b, (_, L) in enumerate(seqs):
        k = min(width, -(-L // page))
        table[b, :k] = torch.tensor(order[len(order) - k:], dtype=torch.int32)
        del order[len(order) - k:]
    longest = max(range(len(seqs) - 1), key=lambda b: seqs[b][0])
    none = (seqs[longest][1] - seqs[longest][0] // 2) // page
    table[longest, none] = pages

    # each row's place: -3 nobody's, -1 before the first position, -2 in no page, else its page
    before, behind = 3, 2
    rows = before + n + behind
    rows += rows % 8 == 0
    where, slot, starts = torch.full((rows,), -3), torch.zeros(rows, dtype=torch.long), [before]
    for b, (m, L) in enumerate(seqs):
        at, pos = starts[-1], torch.arange(L - m, L)
        i = pos.clamp(min=0) // page
        p = torch.where(i < width, table[b].long()[i.clamp(max=width - 1)], torch.full_like(i, -2))
        p = torch.where((p < 0) | (p >= pages), torch.full_like(p, -2), p)
        where[at:at + m], slot[at:at + m] = torch.where(pos < 0, torch.full_like(p, -1), p), pos.clamp(min=0) % page
        starts.append(at + m)
    there = where >= 0
    assert starts[-1] == before + n and int((where == -1).sum()) and int((where == -2).sum()) > 3

    pool = Pool(d, seed=n)
    g = torch.Generator().manual_seed(n)
    pick = torch.randint(0, len(pool.rows), (2, rows, heads), generator=g)
    if joined:
        x = pool.rows[pick].permute(1, 0, 2, 3).reshape(rows, 2 * heads, d).cuda()
        k, v = x[:, :heads], x[:, heads:]
    else:
        k, v = (pool.rows[i].cuda() for i in pick)

    cache = P.PageCache.empty(2, pages, heads, d, page)
    tensors = cache.codes, cache.ratios, cache.exponents
    for t in tensors:
        t.random_(0, 255)
    want = [t.cpu() for t in tensors]
    on = [torch.tensor(x, dtype=torch.int32).cuda() for x in (starts, [L for _, L in seqs])]
    P.store_pages(cache, 1, k, v, table.cuda(), *on)
    pg, sl = where[there], slot[there]
    for kv in (0, 1):
        i = pick[kv][there]
        want[0][1, :, kv].permute(0, 2, 1, 3)[pg, sl] = pool.codes[kv][i]
        # (what the scales of rows of zeros and NaN are is left open: as they are)
        ratios = cache.ratios[1, :, kv].cpu().permute(0, 2, 1, 3)[pg, sl]
        open_ = (pool.bad | pool.none)[i][..., None]
        want[1][1, :, kv].permute(0, 2, 1, 3)[pg, sl] = torch.where(open_, ratios, pool.ratios[i])
        want[2][1, ..., kv].permute(0, 2, 1)[pg, sl] = pool.exponents[i]
    for t, w in zip(tensors, want):
        assert torch.equal(t.cpu(), w)

    to = [torch.full_like(k, 5.0) for _ in range(2)]
    P.load_pages(cache, 1, *to, table.cuda(), *on)
    for kv, y in enumerate(to):
        y = y.cpu()
        want_rows = torch.full((rows, heads, d), 5.0, dtype=BF)
        want_rows[where == -1], want_rows[where == -2] = 0.0, float("nan")
        want_rows[there] = pool.held[pick[kv][there]]
        assert torch.equal(y.isnan(), want_rows.isnan()) and torch.equal(y.nan_to_num(9.0), want_rows.nan_to_num(9.0))
