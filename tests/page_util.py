"""The paged 4-bit cache by its definition, in 64 bits and element by element."""
import torch

BF = torch.bfloat16


def held(x):
    """What rows [..., d] are held as: values (fp64; NaN rows all NaN) and the groups'
    scales [..., d / 32] (0 for rows of zeros and NaN)."""
    x = x.double().unflatten(-1, (-1, 32))
    top = x.abs().amax(-1)
    A = top.amax(-1, keepdim=True)
    bad, none = ~(A < 2.0 ** 100), A < 2.0 ** -100
    A = torch.where(bad | none, torch.ones_like(A), A)
    E = (torch.frexp(A).exponent - 1).double()
    r = torch.where(bad, torch.ones_like(top), top) * 2.0 ** (2.0 - E) / 7.0
    r = r.clamp(min=2.0 ** -14)
    ulp = 2.0 ** (torch.frexp(r).exponent - 4.0)
    s = torch.round(r / ulp) * ulp * 2.0 ** (E - 2.0)
    got = torch.round(torch.where(bad[..., None], torch.zeros_like(x), x) / s[..., None]).clamp(-7, 7) * s[..., None]
    got = torch.where(none[..., None], torch.zeros_like(got), got)
    got = torch.where(bad[..., None], torch.full_like(got, float("nan")), got)
    return got.flatten(-2), torch.where(bad | none, torch.zeros_like(s), s)


def nibble_place(d, value):
    """Where each element's nibble is in a row."""
    e = torch.arange(d)
    if value:
        return ((e % 32) // 4 * (d // 32) + e // 32) * 4 + e % 4
    return ((e % 32) // 8 * (d // 32) + e // 32) * 8 + e % 8


def values(cache, layer):
    """All values that the cache holds, fp64 [pages][2][heads][page][d]."""
    codes, ratios, exps = cache.codes[layer].cpu(), cache.ratios[layer].cpu(), cache.exponents[layer].cpu()
    d = cache.head_dim
    out = []
    for i in (0, 1):
        at = nibble_place(d, i)
        n = (codes[:, i][..., at // 2].long() >> (4 * (at % 2))) & 15
        b = ratios[:, i][..., torch.arange(d) // 32].long()
        x = (n - 8).double() * (1 + (b & 7).double() / 8) * 2.0 ** ((b >> 3) - 15).double()
        e = exps[..., i].double()
        x = x * 2.0 ** (e - 129.0)[..., None]
        out.append(x.masked_fill((e == 255)[..., None], float("nan")))
    return torch.stack(out, 1)


def ints(*values, device="cuda"):
    return torch.tensor(values, dtype=torch.int32, device=device)


def tables(lengths, new, page, pages, seed=0, width=None, device="cuda"):
    """Pages in any order for sequences of those lengths: table (its unused places hold
    pages that are none), starts, lengths."""
    g = torch.Generator().manual_seed(seed)
    order = torch.randperm(pages, generator=g).tolist()
    held_ = [-(-max(0, n) // page) for n in lengths]
    assert sum(held_) <= pages
    width = max(1, *held_) if width is None else width
    rows = []
    for n in held_:
        rows.append([order.pop() for _ in range(n)])
        rows[-1] += [pages + 7 if len(rows) % 2 else -1] * (width - n)
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    return ints(*rows, device=device), ints(*starts, device=device), ints(*lengths, device=device)
