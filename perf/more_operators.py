"""What the operators of a paged key/value cache in 4 bits are measured on.

A sweep's decode holds a cache for every run.  Pages of a few tokens let runs
share what they have in common (a cell of a sweep is the clean run up to its
onset, so it starts as a fork of it), and 4 bits a value let a card hold 3.7
times as many.  A case's "op" names what is done:

* ``store``   ``store_pages`` of new tokens, then ``load_pages`` of the same;
* ``load``    ``load_pages`` of whole sequences;
* ``attend``  ``page_attention`` of each sequence's newest tokens over its pages;
* ``copy``    ``copy_pages``, of the pages that a fork or a compaction moves.

The cache.  A row is one token's key or value of one head, of d elements in groups
of 32.  With A its largest magnitude and E = floor(log2 A), a group's scale is
s = r 2^(E - 2), where r is (the group's largest magnitude) 2^(2 - E) / 7 rounded to
four significant bits, and at least 2^-14; a value is c s with c = x / s rounded to
a whole number between -7 and 7 (ties to even, both).  A row with A below 2^-100
is zero (E = -100), one with A of 2^100 and more or not finite is NaN.
  codes      uint8 [layers][pages][2][heads][page][d / 2]: c + 8 in a nibble, the
             low one first; keys, then values.  Keys' words of 8 elements are
             ordered by their number modulo 4, values' runs of 4 by theirs modulo 8.
  ratios     uint8 [layers][pages][2][heads][page][d / 32]: bits 14 to 7 of r in fp16
  exponents  uint8 [layers][pages][heads][page][2]: E + 127, or 255 for NaN
Sequence b has lengths[b] tokens, in the pages table[b]; its newest are the rows
starts[b] to starts[b + 1] of what is stored, loaded or attends.
"""
import math

import torch

own = False
DEV = "cuda"
BF16 = torch.bfloat16


# --------------------------------------------------------------------------
# the cases
# --------------------------------------------------------------------------
def _case(name, op, **sizes):
    c = dict(op=op, **sizes)
    return c if name is None else dict(c, name=name)


def _tokens(name, op, batch, tokens, low, high, hkv, d, page, joined=False):
    return _case(name, op, batch=batch, tokens=tokens, low=low, high=high, hkv=hkv, d=d, page=page, joined=joined)


def _attend(name, batch, tokens, low, high, hq, hkv, d, page, window=0):
    return _case(name, "attend", batch=batch, tokens=tokens, low=low, high=high, hq=hq, hkv=hkv, d=d, page=page, window=window)


def _copy(name, copied, layers, hkv, d, page, spare):
    return _case(name, "copy", copied=copied, layers=layers, hkv=hkv, d=d, page=page, spare=spare)


def listed():
    return [
        # a step's new token of one run: all latency
        _tokens("store_one_token", "store", 1, 1, 200, 200, 2, 64, 16),
        # a step's new tokens of the ladder's batch, out of the joined projection
        _tokens("store_step_512", "store", 512, 1, 4096, 4352, 8, 128, 64, True),
        # ragged prompts behind what their runs hold already
        _tokens("store_prompts", "store", 7, 4999, 5000, 6001, 8, 128, 64),
        # the spans of some prompts, for attention over many queries at once
        _tokens("load_spans_wide", "load", 12, 0, 3001, 4096, 4, 256, 32),
        # one run of the tiny decoder: all latency
        _attend("attend_one_short", 1, 1, 147, 147, 8, 2, 64, 16),
        # one run over a long context: the keys have to be split
        _attend("attend_one_long", 1, 1, 131072, 131072, 32, 8, 128, 64),
        # a step of 512 runs over prompts of 4096 and what they generated
        _attend("attend_step_512", 512, 1, 4096, 4352, 32, 8, 128, 64),
        # runs of all lengths, from one token
        _attend("attend_ragged", 200, 1, 1, 9000, 32, 8, 128, 32),
        # a layer with a sliding window, wide heads
        _attend("attend_window_wide", 64, 1, 1500, 4000, 8, 4, 256, 128, 1024),
        # a few tokens of each run at once: proposed tokens that are looked at together
        _attend("attend_proposed", 48, 8, 1000, 3000, 32, 8, 128, 64),
        # the begun pages of 20 cells that leave a clean run
        _copy("copy_fork", 20, 36, 8, 128, 64, 44),
        # a third of the pages moved down, after runs have ended
        _copy("copy_compact", 340, 36, 8, 128, 64, 344),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("store", "load", "attend", "attend", "attend", "attend", "copy"))
    d, page = rng.choice((64, 128, 128, 256)), rng.choice((16, 32, 64, 64, 128))
    hkv = rng.choice((1, 2, 4, 8, 8))
    if op == "copy":
        layers = rng.choice((1, 4, 34, 36))
        copied = min(_log(rng, 1, 2000), 340 * 36 * 8 * 64 * 128 // (layers * hkv * page * d))
        return _copy(None, max(1, copied), layers, hkv, d, page, _log(rng, 1, 40))
    batch = _log(rng, 1, 600)
    if op == "attend":
        group = rng.choice((1, 2, 4, 4, 7, 8))
        while hkv * group > 64:
            hkv //= 2
        most = 512 * 4096 * 8 * 128 // (batch * hkv * d)
        high = min(_log(rng, 1, 131072), most)
        low = max(1, int(high * rng.choice((0.0, 0.5, 0.95, 1.0))))
        window = rng.choice((0, 0, 0, _log(rng, 1, 4096)))
        return _attend(None, batch, rng.choice((1, 1, 1, 2, 5, 16)), low, high, hkv * group, hkv, d, page, window)
    most = 7 * 3000 * 8 * 128 // (batch * hkv * d)
    tokens = max(1, min(_log(rng, 1, 8192), most))
    high = tokens if op == "load" else tokens + _log(rng, 1, 2000)
    low = max(tokens if op == "store" else 1, int(high * rng.choice((0.3, 0.9, 1.0))))
    return _tokens(None, op, batch, 0 if op == "load" else tokens, low, high, hkv, d, page, op == "store" and rng.random() < 0.5)


def _share(i, step):
    return (0.5 + i * step) % 1.0


def _lengths(c):
    """Tokens of each sequence, the newest included."""
    return [min(c["high"], int(c["low"] * (c["high"] / c["low"]) ** _share(i, 0.6180339887) + 0.5)) for i in range(c["batch"])]


def _new(c):
    """The newest tokens of each sequence (all of them: 0 in the case)."""
    if c["tokens"] == 0:
        return _lengths(c)
    if c["tokens"] == 1:
        return [1] * c["batch"]
    return [min(n, int(_share(i, 0.4142135624) * c["tokens"]) + 1) for i, n in enumerate(_lengths(c))]


# --------------------------------------------------------------------------
# what a program has in hand
# --------------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV)


def _rows(g, n, hkv, d):
    """Keys and values [n][heads][d]: keys with channels of other sizes than the
    rest, as normed and rotated ones have, values with larger and smaller tokens."""
    k = _randn(g, n, hkv, d) * torch.exp(0.6 * _randn(g, 1, hkv, d))
    v = _randn(g, n, hkv, d) * torch.exp(0.5 * _randn(g, n, hkv, 1))
    return k.to(BF16), v.to(BF16)


def _filled(g, layers, pages, hkv, page, d):
    """A cache whose pages are all filled, as its three tensors."""
    codes = torch.empty((layers, pages, 2, hkv, page, d // 2), dtype=torch.uint8, device=DEV)
    ratios = torch.empty((layers, pages, 2, hkv, page, d // 32), dtype=torch.uint8, device=DEV)
    exponents = torch.empty((layers, pages, hkv, page, 2), dtype=torch.uint8, device=DEV)
    step = max(1, (1 << 27) // (hkv * page * d))
    for l in range(layers):
        for p in range(0, pages, step):
            n = min(step, pages - p)
            for i, x in enumerate(_rows(g, n * page, hkv, d)):
                c, r, e = _quantised(x, i)
                codes[l, p:p + n, i] = c.view(n, page, hkv, -1).transpose(1, 2)
                ratios[l, p:p + n, i] = r.view(n, page, hkv, -1).transpose(1, 2)
                exponents[l, p:p + n, :, :, i] = e.view(n, page, hkv).transpose(1, 2)
    return codes, ratios, exponents


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def prepare(case, seed):
    g, c = _gen(seed), case
    hkv, d, page = c["hkv"], c["d"], c["page"]
    if c["op"] == "copy":
        # (what is copied, where to, and pages that stay as they are)
        n = 2 * c["copied"] + c["spare"]
        cache = _filled(g, 1, n, hkv, page, d)
        cache = tuple(torch.cat([x.roll(l, 1) for l in range(c["layers"])]) for x in cache)
        order = torch.randperm(n, generator=g, device=DEV).tolist()
        st = dict(op="copy", cache=cache, src=order[:c["copied"]], dst=order[c["copied"]:2 * c["copied"]])
    else:
        lengths, new = _lengths(c), _new(c)
        held = [-(-n // page) for n in lengths]
        pages, width = sum(held), max(held)
        order = torch.randperm(pages + 3, generator=g, device=DEV).tolist()
        table, at = [], 0
        for n in held:
            table.append(order[at:at + n] + [-1] * (width - n))
            at += n
        if c["op"] == "store":
            cache = tuple(torch.zeros(shape, dtype=torch.uint8, device=DEV) for shape in (
                (1, pages + 3, 2, hkv, page, d // 2), (1, pages + 3, 2, hkv, page, d // 32), (1, pages + 3, hkv, page, 2)))
        else:
            cache = _filled(g, 1, pages + 3, hkv, page, d)
        starts = [0]
        for n in new:
            starts.append(starts[-1] + n)
        st = dict(op=c["op"], cache=cache, table=_int32(table), starts=_int32(starts), lengths=_int32(lengths),
                  host_lengths=lengths, host_new=new)
        if c["op"] == "attend":
            st.update(q=_randn(g, starts[-1], c["hq"], d).to(BF16), scale=1.0 / math.sqrt(d), window=c["window"])
        elif c["op"] == "store":
            k, v = _rows(g, starts[-1], hkv, d)
            if c["joined"]:
                kv = torch.cat([k, v], 1)
                k, v = kv[:, :hkv], kv[:, hkv:]
            st.update(k=k, v=v)
        if c["op"] != "attend":
            st.update(to=[torch.empty((starts[-1], hkv, d), dtype=BF16, device=DEV) for _ in range(2)])
    if own:
        from paper_2605_30574_gb300.decoder.pages import PageCache
        st["cache"] = PageCache(*st["cache"])
    return st


# --------------------------------------------------------------------------
# the plain forms, in 32 bits
# --------------------------------------------------------------------------
def _power(e):
    """2^e, exactly, of whole numbers between -126 and 127."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _quantised(x, values):
    """Rows [...][d] of keys (values 0) or values (1): codes as they are stored,
    ratios and exponents."""
    x = x.float().unflatten(-1, (-1, 32))
    most = x.abs().amax(-1)
    A = most.amax(-1, keepdim=True)
    bad, none = ~(A < 2.0 ** 100), A < 2.0 ** -100
    E = torch.frexp(A).exponent - 1
    E = torch.where(bad | none, torch.full_like(E, -100), E)
    unit = _power(E - 2)
    least = torch.full_like(most, 2.0 ** -14)
    # (a division by a tensor: one by a number may be a product with its inverse)
    m, e = torch.frexp(torch.maximum(most * _power(2 - E) / torch.full_like(most, 7.0), least))
    r = torch.where(bad | none, least, (m * 16.0).round() * _power(e - 4))
    c = (x / (r * unit)[..., None]).round().clamp(-7.0, 7.0)
    c = torch.where((bad | none)[..., None], torch.zeros_like(c), c)
    c = (c + 8.0).to(torch.uint8)
    d = 32 * c.shape[-2]
    # (words t + 4 i of keys, runs t + 8 i of values, ordered by t)
    c = c.unflatten(-1, (8, 4) if values else (4, 8)).transpose(-3, -2).reshape(*c.shape[:-2], d // 2, 2)
    codes = c[..., 0] | (c[..., 1] << 4)
    ratios = (r.half().view(torch.int16) >> 7).to(torch.uint8)
    exponents = torch.where(bad, torch.full_like(E, 255), E + 127)[..., 0].to(torch.uint8)
    return codes, ratios, exponents


def _values(codes, ratios, exponents, values):
    """The rows that codes, ratios and exponents stand for, in fp32."""
    d = 2 * codes.shape[-1]
    c = torch.stack([codes & 15, codes >> 4], -1).flatten(-2)
    c = c.unflatten(-1, (8, d // 32, 4) if values else (4, d // 32, 8)).transpose(-3, -2).reshape(*codes.shape[:-1], d // 32, 32)
    r = (ratios.to(torch.int16) << 7).view(torch.float16).float()
    unit = _power(exponents.int().clamp(max=254) - 129)
    unit = torch.where(exponents == 255, torch.full_like(unit, float("nan")), unit)
    return ((c.float() - 8.0) * (r * unit[..., None])[..., None]).flatten(-2)


def _tokens_at(st):
    """Per row of the newest tokens its page and its place in it."""
    starts, lengths, table, page = st["starts"].long(), st["lengths"].long(), st["table"], st["cache"][0].shape[-2]
    new = starts[1:] - starts[:-1]
    b = torch.repeat_interleave(torch.arange(len(new), device=DEV), new, output_size=sum(st["host_new"]))
    at = torch.arange(len(b), device=DEV) - starts[b] + (lengths - new)[b]
    return table[b, at // page].long(), at % page


def _store_plain(st):
    codes, ratios, exponents = (x[0] for x in st["cache"])
    page, slot = _tokens_at(st)
    for i, x in enumerate((st["k"], st["v"])):
        c, r, e = _quantised(x, i)
        codes[page, i, :, slot] = c
        ratios[page, i, :, slot] = r
        exponents[page, :, slot, i] = e


def _load_plain(st):
    codes, ratios, exponents = (x[0] for x in st["cache"])
    page, slot = _tokens_at(st)
    for i, to in enumerate(st["to"]):
        to.copy_(_values(codes[page, i, :, slot], ratios[page, i, :, slot], exponents[page, :, slot, i], i))
    return dict(k=st["to"][0], v=st["to"][1])


def _attend_plain(st):
    codes, ratios, exponents = (x[0] for x in st["cache"])
    q, scale, window, table = st["q"], st["scale"], st["window"], st["table"].long().clamp(min=0)
    hkv, page, half = codes.shape[2:]
    Hq, d = q.shape[1:]
    lengths, new = st["host_lengths"], st["host_new"]
    out = torch.empty_like(q)
    first, row = 0, 0
    while first < len(lengths):
        # as many sequences as make a batch of some size, padded to the longest
        last, most = first, 0
        while last < len(lengths) and (last == first or max(most, lengths[last]) * (last - first + 1) * hkv * d <= 1 << 28):
            most = max(most, lengths[last])
            last += 1
        width, n = -(-most // page), max(new[first:last])
        ids = table[first:last, :width]
        k, v = (_values(codes[ids, i], ratios[ids, i], exponents[ids][..., i], i).transpose(2, 3).flatten(1, 2) for i in (0, 1))
        tokens = torch.arange(n, device=DEV)
        count = st["starts"][first + 1:last + 1, None] - st["starts"][first:last, None]
        at = st["lengths"][first:last, None] - count + tokens                     # [b][n]: positions of the queries
        rows = (st["starts"][first:last, None] + tokens).clamp(max=q.shape[0] - 1)
        x = q[rows.long()].float().unflatten(2, (hkv, -1))                        # [b][n][hkv][G][d]
        s = torch.einsum("bnhgd,bjhd->bhgnj", x, k) * scale
        j = torch.arange(width * page, device=DEV)
        seen = j <= at[..., None]
        if window:
            seen &= j > at[..., None] - window
        s.masked_fill_(~seen[:, None, None], float("-inf"))
        p = (s - s.amax(-1, keepdim=True).clamp(min=-1e30)).exp()
        total = p.sum(-1, keepdim=True)
        p = p / torch.where(total == 0, torch.ones_like(total), total)
        v = v.masked_fill(~seen.any(1)[..., None, None], 0.0)
        got = torch.einsum("bhgnj,bjhd->bnhgd", p, v).flatten(2, 3).to(BF16)
        keep = (tokens < count)
        out[row:row + sum(new[first:last])] = got[keep]
        row += sum(new[first:last])
        first = last
    return out


def _copy_plain(st):
    src, dst = (torch.tensor(st[n], device=DEV) for n in ("src", "dst"))
    for x in st["cache"]:
        x[:, dst] = x[:, src]


# --------------------------------------------------------------------------
# one pass
# --------------------------------------------------------------------------
def _run_own(st):
    from paper_2605_30574_gb300.decoder import pages as P
    cache = st["cache"]
    if st["op"] == "copy":
        P.copy_pages(cache, st["src"], st["dst"])
        return dict(codes=cache.codes, ratios=cache.ratios, exponents=cache.exponents)
    where = (st["table"], st["starts"], st["lengths"])
    if st["op"] == "attend":
        return P.page_attention(cache, 0, st["q"], *where, scale=st["scale"], window=st["window"])
    if st["op"] == "store":
        P.store_pages(cache, 0, st["k"], st["v"], *where)
    P.load_pages(cache, 0, *st["to"], *where)
    return dict(k=st["to"][0], v=st["to"][1])


def run(st):
    if own:
        return _run_own(st)
    if st["op"] == "copy":
        _copy_plain(st)
        return dict(codes=st["cache"][0], ratios=st["cache"][1], exponents=st["cache"][2])
    if st["op"] == "attend":
        return _attend_plain(st)
    if st["op"] == "store":
        _store_plain(st)
    return _load_plain(st)


def _row_bytes(c):
    """A token's keys and values of all heads."""
    return c["hkv"] * (c["d"] + c["d"] // 16 + 2)


def _seen(c):
    """Per sequence its newest tokens and the keys that any of them sees, and all
    pairs of a query and a key."""
    for L, n in zip(_lengths(c), _new(c)):
        w = c["window"] or L
        yield n, min(L, w + n - 1), sum(min(w, L - n + i + 1) for i in range(n))


def work(case):
    c = case
    if c["op"] == "copy":
        return {"bytes": 2 * c["copied"] * c["layers"] * c["page"] * _row_bytes(c), "flops": 0}
    if c["op"] == "attend":
        each = list(_seen(c))
        return {"bytes": sum(k for _, k, _ in each) * _row_bytes(c) + sum(4 * n * c["hq"] * c["d"] for n in _new(c)),
                "flops": 4 * sum(p for _, _, p in each) * c["hq"] * c["d"]}
    rows = sum(_new(c)) * c["hkv"]
    one = rows * 4 * c["d"] + sum(_new(c)) * _row_bytes(c)
    return {"bytes": one * (2 if c["op"] == "store" else 1), "flops": rows * 2 * c["d"] * (6 if c["op"] == "store" else 2)}


# --------------------------------------------------------------------------
# the definitions in 64 bits
# --------------------------------------------------------------------------
def _exact_values(codes, ratios, exponents, values):
    """Rows [...][d], element by element: where its nibble is and what it stands for."""
    d = 2 * codes.shape[-1]
    e = torch.arange(d, device=codes.device)
    if values:
        place = ((e % 32) // 4 * (d // 32) + e // 32) * 4 + e % 4
    else:
        place = ((e % 32) // 8 * (d // 32) + e // 32) * 8 + e % 8
    nibble = (codes[..., place // 2].long() >> (4 * (place % 2))) & 15
    byte = ratios[..., e // 32].long()
    x = (nibble - 8).double() * (1.0 + (byte & 7).double() / 8.0) * torch.exp2((byte >> 3).double() - 15.0)
    x = x * torch.exp2(exponents.double() - 129.0)[..., None]
    return x.masked_fill((exponents == 255)[..., None], float("nan"))


def _exact_rounded(x):
    """What rows [...][d] are held as."""
    x = x.double().unflatten(-1, (-1, 32))
    top = x.abs().amax(-1)
    A = top.amax(-1, keepdim=True)
    bad, none = ~(A < 2.0 ** 100), A < 2.0 ** -100
    A = torch.where(bad | none, torch.ones_like(A), A)
    E = torch.floor(torch.log2(A))
    E = torch.where(torch.exp2(E) > A, E - 1, torch.where(torch.exp2(E + 1) <= A, E + 1, E))
    want = (top * torch.exp2(2.0 - E) / 7.0).clamp(min=2.0 ** -14)
    want = torch.where(want.isnan(), torch.ones_like(want), want)
    ulp = torch.exp2(torch.floor(torch.log2(want)) - 3.0)
    s = (torch.round(want / ulp) * ulp * torch.exp2(E - 2.0))[..., None]
    got = torch.clamp(torch.round(x / s), -7, 7) * s
    got = torch.where(none[..., None], torch.zeros_like(got), got)
    return got.masked_fill(bad[..., None], float("nan")).flatten(-2)


def _exact_attend(st):
    codes, ratios, exponents = (x[0] for x in st["cache"])
    q, scale, window, page = st["q"], st["scale"], st["window"], codes.shape[-2]
    hkv = codes.shape[2]
    G = q.shape[1] // hkv
    out, row = torch.zeros(q.shape, dtype=torch.float64, device=DEV), 0
    for b, (L, n) in enumerate(zip(st["host_lengths"], st["host_new"])):
        lo = max(0, L - n + 1 - window) // page if window else 0
        ids = st["table"][b, lo:-(-L // page)].long()
        for h in range(hkv):
            k, v = (_exact_values(codes[ids, i, h].flatten(0, 1), ratios[ids, i, h].flatten(0, 1),
                                  exponents[ids, h, :, i].flatten(0, 1), i) for i in (0, 1))
            k, v = k[:L - lo * page], v[:L - lo * page]
            s = scale * (q[row:row + n, h * G:(h + 1) * G].double().flatten(0, 1) @ k.T)     # [n G][keys]
            at = L - n + torch.arange(n, device=DEV).repeat_interleave(G)[:, None]
            j = lo * page + torch.arange(len(k), device=DEV)
            hidden = (j > at) | (j <= at - window if window else j < 0)
            p = torch.softmax(s.masked_fill(hidden, float("-inf")), -1).nan_to_num(0.0)
            out[row:row + n, h * G:(h + 1) * G] = (p @ v).view(n, G, -1)
        row += n
    return out


def exact(case, seed):
    plain = prepare(case, seed)
    cache = plain["cache"]
    if not isinstance(cache, tuple):
        plain["cache"] = cache = (cache.codes, cache.ratios, cache.exponents)
    if case["op"] == "attend":
        return _exact_attend(plain)
    if case["op"] == "copy":
        got = [x.clone() for x in cache]
        for s, t in zip(plain["src"], plain["dst"]):
            for x, y in zip(got, cache):
                x[:, t] = y[:, s]
        return dict(zip(("codes", "ratios", "exponents"), got))
    if case["op"] == "store":
        return dict(k=_exact_rounded(plain["k"]), v=_exact_rounded(plain["v"]))
    page, slot = _tokens_at(plain)
    codes, ratios, exponents = (x[0] for x in cache)
    return {name: _exact_values(codes[page, i, :, slot], ratios[page, i, :, slot], exponents[page, :, slot, i], i)
            for i, name in enumerate("kv")}
