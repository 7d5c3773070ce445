"""What the decoder's scoring and training operators are measured on.

A probe of the prompt KV cache needs more than the greedy tokens of a spliced
decode: how likely the clean run's tokens stay, how far the distribution moved
from the clean run's, and the gradient of that with respect to the K and V of
the prompt span.  Three operators give these, and a case's "op" names one:

* ``score``    ``token_logprobs``: per row of logits the log probability of a
               given token, the entropy, and the ``top`` most likely tokens;
* ``distill``  ``distill_loss_and_grad``: the divergence of the rows'
               distributions from a teacher's ``top`` alternatives, with its
               gradient ("rest": all other tokens together count as one more);
* ``attn``     ``attention_backward``: the gradients of causal attention of
               ``tq`` queries, the last positions of ``tk``, with respect to
               queries, keys and values.

Rows of logits are those of a decode step (one per cell of a sweep), or of a
continuation scored at once.
"""
import math

import torch

own = False
DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
NONE = float("-inf")


# --------------------------------------------------------------------------
# the cases
# --------------------------------------------------------------------------
def _score(name, rows, vocab, dtype, top, temperature=1.0, banned=False):
    c = dict(op="score", rows=rows, vocab=vocab, dtype=dtype, top=top, temperature=temperature, banned=banned)
    return c if name is None else dict(c, name=name)


def _distill(name, rows, vocab, dtype, top, rest, temperature=1.0, skipped=False):
    c = dict(op="distill", rows=rows, vocab=vocab, dtype=dtype, top=top, rest=rest, temperature=temperature, skipped=skipped)
    return c if name is None else dict(c, name=name)


def _attn(name, batch, tq, tk, hq, hkv, d):
    c = dict(op="attn", batch=batch, tq=tq, tk=tk, hq=hq, hkv=hkv, d=d)
    return c if name is None else dict(c, name=name)


def listed():
    return [
        # one sequence's step: all latency
        _score("score_one_row", 1, 151936, "f32", 20),
        # the tiny sweep's batch of 80 cells
        _score("score_tiny_sweep", 80, 512, "f32", 5),
        # the donor-noise ladder's batch of 512 cells
        _score("score_ladder_step", 512, 151936, "f32", 20),
        # a long continuation at once, in the weights' own type, of an odd
        # vocabulary with banned tokens, with a teacher's worth of alternatives
        _score("score_long_odd_bf16", 2047, 100003, "bf16", 64, 0.7, True),
        # the tiny sweep against its clean run
        _distill("distill_tiny_sweep", 80, 512, "f32", 8, False, 2.0),
        # the ladder's batch against its clean run, the rest counted
        _distill("distill_ladder_step", 512, 151936, "f32", 32, True),
        # a long ragged batch: rows of padding, odd rows that start anywhere
        _distill("distill_long_odd_bf16", 1999, 100003, "bf16", 64, True, 1.5, True),
        # a short continuation of the tiny sweep's prompt
        _attn("attn_tiny", 1, 16, 144, 8, 2, 64),
        # a prompt of middling length
        _attn("attn_prefill_1024", 1, 1024, 1024, 32, 8, 128),
        # the ladder's prompt
        _attn("attn_prefill_4096", 1, 4096, 4096, 32, 8, 128),
        # continuations of that prompt, a few cells at once
        _attn("attn_continue_4096", 4, 100, 4196, 32, 8, 128),
        # the wide heads, an odd length
        _attn("attn_wide_odd", 2, 1003, 1003, 8, 4, 256),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("score", "distill", "attn"))
    if op == "attn":
        d = rng.choice((64, 128, 128, 256))
        group = rng.choice((1, 2, 4, 4, 7, 8))
        hkv = rng.choice((1, 2, 4, 8))
        while hkv * group > 32:
            group //= 2
        tq = _log(rng, 1, 4096)
        tk = max(1, tq + rng.choice((0, 0, 1, -1)) * _log(rng, 1, 4096 if rng.random() < 0.5 else 64))
        batch = rng.choice((1, 1, 2, 3, 5))
        while batch > 1 and batch * tq * tk * hkv * group * d > 4096 * 4096 * 32 * 64:
            batch -= 1
        tk = min(tk, 4096 * 4096 * 32 * 128 // (tq * hkv * group * d))
        return _attn(None, batch, tq, tk, hkv * group, hkv, d)
    vocab = _log(rng, 257, 160000)
    rows = min(_log(rng, 1, 2048), 90_000_000 // vocab)
    dtype = rng.choice(("f32", "f32", "bf16"))
    temperature = rng.choice((1.0, 1.0, 0.6, 2.0))
    if op == "score":
        return _score(None, rows, vocab, dtype, rng.choice((0, 1, 5, 20, 20, 50, 128)), temperature, rng.random() < 0.3)
    return _distill(None, rows, vocab, dtype, rng.choice((1, 8, 20, 32, 64, 128)), rng.random() < 0.5, temperature,
                    rng.random() < 0.3)


# --------------------------------------------------------------------------
# what a program has in hand
# --------------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV)


def prepare(case, seed):
    g = _gen(seed)
    if case["op"] == "attn":
        B, Tq, Tk, Hq, Hkv, d = (case[n] for n in ("batch", "tq", "tk", "hq", "hkv", "d"))
        bf = torch.bfloat16
        # normed heads: elements of unit variance; later positions' gradients
        # larger and smaller by some factors of two, as a loss gives them
        q, dout = _randn(g, B, Tq, Hq, d).to(bf), _randn(g, B, Tq, Hq, d)
        dout = (dout * torch.exp2(_randn(g, B, Tq, 1, 1))).to(bf)
        k, v = _randn(g, B, Hkv, Tk, d).to(bf), _randn(g, B, Hkv, Tk, d).to(bf)
        scale = 1.0 / math.sqrt(d)
        out, lse = _attention(q, k, v, scale)
        return dict(op="attn", q=q, k=k, v=v, dout=dout, out=out.to(bf), lse=lse, scale=scale)
    rows, V, dtype, top = case["rows"], case["vocab"], TYPES[case["dtype"]], case["top"]
    # logits of a model that is sure of some tokens and not of others
    x = _randn(g, rows, V)
    x *= 1.0 + 2.0 * torch.rand(rows, 1, generator=g, device=DEV)
    at = torch.randint(0, V, (rows, 4), generator=g, device=DEV)
    x.scatter_add_(1, at, 4.0 + 8.0 * torch.rand(rows, 4, generator=g, device=DEV))
    if case["op"] == "score":
        if case["banned"]:
            x.masked_fill_(torch.rand(V, generator=g, device=DEV) < 0.05, NONE)
        logits = x.to(dtype)
        # the greedy token for most rows, any for the others, none for a few
        tokens = torch.where(torch.rand(rows, generator=g, device=DEV) < 0.7, logits.argmax(-1), at[:, 0])
        tokens = torch.where(torch.rand(rows, generator=g, device=DEV) < 0.02, torch.full_like(tokens, -1), tokens)
        return dict(op="score", logits=logits, tokens=tokens, top=top, temperature=case["temperature"])
    # the teacher: the same rows, moved a little
    t = x + 0.7 * _randn(g, rows, V)
    t /= case["temperature"]
    teacher, ids = t.topk(top, dim=-1)
    teacher = teacher - t.logsumexp(-1, keepdim=True)
    weight = torch.full((rows,), 1.0 / rows, device=DEV)
    if case["skipped"]:
        weight *= torch.rand(rows, generator=g, device=DEV) < 0.9
    return dict(op="distill", logits=x.to(dtype), ids=ids, teacher=teacher, weight=weight, rest=case["rest"],
                temperature=case["temperature"])


# --------------------------------------------------------------------------
# the plain forms, in 32 bits
# --------------------------------------------------------------------------
def _visible(Tq, Tk):
    """[Tq][Tk]: query i is position Tk - Tq + i and sees the keys up to it."""
    i = torch.arange(Tq, device=DEV)[:, None] + (Tk - Tq)
    return torch.arange(Tk, device=DEV)[None, :] <= i


def _by_heads(x, Hkv):
    """[B][T][Hq][d] -> [B][Hkv][G][T][d] in fp32."""
    return x.float().unflatten(2, (Hkv, x.shape[2] // Hkv)).permute(0, 2, 3, 1, 4)


def _weights(q, k, scale):
    """Attention weights [B][Hkv][G][Tq][Tk] and their rows' log sums."""
    Hkv, Tq, Tk = k.shape[1], q.shape[1], k.shape[2]
    s = _by_heads(q, Hkv) @ k.float()[:, :, None].transpose(-1, -2)
    s *= scale
    s.masked_fill_(~_visible(Tq, Tk), NONE)
    m = s.amax(-1, keepdim=True)
    s -= torch.where(m == NONE, torch.zeros_like(m), m)
    p = s.exp_()
    l = p.sum(-1, keepdim=True)
    p /= torch.where(l == 0, torch.ones_like(l), l)
    return p, (m + l.log())[..., 0].flatten(1, 2)


def _back(x):
    """[B][Hkv][G][T][d] -> [B][T][Hq][d]."""
    return x.permute(0, 3, 1, 2, 4).flatten(2, 3)


def _attention(q, k, v, scale):
    p, lse = _weights(q, k, scale)
    return _back(p @ v.float()[:, :, None]), lse


def _attn_plain(st):
    q, k, v, dout, scale = st["q"], st["k"], st["v"], st["dout"], st["scale"]
    Hkv = k.shape[1]
    p, _ = _weights(q, k, scale)
    go = _by_heads(dout, Hkv)
    dv = (p.transpose(-1, -2) @ go).sum(2)
    ds = go @ v.float()[:, :, None].transpose(-1, -2)
    ds -= (ds * p).sum(-1, keepdim=True)
    ds *= p
    ds *= scale
    dq = _back(ds @ k.float()[:, :, None])
    dk = (ds.transpose(-1, -2) @ _by_heads(q, Hkv)).sum(2)
    return dict(dq=dq.to(q.dtype), dk=dk.to(k.dtype), dv=dv.to(v.dtype))


def _score_plain(st):
    x = st["logits"].float() / st["temperature"]
    m = x.amax(-1, keepdim=True)
    z = x - torch.where(m == NONE, torch.zeros_like(m), m)
    e = z.exp()
    s = e.sum(-1, keepdim=True)
    log_s = s.log()
    tokens = st["tokens"]
    logprobs = z.gather(1, tokens.clamp(min=0)[:, None]) - log_s
    logprobs = torch.where(tokens < 0, torch.zeros_like(logprobs[:, 0]), logprobs[:, 0])
    entropy = (log_s - torch.where(e > 0, e * z, torch.zeros_like(e)).sum(-1, keepdim=True) / s)[:, 0]
    got = dict(logprobs=logprobs, entropy=entropy)
    if st["top"]:
        # (a stable order: the lowest index first among equals)
        ids = st["logits"].sort(dim=-1, descending=True, stable=True).indices[:, :st["top"]].contiguous()
        got.update(top_logprobs=z.gather(1, ids) - log_s, top_ids=ids)
    return got


def _distill_plain(st):
    x, ids, teacher, T = st["logits"].float() / st["temperature"], st["ids"], st["teacher"], st["temperature"]
    log_p = x - x.amax(-1, keepdim=True)
    log_p -= log_p.exp().sum(-1, keepdim=True).log()
    p = log_p.exp()
    if st["rest"]:
        q = teacher.exp()
        q_rest = (1.0 - q.sum(-1, keepdim=True)).clamp(min=0)
        p_rest = p.scatter(1, ids, 0.0).sum(-1, keepdim=True)
        loss = (q * (teacher - log_p.gather(1, ids))).sum(-1)
        loss = loss + torch.where(q_rest > 0, q_rest * (q_rest.log() - p_rest.log()), torch.zeros_like(q_rest))[:, 0]
        top = p.gather(1, ids) - q
        grad = (p * (1.0 - q_rest / p_rest)).scatter(1, ids, top)
    else:
        log_q = teacher - teacher.logsumexp(-1, keepdim=True)
        q = log_q.exp()
        loss = (q * (log_q - log_p.gather(1, ids))).sum(-1)
        grad = p.scatter_add(1, ids, -q)
    weight = st["weight"]
    return dict(loss=loss * weight, grad=(grad * (weight / T)[:, None]).to(st["logits"].dtype))


# --------------------------------------------------------------------------
# the framework's calls
# --------------------------------------------------------------------------
def _score_own(st):
    from paper_2605_30574_gb300.decoder.scoring import token_logprobs
    got = token_logprobs(st["logits"], st["tokens"], top=st["top"], temperature=st["temperature"])
    out = dict(logprobs=got.logprobs, entropy=got.entropy)
    if st["top"]:
        out.update(top_logprobs=got.top_logprobs, top_ids=got.top_ids)
    return out


def _distill_own(st):
    from paper_2605_30574_gb300.decoder.scoring import distill_loss_and_grad
    loss, grad = distill_loss_and_grad(st["logits"], st["ids"], st["teacher"], weight=st["weight"], rest=st["rest"],
                                       temperature=st["temperature"])
    return dict(loss=loss, grad=grad)


def _attn_own(st):
    from paper_2605_30574_gb300.decoder.attention import attention_backward
    dq, dk, dv = attention_backward(st["dout"], st["q"], st["k"], st["v"], st["out"], st["lse"], st["scale"])
    return dict(dq=dq, dk=dk, dv=dv)


# --------------------------------------------------------------------------
# one pass
# --------------------------------------------------------------------------
def run(st):
    if own:
        return {"score": _score_own, "distill": _distill_own, "attn": _attn_own}[st["op"]](st)
    return {"score": _score_plain, "distill": _distill_plain, "attn": _attn_plain}[st["op"]](st)


def work(case):
    if case["op"] == "attn":
        B, Tq, Tk, Hq, Hkv, d = (case[n] for n in ("batch", "tq", "tk", "hq", "hkv", "d"))
        first = max(0, Tq - Tk)
        pairs = sum(Tk - Tq + i + 1 for i in range(first, Tq))
        return {"bytes": B * (8 * Tq * Hq * d + 8 * Tk * Hkv * d + 4 * Tq * Hq), "flops": 10 * B * Hq * pairs * d}
    rows, V, K, size = case["rows"], case["vocab"], case["top"], 4 if case["dtype"] == "f32" else 2
    if case["op"] == "score":
        return {"bytes": rows * (V * size + 16 + 12 * K), "flops": 5 * rows * V}
    return {"bytes": rows * (2 * V * size + 8 + 12 * K), "flops": 8 * rows * V}


# --------------------------------------------------------------------------
# the definitions in 64 bits
# --------------------------------------------------------------------------
def _exact_attn(st, scale):
    q, k, v, go = (st[n].double() for n in ("q", "k", "v", "dout"))
    B, Tq, Hq, d = q.shape
    Hkv, Tk = k.shape[1:3]
    dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    seen = _visible(Tq, Tk)
    for b in range(B):
        for h in range(Hq):
            kv = h // (Hq // Hkv)
            s = (scale * (q[b, :, h] @ k[b, kv].T)).masked_fill(~seen, NONE)
            p = torch.softmax(s, -1).nan_to_num(0.0)          # (a row that sees no key has no weights)
            g = go[b, :, h]
            o = p @ v[b, kv]
            ds = p * (g @ v[b, kv].T - (g * o).sum(-1, keepdim=True))
            dv[b, kv] += p.T @ g
            dk[b, kv] += scale * (ds.T @ q[b, :, h])
            dq[b, :, h] = scale * (ds @ k[b, kv])
    return dict(dq=dq, dk=dk, dv=dv)


def _exact_score(st):
    rows = []
    for x, t in zip(st["logits"].split(256), st["tokens"].split(256)):
        lp = torch.log_softmax(x.double() / st["temperature"], -1)
        p = lp.exp()
        one = lp.gather(1, t.clamp(min=0)[:, None])[:, 0].masked_fill(t < 0, 0.0)
        H = -torch.where(p > 0, p * lp, torch.zeros_like(p)).sum(-1)
        rows.append((one, H, lp.topk(st["top"], -1).values if st["top"] else one))
    one, H, top = (torch.cat(c) for c in zip(*rows))
    got = dict(logprobs=one, entropy=H)
    if st["top"]:
        got.update(top_logprobs=top, top_ids=None)
    return got


def _exact_distill(st):
    loss, grad = [], []
    T = st["temperature"]
    for x, ids, t, w in zip(*(st[n].split(256) for n in ("logits", "ids", "teacher", "weight"))):
        lp, t, w = torch.log_softmax(x.double() / T, -1), t.double(), w.double()
        target = torch.zeros_like(lp)
        if st["rest"]:
            q = t.exp()
            inside = torch.zeros_like(lp, dtype=torch.bool).scatter_(1, ids, True)
            qr = (1.0 - q.sum(-1)).clamp(min=0)
            lpr = torch.logsumexp(lp.masked_fill(inside, NONE), -1)
            l = (q * (t - lp.gather(1, ids))).sum(-1) + torch.where(qr > 0, qr * (qr.log() - lpr), torch.zeros_like(qr))
            # the teacher's distribution with its rest shared out as the student does
            target = (lp - lpr[:, None]).exp() * qr[:, None]
            target = target.masked_fill(inside, 0.0).scatter_add(1, ids, q)
        else:
            q = torch.softmax(t, -1)
            l = (q * (q.log() - lp.gather(1, ids))).sum(-1)
            target.scatter_add_(1, ids, q)
        loss.append(w * l)
        grad.append((w / T)[:, None] * (lp.exp() - target))
    return dict(loss=torch.cat(loss), grad=torch.cat(grad))


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "attn":
        return _exact_attn(st, st["scale"])
    return _exact_score(st) if case["op"] == "score" else _exact_distill(st)
