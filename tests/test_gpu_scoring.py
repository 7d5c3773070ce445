"""Token scores and the distillation loss against their definitions in fp64.

Tolerances.  The row sums are fp32 sums of at most a few hundred elements per
lane, then a tree, of terms that are each within about 2^-21 (the exponential's
own error, and its argument's rounding times the argument, 2^-24 x 32 at the
most where a term still counts): log s is within 2^-20 of exact, absolutely.  A
log probability is (x - m) / T - log s, two more roundings of its own size; an
entropy is log s minus a mean of (x - m), of the same error relative to the
magnitudes summed.  So |error| <= 2^-19 (1 + |value| + spread), with the spread
the largest |z - m| that carries weight, below 32.  A gradient element is
w / T (p - q) with p and q each within 2^-20 relative: |error| <= 2^-19 w / T (p +
q), plus half a unit of its type.  The loss is a sum of q times differences of
log probabilities: |error| <= 2^-19 sum q (1 + |log q| + |log p|).
"""
import math

import pytest
import torch

from paper_2605_30574_gb300 import build as B
from paper_2605_30574_gb300 import decoder as K
from paper_2605_30574_gb300.decoder import scoring

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
HALF_ULP = {F32: 2.0 ** -24, BF16: 2.0 ** -8, F16: 2.0 ** -11}
EPS = 2.0 ** -19
INF = float("inf")


@pytest.fixture(scope="module", autouse=True)
def _built():
    B.build()
    yield
    K.check_device_error()


def gen(seed=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def logits_of(g, rows, V, dtype, spread=3.0):
    return (torch.randn(rows, V, generator=g, device="cuda") * spread).to(dtype)


def plain_scores(x, tokens, top, T):
    """fp64, rows with something above -inf and no NaN."""
    z = x.double() / T
    lp = torch.log_softmax(z, -1)
    p = lp.exp()
    H = -torch.where(p > 0, p * lp, torch.zeros_like(p)).sum(-1)
    order = x.float().sort(dim=-1, descending=True, stable=True).indices[:, :top]
    one = lp.gather(1, tokens.clamp(min=0)[:, None])[:, 0].masked_fill(tokens < 0, 0.0)
    return one, H, lp.gather(1, order), order


def near(got, want, bound):
    got = got.double()
    assert torch.equal(got.isnan(), want.isnan())
    same = (got == want) | got.isnan()
    off = ((got - want).abs() / bound).masked_fill(same, 0.0)
    assert float(off.max() if off.numel() else 0) <= 1.0, float(off.max())


def check_scores(x, tokens, top, T=1.0):
    got = scoring.token_logprobs(x, tokens, top=top, temperature=T)
    one, H, best, order = plain_scores(x, tokens, top, T)
    near(got.logprobs, one, EPS * (33 + one.abs()))
    near(got.entropy, H, EPS * (33 + H.abs()))
    if top:
        assert torch.equal(got.top_ids, order)
        near(got.top_logprobs, best, EPS * (33 + best.abs()))
    else:
        assert got.top_ids is None and got.top_logprobs is None
    return got


# a row of one token; less than a word, odd starts of every row; no split, two
# looks of a warp, splits over a cluster; every width of the list
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("rows,V,top", [(1, 1, 1), (5, 3, 3), (9, 33, 20), (3, 257, 128), (80, 512, 5), (7, 4099, 33),
                                        (2, 8191, 64), (3, 70001, 100), (1, 151936, 20), (300, 10007, 1), (2, 50001, 0)])
def test_scores(rows, V, top, dtype):
    g = gen(V)
    x = logits_of(g, rows, V, dtype)
    tokens = torch.randint(0, V, (rows,), generator=g, device="cuda")
    tokens[0] = -1
    check_scores(x, tokens, top, 1.0 if rows % 2 else 0.7)


@pytest.mark.parametrize("order", ["ascending", "descending", "equal", "few values"])
@pytest.mark.parametrize("top", [5, 128])
def test_scores_of_ordered_rows(order, top):
    V = 40001
    x = torch.linspace(-9, 9, V, device="cuda").repeat(3, 1)
    if order == "descending":
        x = x.flip(-1).contiguous()
    elif order == "equal":
        x = torch.zeros_like(x)
        x[1] = -0.0
        x[2, ::2] = -0.0
    elif order == "few values":
        x = torch.randint(0, 3, x.shape, generator=gen(3), device="cuda").float()
    check_scores(x, torch.tensor([0, V - 1, 17], device="cuda"), top)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_scores_of_masked_rows(dtype):
    V = 20011
    g = gen(7)
    x = logits_of(g, 8, V, dtype)
    low = torch.finfo(dtype).min
    x[0, torch.rand(V, generator=g, device="cuda") < 0.9] = -INF
    x[1, :-3] = -INF                    # fewer tokens than are asked for
    x[2, :] = -INF                      # none
    x[3, torch.rand(V, generator=g, device="cuda") < 0.9] = low
    x[4, :] = low                       # all alike
    x[5, 5:] = low
    x[6, 11] = float("nan")
    x[7, V - 1] = INF
    tokens = torch.tensor([3, V - 1, 5, 8, 9, 2, 1, 0], device="cuda")
    got = scoring.token_logprobs(x, tokens, top=20)
    fine = [0, 1, 3, 4, 5]
    one, H, best, order = plain_scores(x[fine], tokens[fine], 20, 1.0)
    near(got.logprobs[fine], one, EPS * (33 + one.abs()))
    near(got.entropy[fine], H, EPS * (33 + H.abs()))
    assert torch.equal(got.top_ids[fine], order)
    near(got.top_logprobs[fine], best, EPS * (33 + best.abs()))
    assert got.logprobs[2] == -INF and got.entropy[2] == 0 and bool((got.top_logprobs[2] == -INF).all())
    assert got.top_ids[2].tolist() == list(range(20))
    for r in (6, 7):
        assert bool(got.logprobs[r].isnan()) and bool(got.entropy[r].isnan()) and bool(got.top_logprobs[r].isnan().all())
    assert got.top_ids[7, 0] == V - 1
    assert 11 not in got.top_ids[6].tolist()


def test_scores_of_a_token_outside():
    x = logits_of(gen(1), 4, 100, F32)
    got = scoring.token_logprobs(x, torch.tensor([100, -1, -100, 1 << 40], device="cuda"))
    assert bool(got.logprobs[[0, 3]].isnan().all()) and got.logprobs[1:3].tolist() == [0.0, 0.0]
    assert scoring.token_logprobs(x).logprobs is None


def test_scores_of_views_shapes_and_streams():
    g = gen(2)
    padded = logits_of(g, 6, 1040, BF16)
    tokens = torch.randint(0, 1001, (6,), generator=g, device="cuda")
    want = scoring.token_logprobs(padded[:, 3:1004].contiguous(), tokens, top=9)
    for x in (padded[:, 3:1004], padded[:, 3:1004].t().contiguous().t()):
        got = scoring.token_logprobs(x, tokens.int(), top=9)
        for a, b in zip(got, want):
            assert torch.allclose(a, b, rtol=1e-5, atol=1e-5)
    got = scoring.token_logprobs(padded[:, 3:1004].unflatten(0, (2, 3)), tokens.view(2, 3), top=9)
    assert got.top_ids.shape == (2, 3, 9) and torch.equal(got.top_ids.view(6, 9), want.top_ids)
    one = scoring.token_logprobs(padded[0, 3:1004], tokens[0], top=9)
    assert one.entropy.shape == () and torch.equal(one.top_ids, want.top_ids[0])
    none = scoring.token_logprobs(padded[:0], tokens[:0], top=4)
    assert none.top_ids.shape == (0, 4) and none.entropy.shape == (0,)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        x = padded * 2
        again = scoring.token_logprobs(x, tokens, top=9)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(again.top_ids, scoring.token_logprobs(padded * 2, tokens, top=9).top_ids)


def test_scores_same_bits():
    x = logits_of(gen(9), 40, 151936, F32)
    tokens = x.argmax(-1)
    a, b = (scoring.token_logprobs(x, tokens, top=64) for _ in range(2))
    assert all(torch.equal(u, v) for u, v in zip(a, b))


# ---- distillation ----

def plain_distill(x, ids, teacher, weight, rest, T):
    """Loss and gradient in fp64, and the sizes that their errors go by."""
    x, t = x.double(), teacher.double()
    rows, V = x.shape
    there = ids >= 0
    at = ids.clamp(min=0)
    z = x / T
    empty = (x == -INF).all(-1, keepdim=True)
    lp = torch.log_softmax(torch.where(empty, torch.zeros_like(z), z), -1).masked_fill(empty, -INF)
    p = lp.exp()
    t = torch.where(there, t, torch.full_like(t, -INF))
    any_q = (t > -INF).any(-1, keepdim=True)
    if rest:
        q = t.exp()
    else:
        q = torch.where(any_q, torch.softmax(torch.where(any_q, t, torch.zeros_like(t)), -1), torch.zeros_like(t))
    target = torch.zeros(rows, V + 1, dtype=torch.double, device="cuda")
    slots = torch.where(there, ids, torch.full_like(ids, V))
    target.scatter_add_(1, slots, q)
    term = torch.where(q > 0, q * (q.log() - lp.gather(1, at)), torch.zeros_like(q))
    size = torch.where(q > 0, q * (1 + q.log().abs() + lp.gather(1, at).abs()), torch.zeros_like(q)).sum(-1)
    loss = term.sum(-1)
    grad = p * q.sum(-1, keepdim=True) - target[:, :V] if not rest else None
    mass = p + target[:, :V]
    if rest:
        inside = torch.zeros(rows, V + 1, dtype=torch.bool, device="cuda").scatter_(1, slots, True)[:, :V]
        qr = (1 - q.sum(-1)).clamp(min=0)
        lpr = torch.logsumexp(lp.masked_fill(inside, -INF), -1)
        loss = loss + torch.where(qr > 0, qr * (qr.log() - lpr), torch.zeros_like(qr))
        size = size + torch.where(qr > 0, 1 + qr * (qr.log().abs() + lpr.abs()), torch.zeros_like(qr))
        within = torch.where((lpr > -INF)[:, None], (lp - lpr[:, None]).exp(), torch.zeros_like(lp))
        share = torch.where(inside, torch.zeros_like(p), within) * qr[:, None]
        grad = p - target[:, :V] - share
        # (the teacher's rest is 1 less a sum: known to 2^-23 or so of 1)
        mass = mass + share + torch.where(inside, torch.zeros_like(p), within) * 2.0 ** -4
    w = torch.ones(rows, dtype=torch.double, device="cuda") if weight is None else weight.double()
    return (torch.where(w == 0, torch.zeros_like(w), loss * w), torch.where(w[:, None] == 0, torch.zeros_like(grad), grad * (w / T)[:, None]),
            size * w, mass * (w / T)[:, None])


def check_distill(x, ids, teacher, weight=None, rest=False, T=1.0):
    loss, grad = scoring.distill_loss_and_grad(x, ids, teacher, weight=weight, rest=rest, temperature=T)
    want, dwant, size, mass = plain_distill(x, ids, teacher, weight, rest, T)
    near(loss, want, EPS * size + 1e-30)
    near(grad, dwant, EPS * mass + HALF_ULP[x.dtype] * dwant.abs() + (2.0 ** -25 if x.dtype is F16 else 1e-37))
    # the differentiable form
    xg = x.detach().requires_grad_()
    each = scoring.distill_loss(xg, ids, teacher, weight=weight, rest=rest, temperature=T)
    assert torch.equal(each.detach(), loss) or bool(loss.isnan().any())
    up = torch.linspace(0.5, 2.0, x.shape[0], device="cuda")
    (d,) = torch.autograd.grad(each, xg, up)
    near(d, dwant * up.double()[:, None],
         EPS * 2 * mass * up.double()[:, None] + 2 * HALF_ULP[x.dtype] * dwant.abs() * 2 + (2.0 ** -25 if x.dtype is F16 else 1e-37))
    return loss, grad


def teacher_of(g, x, top, T=1.0):
    t = (x.float() + 0.5 * torch.randn(x.shape, generator=g, device="cuda")) / T
    best, ids = t.topk(top, -1)
    return ids, best - t.logsumexp(-1, keepdim=True)


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("rows,V,top", [(1, 2, 1), (5, 7, 3), (9, 33, 20), (3, 257, 128), (80, 512, 8), (7, 4099, 33),
                                        (3, 70001, 100), (2, 151936, 20), (300, 10007, 1), (2, 300001, 128)])
def test_distill(rows, V, top, dtype, rest):
    g = gen(V)
    x = logits_of(g, rows, V, dtype)
    T = 1.0 if rows % 2 else 1.7
    ids, teacher = teacher_of(g, x, top, T)
    weight = torch.rand(rows, generator=g, device="cuda") + 0.1 if rows > 3 else None
    if weight is not None:
        weight[1] = 0
    check_distill(x, ids, teacher, weight, rest, T)


@pytest.mark.parametrize("rest", [False, True])
def test_distill_of_odd_alternatives(rest):
    g = gen(5)
    V = 9001
    x = logits_of(g, 9, V, F32)
    ids, teacher = teacher_of(g, x, 6)
    ids[0, 3:] = -1                                  # fewer of them
    ids[1] = -1                                      # none
    teacher[2, 2:] = -INF                            # no weight on some
    ids[3, 4] = ids[3, 1]                            # the same token twice
    ids[4, 0], ids[4, 1], ids[4, 2] = 0, V - 1, V - 2    # a row's ends
    x[5, ids[5, 1:]] = -INF                          # tokens the student cannot say
    teacher[5, 1:] = -INF
    x[6, :] = -INF
    x[6, ids[6, 0]] = 2.0                            # only one it can
    teacher[6, 1:] = -INF
    teacher[6, 0] = 0.0
    weight = torch.ones(9, device="cuda")
    x[7, 100] = float("nan")                         # a row that is left out
    weight[7] = 0
    loss, grad = check_distill(x, ids, teacher, weight, rest)
    assert loss[1] == 0 and not grad[1].any() and loss[7] == 0 and not grad[7].any()
    assert abs(float(loss[6])) < 1e-6 and not grad[6].any()


@pytest.mark.parametrize("rest", [False, True])
def test_distill_of_rows_without_an_answer(rest):
    g = gen(6)
    V = 4000
    x = logits_of(g, 4, V, F32)
    ids, teacher = teacher_of(g, x, 5)
    x[0, ids[0, 2]] = -INF                           # the teacher's, not the student's
    x[1, :] = -INF
    ids[2, 1] = V                                    # no token
    x[3, 77] = float("nan")
    loss, grad = scoring.distill_loss_and_grad(x, ids, teacher, rest=rest)
    want, dwant, size, mass = plain_distill(x[:2], ids[:2], teacher[:2], None, rest, 1.0)
    assert bool((loss[:2] == INF).all()) and bool((want == INF).all())
    assert bool(grad[:2].isfinite().all())
    near(grad[:1], dwant[:1], EPS * mass[:1] + 1e-7 * dwant[:1].abs() + 1e-37)
    q = torch.zeros(V, device="cuda").scatter_(0, ids[1], teacher[1].exp() if rest else torch.softmax(teacher[1], -1))
    assert torch.allclose(grad[1], -q, rtol=1e-5, atol=0)
    assert bool(loss[2:].isnan().all()) and bool(grad[2:].isnan().any(-1).all())


def test_distill_by_differences():
    """The gradient against differences of the fp64 definition's loss."""
    g = gen(8)
    V, T = 301, 1.3
    x = logits_of(g, 2, V, F32)
    for rest in (False, True):
        ids, teacher = teacher_of(g, x, 12, T)
        grad = scoring.distill_loss_and_grad(x, ids, teacher, rest=rest, temperature=T)[1].double()
        by = torch.randn(2, V, generator=g, device="cuda", dtype=torch.double)
        h = 1e-4
        up, down = (plain_distill(x.double() + s * h * by, ids, teacher, None, rest, T)[0] for s in (1, -1))
        slope = (up - down) / (2 * h)
        # (central differences: h^2 / 6 of the third derivative, below 10 |by|^3 here)
        near((grad * by).sum(-1), slope, EPS * 4 * (grad * by).abs().sum(-1) + 1e-6)


def test_distill_one_alternative_is_cross_entropy():
    g = gen(4)
    x = logits_of(g, 12, 1003, F32)
    t = torch.randint(0, 1003, (12,), generator=g, device="cuda")
    loss = scoring.distill_loss(x, t[:, None], torch.zeros(12, 1, device="cuda"))
    got = scoring.token_logprobs(x, t).logprobs
    assert torch.allclose(loss, -got, rtol=1e-5, atol=1e-5)


def test_distill_views():
    g = gen(3)
    padded = logits_of(g, 8, 1040, BF16)
    x = padded[:, 5:1004]
    ids, teacher = teacher_of(g, x, 9)
    want = scoring.distill_loss_and_grad(x.contiguous(), ids, teacher)
    got = scoring.distill_loss_and_grad(x.unflatten(0, (2, 4)), ids.view(2, 4, 9).int(), teacher.view(2, 4, 9).double())
    assert got[0].shape == (2, 4) and got[1].shape == (2, 4, 999)
    assert torch.allclose(got[0].flatten(), want[0], rtol=1e-5) and torch.allclose(got[1].flatten(0, 1).float(), want[1].float(), rtol=2 ** -7, atol=1e-6)
    wide = ids.repeat(1, 2)[:, :9]
    assert torch.equal(scoring.distill_loss_and_grad(x.contiguous(), wide, teacher)[0], want[0])
    lead = x.contiguous().requires_grad_()
    scoring.distill_loss(lead.unflatten(0, (4, 2)), ids.view(4, 2, 9), teacher.view(4, 2, 9)).sum().backward()
    assert torch.equal(lead.grad, want[1])


def test_graph():
    """Both operators in a captured graph."""
    g = gen(11)
    x = logits_of(g, 16, 5003, F32)
    ids, teacher = teacher_of(g, x, 8)
    tokens = x.argmax(-1)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        scoring.token_logprobs(x, tokens, top=4)
        scoring.distill_loss_and_grad(x, ids, teacher)
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a = scoring.token_logprobs(x, tokens, top=4)
        b = scoring.distill_loss_and_grad(x, ids, teacher)
    x.copy_(logits_of(g, 16, 5003, F32))
    graph.replay()
    for u, v in zip((*a, *b), (*scoring.token_logprobs(x, tokens, top=4), *scoring.distill_loss_and_grad(x, ids, teacher))):
        assert torch.equal(u, v)


def test_refusals():
    x = torch.zeros(4, 300, device="cuda")
    t = torch.zeros(4, dtype=torch.long, device="cuda")
    ids, teacher = torch.zeros(4, 3, dtype=torch.long, device="cuda"), torch.zeros(4, 3, device="cuda")
    for error, call in [
            (TypeError, lambda: scoring.token_logprobs(x.double(), t)),
            (TypeError, lambda: scoring.token_logprobs(x, t.float())),
            (ValueError, lambda: scoring.token_logprobs(x.cpu(), t)),
            (ValueError, lambda: scoring.token_logprobs(x, t.cpu())),
            (ValueError, lambda: scoring.token_logprobs(x, t[:3])),
            (ValueError, lambda: scoring.token_logprobs(x, t, top=129)),
            (ValueError, lambda: scoring.token_logprobs(x[:, :5], t, top=6)),
            (ValueError, lambda: scoring.token_logprobs(x, t, top=-1)),
            (ValueError, lambda: scoring.token_logprobs(x, t, temperature=0.0)),
            (ValueError, lambda: scoring.token_logprobs(x, t, temperature=math.nan)),
            (ValueError, lambda: scoring.token_logprobs(x[:, :0])),
            (ValueError, lambda: scoring.distill_loss(x, ids[:, :0], teacher[:, :0])),
            (ValueError, lambda: scoring.distill_loss(x, ids, teacher[:, :2])),
            (ValueError, lambda: scoring.distill_loss(x, ids, teacher, weight=torch.ones(3, device="cuda"))),
            (ValueError, lambda: scoring.distill_loss(x, ids, teacher.cpu())),
            (ValueError, lambda: scoring.distill_loss(x, ids, teacher, temperature=-1.0)),
            (TypeError, lambda: scoring.distill_loss(x, ids.float(), teacher)),
            (TypeError, lambda: scoring.distill_loss(x, ids, ids)),
            (ValueError, lambda: scoring.distill_loss(torch.empty(1, 1 << 20, device="cuda"), ids[:1], teacher[:1])),
            (ValueError, lambda: scoring.distill_loss(x, ids.repeat(1, 50), teacher.repeat(1, 50)))]:
        with pytest.raises(error):
            call()
    # a failed launch comes back as an error
    assert K.lib().decoder_token_scores(None, 7, 0, 1, 1, None, 0, 1.0, None, None, None, None, None) != 0
