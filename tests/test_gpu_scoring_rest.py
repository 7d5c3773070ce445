"""The distillation's rest (all tokens but the teacher's, as one outcome) against
its definition in fp64, where the others lie far below or above the teacher's.

Tolerances.  As for the other scores, log probabilities and weights are within
2^-19 of their size.  What the teacher leaves of 1 is 1 less a sum of up to 128
exponentials, each within 2^-23 of itself: known to 2^-22, which the loss has
times |log q_rest - log p_rest|, and the others' gradients times their share of
p_rest.
"""
import pytest
import torch

from paper_2605_30574_gb300 import build as B
from paper_2605_30574_gb300 import decoder as K
from paper_2605_30574_gb300.decoder import scoring

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
HALF_ULP = {F32: 2.0 ** -24, BF16: 2.0 ** -8, F16: 2.0 ** -11}
EPS, KNOWN = 2.0 ** -19, 2.0 ** -22
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


def definition(x, ids, teacher, T, known=None):
    """Loss and gradient with the rest counted, in fp64, and their bounds; `known`
    is how well the rows' rests are."""
    known = torch.full(x.shape[:1], KNOWN, device="cuda", dtype=torch.double) if known is None else known
    lp, t = torch.log_softmax(x.double() / T, -1), teacher.double()
    q, inside = t.exp(), torch.zeros(x.shape, dtype=torch.bool, device="cuda").scatter_(1, ids, True)
    rest = (1 - q.sum(-1)).clamp(min=0)
    lpr = torch.logsumexp(lp.masked_fill(inside, -INF), -1)
    zero = torch.zeros_like(rest)
    at = lp.gather(1, ids)
    loss = torch.where(q > 0, q * (t - at), torch.zeros_like(q)).sum(-1) + torch.where(rest > 0, rest * (rest.log() - lpr), zero)
    size = torch.where(q > 0, q * (1 + t.abs() + at.abs()), torch.zeros_like(q)).sum(-1)
    apart = torch.where(rest > 0, 1 + rest.log().abs() + lpr.abs(), zero)
    share = torch.where((lpr > -INF)[:, None], (lp - lpr[:, None]).exp(), torch.zeros_like(lp)).masked_fill(inside, 0)
    target = torch.zeros_like(lp).scatter_add_(1, ids, q) + share * rest[:, None]
    return loss, (lp.exp() - target) / T, EPS * (size + rest * apart) + known * apart, (EPS * (lp.exp() + target) + known[:, None] * share) / T


def near(got, want, bound):
    got = got.double()
    assert torch.equal(got.isnan(), want.isnan())
    off = ((got - want).abs() / bound).masked_fill((got == want) | got.isnan(), 0.0)
    assert float(off.max()) <= 1.0, float(off.max())


def check(x, ids, teacher, T=1.0):
    loss, grad = scoring.distill_loss_and_grad(x, ids, teacher, rest=True, temperature=T)
    want, dwant, off, doff = definition(x, ids, teacher, T)
    near(loss, want, off + 1e-30)
    near(grad, dwant, doff + HALF_ULP[x.dtype] * dwant.abs() + (2.0 ** -25 if x.dtype is F16 else 1e-37))
    leaf = x.detach().requires_grad_()
    each = scoring.distill_loss(leaf, ids, teacher, rest=True, temperature=T)
    assert torch.equal(each.detach(), loss)
    (again,) = torch.autograd.grad(each.sum(), leaf)
    assert torch.equal(again, grad)
    return loss, grad


@pytest.mark.parametrize("T", [1.0, 0.1])
@pytest.mark.parametrize("gap", [30, 60, 86, 88, 100, 300, 2000, -60, -100, -2000])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("V,top", [(4, 2), (1003, 40), (60011, 128)])
def test_others_far_from_the_teachers(V, top, dtype, gap, T):
    """The others' logits `gap` nats below the teacher's, by the temperature."""
    g = gen(V + top)
    x = torch.randn(6, V, generator=g, device="cuda")
    ids = torch.rand(6, V, generator=g, device="cuda").topk(top, -1).indices
    x -= gap
    x.scatter_(1, ids, torch.randn(6, top, generator=g, device="cuda"))
    x = (x * T).to(dtype)
    left = torch.tensor([0.3, 0.2, 1e-2, 1e-4, 0.999, 0.5], device="cuda")
    teacher = torch.log_softmax(torch.randn(6, top, generator=g, device="cuda"), -1) + torch.log1p(-left)[:, None]
    loss, grad = check(x, ids, teacher, T)
    assert bool(loss.isfinite().all())
    # what the others gain, the teacher's lose
    off = (HALF_ULP[dtype] + EPS) * grad.double().abs().sum(-1) + KNOWN / T + (V * 2.0 ** -25 if dtype is F16 else 0)
    assert bool((grad.double().sum(-1).abs() <= off + EPS / T).all())


def test_two_alternatives_and_two_others_a_long_way_off():
    x = torch.tensor([[0.0, -1.0, -89.0, -90.0]], device="cuda")
    ids = torch.tensor([[0, 1]], device="cuda")
    teacher = torch.tensor([[0.5, 0.3]], device="cuda").log()
    loss, grad = check(x, ids, teacher)
    assert 17 < float(loss) < 19 and abs(float(grad[0, 2:].sum()) + 0.2) < 1e-6


# ---- what rounding leaves of 1 ----
#
# K log probabilities that are a whole distribution are each off by some units of
# 2^-24 of themselves and of their sum's logarithm; e^ of them by 2^-23 of itself.
# Up to 4 x 2^-23 sum q (1 + |log q|) in all is no weight.

def slack(teacher):
    t = teacher.double()
    return 2.0 ** -21 * torch.where(t > -INF, t.exp() * (1 + t.abs()), torch.zeros_like(t)).sum(-1)


@pytest.mark.parametrize("T", [1.0, 0.6])
@pytest.mark.parametrize("others", ["none", "-inf", "lowest"])
@pytest.mark.parametrize("top", [2, 20, 128])
def test_alternatives_that_are_all_a_row_can_say(top, others, T):
    """A row against itself, the other tokens missing or masked."""
    g, rows = gen(top), 400
    V = top if others == "none" else 1003
    x = torch.full((rows, V), -INF if others == "-inf" else torch.finfo(F32).min, device="cuda")
    ids = torch.rand(rows, V, generator=g, device="cuda").topk(top, -1).indices
    x.scatter_(1, ids, 2 * torch.randn(rows, top, generator=g, device="cuda"))
    own = scoring.token_logprobs(x, top=top, temperature=T)
    for at, teacher in ((own.top_ids, own.top_logprobs), (ids, torch.log_softmax(x.gather(1, ids) / T, -1))):
        assert bool(((1 - teacher.exp().sum(-1)) != 0).any())
        loss, grad = scoring.distill_loss_and_grad(x, at, teacher, rest=True, temperature=T)
        q = teacher.double().exp()
        assert bool((loss.double().abs() <= EPS * (q * (1 + 2 * teacher.double().abs())).sum(-1)).all())
        inside = grad.gather(1, at).double()
        assert bool((inside.abs() <= 2 * EPS * q / T).all())
        assert not grad.scatter(1, at, 0.0).any()
        assert torch.equal(scoring.distill_loss(x, at, teacher, rest=True, temperature=T), loss)


@pytest.mark.parametrize("gap", [0, 20, 100, 1000])
def test_alternatives_that_are_all_a_teacher_says(gap):
    """The student can say others, the teacher none but by rounding."""
    g, V, top = gen(gap), 701, 30
    x = torch.randn(200, V, generator=g, device="cuda") - gap
    ids = torch.rand(200, V, generator=g, device="cuda").topk(top, -1).indices
    x.scatter_(1, ids, torch.randn(200, top, generator=g, device="cuda"))
    teacher = torch.log_softmax(2 * torch.randn(200, top, generator=g, device="cuda"), -1)
    loss, grad = scoring.distill_loss_and_grad(x, ids, teacher, rest=True)
    want, dwant, off, doff = definition(x, ids, teacher, 1.0, slack(teacher))
    near(loss, want, off)
    near(grad, dwant, doff + HALF_ULP[F32] * dwant.abs() + 1e-37)
    # and what is left by rounding is nothing
    share = -grad.scatter(1, ids, 0.0).double()
    assert bool((share <= 0).all())


def test_a_rest_of_weight_is_kept():
    """Of 1e-5 on: +inf where no other token can be said, the definition else."""
    g, V, top = gen(1), 501, 12
    x = torch.randn(3, V, generator=g, device="cuda")
    ids = torch.rand(3, V, generator=g, device="cuda").topk(top, -1).indices
    teacher = torch.log_softmax(torch.randn(3, top, generator=g, device="cuda"), -1) + torch.log1p(torch.tensor([[-1e-5]], device="cuda"))
    check(x, ids, teacher)
    none = torch.full_like(x, -INF).scatter(1, ids, x.gather(1, ids))
    loss, grad = scoring.distill_loss_and_grad(none, ids, teacher, rest=True)
    assert bool((loss == INF).all()) and bool(grad.isfinite().all())


@pytest.mark.parametrize("T", [1.5, 1.0])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_small_divergences(dtype, T):
    """Of rows that the teacher has all but right: the loss is a small difference
    of log probabilities.  The row's sums are rounded (2^-24) independently from row
    to row; what all rows share may not come to more."""
    g, rows, V = gen(21), 1000, 20011
    x = torch.randn(rows, V, generator=g, device="cuda") * (1 + 2 * torch.rand(rows, 1, generator=g, device="cuda"))
    x.scatter_add_(1, torch.randint(0, V, (rows, 4), generator=g, device="cuda"), 4 + 8 * torch.rand(rows, 4, generator=g, device="cuda"))
    t = (x + 0.1 * torch.randn(rows, V, generator=g, device="cuda")) / T
    teacher, ids = t.topk(40, -1)
    teacher = teacher - t.logsumexp(-1, keepdim=True)
    x = x.to(dtype)
    loss = scoring.distill_loss(x, ids, teacher, rest=True, temperature=T)
    want = definition(x, ids, teacher, T)[0]
    off = (loss.double() - want).square().mean().sqrt()
    assert float(off) <= 2.0 ** -24, float(off)


@pytest.mark.parametrize("gap", [20, 40, 44, 60])
def test_shares_of_the_rest_over_many_nats(gap):
    """Each other token's share of what the rest gives, down to e^-50 of the
    largest: its exponent, of up to 50, is rounded by 2^-24 of itself twice."""
    V = 701
    x = torch.linspace(0, -50, V, device="cuda")[None] - gap
    ids = torch.tensor([[5, 350, 700]], device="cuda")
    x[0, ids[0]] = torch.tensor([0.0, -1.0, -2.0], device="cuda")
    teacher = torch.tensor([[0.4, 0.2, 0.1]], device="cuda").log()
    _, grad = scoring.distill_loss_and_grad(x, ids, teacher, rest=True)
    _, want, _, _ = definition(x, ids, teacher, 1.0)
    assert bool(((grad.double() - want).abs() <= (EPS + 100 * 2.0 ** -24) * want.abs() + 2 * EPS * torch.softmax(x.double(), -1)).all())
