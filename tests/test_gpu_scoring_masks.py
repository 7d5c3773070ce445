"""Divergences where logits are masked, by -inf or by their type's lowest value,
and temperatures at and past the ends of their range.

Tolerance: 2^-19 of the loss' terms, as tests/test_gpu_scoring.py derives it; a
term that is past the range of fp32 is an infinity.
"""
import pytest
import torch

from paper_2605_30574_gb300 import build as B
from paper_2605_30574_gb300 import decoder as K
from paper_2605_30574_gb300.decoder import scoring

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
EPS, INF = 2.0 ** -19, float("inf")


@pytest.fixture(scope="module", autouse=True)
def _built():
    B.build()
    yield
    K.check_device_error()


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("top", [5, 33, 40, 64, 65, 128])
def test_tokens_that_cannot_be_said_among_many(top, rest):
    """One alternative of -inf among others: the loss is +inf wherever it stands."""
    V = 3001
    g = torch.Generator(device="cuda")
    g.manual_seed(top)
    x = torch.randn(top + 1, V, generator=g, device="cuda")
    ids = torch.rand(top + 1, V, generator=g, device="cuda").topk(top, -1).indices
    teacher = torch.log_softmax(torch.randn(top + 1, top, generator=g, device="cuda"), -1) - 0.1
    at = torch.arange(top, device="cuda")
    x[at, ids[at, at]] = -INF
    loss, grad = scoring.distill_loss_and_grad(x, ids, teacher, rest=rest)
    assert bool((loss[:top] == INF).all()), loss
    assert bool(loss[top].isfinite()) and bool(grad.isfinite().all())
    assert torch.equal(scoring.distill_loss(x, ids, teacher, rest=rest), loss)


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("T", [1.0, 0.6, 3.0])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_a_teachers_token_of_the_lowest_logit(dtype, T, rest):
    V, low = 1003, torch.finfo(dtype).min
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    x = torch.randn(5, V, generator=g, device="cuda").to(dtype)
    ids = torch.tensor([[3, 1000, 77]], device="cuda").repeat(5, 1)
    x[0, 77] = low                       # of weight 0.1 to the teacher
    x[1, [3, 1000]] = low                # of 0.7
    x[2] = low                           # all alike
    x[3, :] = low
    x[3, 500] = 1.0                      # one token that can be said, not the teacher's
    x[4, 3], x[4, 77] = -low, low        # further apart than the type reaches
    teacher = torch.tensor([[0.5, 0.2, 0.1]], device="cuda").log().repeat(5, 1)
    loss, grad = scoring.distill_loss_and_grad(x, ids, teacher, rest=rest, temperature=T)
    z = x.double() / T
    lp, t = torch.log_softmax(z, -1), teacher.double()
    t = t if rest else torch.log_softmax(t, -1)
    q, at = t.exp(), lp.gather(1, ids)
    want, size = (q * (t - at)).sum(-1), (q * (1 + t.abs() + at.abs())).sum(-1)
    target = torch.zeros_like(lp).scatter_(1, ids, q)
    if rest:
        left = 1 - q.sum(-1)
        lpr = torch.logsumexp(lp.scatter(1, ids, -INF), -1)
        want, size = want + left * (left.log() - lpr), size + 1 + left * (left.log().abs() + lpr.abs())
        # (from the logits: log probabilities of 1e38 have no digits for the others' own)
        target += torch.softmax(z.scatter(1, ids, -INF), -1) * left[:, None]
    top = torch.finfo(F32).max
    assert not loss.isnan().any()
    assert bool((torch.where(want > top, loss == INF, (loss.double() - want).abs() <= EPS * size)).all()), (loss, want)
    dwant = (lp.exp() - target) / T
    ulp = {F32: 2.0 ** -24, BF16: 2.0 ** -8, F16: 2.0 ** -11}[dtype]
    assert bool(((grad.double() - dwant).abs() <= (EPS * (lp.exp() + target) + 2.0 ** -22) / T + ulp * dwant.abs() + 2.0 ** -25).all())


@pytest.mark.parametrize("T", [2.0 ** -127, 1e-30, 1e30, 2.0 ** 120])
def test_temperatures_at_the_ends(T):
    V = 1003
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    x = torch.randn(4, V, generator=g, device="cuda")
    x[1:, torch.rand(V, generator=g, device="cuda") < 0.5] = -INF
    x[2, 7:300] = torch.finfo(F32).min
    x[3] *= T ** 0.5
    ids = x.topk(3, -1).indices
    teacher = torch.tensor([[0.5, 0.2, 0.1]], device="cuda").log().repeat(4, 1)
    got = scoring.token_logprobs(x, ids[:, 0], top=5, temperature=T)
    loss, grad = scoring.distill_loss_and_grad(x, ids, teacher, temperature=T)
    z = x.double() / T
    lp = torch.log_softmax(z, -1)
    p = lp.exp()
    assert bool(((got.logprobs.double() - lp.gather(1, ids[:, :1])[:, 0]).abs() <= EPS * 40).all())
    H = -torch.where(p > 0, p * lp, torch.zeros_like(p)).sum(-1)
    assert bool(((got.entropy.double() - H).abs() <= EPS * 40).all())
    t = torch.log_softmax(teacher.double(), -1)
    q, at = t.exp(), lp.gather(1, ids)
    want, size = (q * (t - at)).sum(-1), (q * (1 + t.abs() + at.abs())).sum(-1)
    assert bool((torch.where(want > torch.finfo(F32).max, loss == INF, (loss.double() - want).abs() <= EPS * size)).all()), (loss, want)
    target = torch.zeros_like(lp).scatter_(1, ids, q)
    assert bool(((grad.double() - (p - target) / T).abs() <= EPS * (p + target) / T + 1e-37).all())


def test_temperatures_past_the_ends_are_refused():
    x = torch.zeros(2, 9, device="cuda")
    ids, teacher = torch.zeros(2, 1, dtype=torch.long, device="cuda"), torch.zeros(2, 1, device="cuda")
    for T in (3e-39, 1e-45, 1e-310, 2e36, 1e45, 1e300, INF):
        for call in (lambda: scoring.token_logprobs(x, temperature=T), lambda: scoring.distill_loss(x, ids, teacher, temperature=T),
                     lambda: scoring.distill_loss_and_grad(x, ids, teacher, temperature=T)):
            with pytest.raises(ValueError, match="temperature"):
                call()


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_rows_with_infinity_or_nan(dtype, rest):
    """Their loss and gradient are NaN, whatever the teacher's tokens are."""
    V, low = 517, torch.finfo(dtype).min
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    x = torch.randn(8, V, generator=g, device="cuda").to(dtype)
    ids = torch.tensor([[3, 500, 77]], device="cuda").repeat(8, 1)
    teacher = torch.tensor([[0.5, 0.2, 0.1]], device="cuda").log().repeat(8, 1)
    for r, bad in enumerate((INF, float("nan"))):
        x[4 * r:4 * r + 4, 100] = bad
        x[4 * r + 1, ids[0]] = -INF
        x[4 * r + 2, ids[0]] = low
        x[4 * r + 3, :] = -INF
        x[4 * r + 3, 100] = bad
    loss, grad = scoring.distill_loss_and_grad(x, ids, teacher, rest=rest, temperature=0.6)
    assert bool(loss.isnan().all()), loss
    assert bool(grad.isnan().any(-1).all())
    assert bool(scoring.distill_loss(x, ids, teacher, rest=rest, temperature=0.6).isnan().all())


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_rows_without_alternatives(dtype, rest):
    """No loss and no gradient, whatever else they hold."""
    x = torch.randn(7, 517, device="cuda").to(dtype)
    x[1, 5], x[2, 516], x[3, 0] = float("nan"), INF, -INF
    x[4], x[5], x[6] = -INF, float("nan"), torch.finfo(dtype).min
    teacher = torch.full((7, 40), -3.0, device="cuda")
    cases = [(torch.full((7, 40), -1, device="cuda"), teacher)]
    if not rest:
        cases.append((torch.arange(40, device="cuda").repeat(7, 1), torch.full_like(teacher, -INF)))
    for ids, t in cases:
        for y in (x, torch.cat([x, x], -1)[:, 3:520], x[:, 2:3]):
            if ids.max() < y.shape[1]:
                loss, grad = scoring.distill_loss_and_grad(y, ids, t, rest=rest)
                assert not loss.any() and not grad.any(), loss
                assert not scoring.distill_loss(y, ids, t, rest=rest).any()


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_an_id_past_the_vocabulary_makes_its_row_nan(dtype, rest):
    x = torch.randn(4, 517, device="cuda").to(dtype)
    x[2:] = -INF
    ids = torch.tensor([[517], [5], [600], [5]], device="cuda")
    loss, grad = scoring.distill_loss_and_grad(x, ids, torch.zeros(4, 1, device="cuda"), rest=rest)
    assert loss.isnan().tolist() == [True, False, True, False]
    assert grad.isnan().all(-1).tolist() == [True, False, True, False] and not grad[[1, 3]].isnan().any()


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("top", [5, 20, 64])
def test_divergences_at_the_end_of_the_range(top, rest):
    """All that the teacher says masked by the lowest value: as much as a logit
    can be, or +inf."""
    g = torch.Generator(device="cuda")
    g.manual_seed(top)
    low = torch.finfo(F32).min
    x = torch.randn(400, 517, generator=g, device="cuda")
    ids = torch.rand(400, 517, generator=g, device="cuda").topk(top, -1).indices
    x.scatter_(1, ids, low)
    teacher = torch.log_softmax(torch.randn(400, top, generator=g, device="cuda"), -1)
    loss, grad = scoring.distill_loss_and_grad(x, ids, teacher, rest=rest)
    assert bool((loss >= -low * (1 - 1e-6)).all()), loss
    assert bool(grad.isfinite().all())
