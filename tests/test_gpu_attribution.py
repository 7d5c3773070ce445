"""Attribution of a splice: the decoder's continuation through the differentiable
attention against its decode, and its gradients against plain torch's.

Tolerances.  Both sides round hidden states to bf16 (2^-8) at the same dozen
places per layer and differ in the attention's rounding: as for the decoder's own
tests, logits within 4 x 2^-8 of their row's size, relative in the 2-norm; an
attribution is a sum of products with gradients that pass the same roundings
backward, so the 2-norm over a layer's positions is held to 8 x 2^-8.
"""
import pytest
import torch

from paper_2605_30574_gb300 import attribution as X
from paper_2605_30574_gb300 import build as B
from paper_2605_30574_gb300 import decoder as K
from paper_2605_30574_gb300.decoder import attention as A
from paper_2605_30574_gb300.decoder import scoring
from paper_2605_30574_gb300.model import RandomDecoder, SpliceDecode, tiny_dims
from paper_2605_30574_gb300.synth import workloads as W

pytestmark = pytest.mark.gpu
STEPS, KINDS = 12, (W.BLANK, W.ZERO, W.DIFF_ALGO)


@pytest.fixture(scope="module")
def run():
    B.build()
    dims = tiny_dims()
    model = RandomDecoder(dims, seed=3)
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    prompts = torch.randint(0, dims.vocab, (2, 75), generator=g, device="cuda")
    r = SpliceDecode(model, prompts, KINDS, [W.Seq(p, k, L, 0) for p in (0, 1) for k in range(3) for L in (0, dims.num_layers)],
                     STEPS + 1, 4, 2, filler=64)
    yield r
    K.check_device_error()
    r.close()


def plain_gradients(q, k, v, scale=None):
    """The kernels' output with fp32 torch's gradients.  (The runs' divergence is
    the square of small differences of logits: two forward passes that round
    differently would not tell the same one.)"""
    T, Tk, G = q.shape[0], k.shape[1], q.shape[1] // k.shape[0]
    kh, vh = k.float().repeat_interleave(G, 0), v.float().repeat_interleave(G, 0)
    s = scale * q.float().transpose(0, 1) @ kh.transpose(-1, -2)
    seen = torch.arange(Tk, device=q.device)[None] <= torch.arange(T, device=q.device)[:, None] + (Tk - T)
    plain = (torch.softmax(s.masked_fill(~seen, float("-inf")), -1) @ vh).transpose(0, 1)
    ours = A.attention_forward(q.detach(), k.detach(), v.detach(), scale)[0].float()
    return (plain + (ours - plain).detach()).to(q.dtype).contiguous()


def rel(a, b):
    return float((a.double() - b.double()).norm() / b.double().norm())


def test_continuation_is_the_decodes(run):
    """Teacher-forced logits of a clean and of a spliced cell, step by step."""
    tokens = run.decode(STEPS)
    assert len(run.seqs) == 12
    steps = [run.step(t, tokens[:, t - 1]) for t in range(1, STEPS)]
    for b, cell in enumerate(run.seqs):
        with torch.no_grad():
            got = X.continuation_logits(run.model, tokens[b, :STEPS - 1], *X.spliced_spans(run, cell.prompt, cell.slot, cell.L))
        want = torch.stack([s[b] for s in steps])
        assert rel(got, want) < 4 * 2.0 ** -8, (cell, rel(got, want))


@pytest.mark.parametrize("slot", range(len(KINDS)))
@pytest.mark.parametrize("L", [0, 2])
def test_attribution_against_plain_torch(run, monkeypatch, slot, L):
    tokens = run.decode(STEPS + 1)[1]
    got = X.attribute(run, 0, slot, tokens, L, top=16)
    assert got.divergence.shape == (STEPS,) and bool((got.divergence > 0).all())
    assert not got.attribution[:L].any() and bool(got.attribution[L:].any(-1).all())
    monkeypatch.setattr(A, "attention", plain_gradients)
    want = X.attribute(run, 0, slot, tokens, L, top=16)
    assert rel(got.divergence, want.divergence) < 4 * 2.0 ** -8
    assert rel(got.spliced_logprobs, want.spliced_logprobs) < 4 * 2.0 ** -8
    for l in range(L, run.model.dims.num_layers):
        assert rel(got.attribution[l], want.attribution[l]) < 8 * 2.0 ** -8, l


def test_no_splice_no_divergence(run):
    """A clean span's divergence from itself is rounding, and restoring every
    layer of a splice gives it."""
    tokens = run.decode(STEPS + 1)[0]
    N = run.model.dims.num_layers
    clean = X.attribute(run, 0, 0, tokens, L=N - 1, top=16)
    assert float(clean.divergence.mean()) > 0
    back = X.restored(run, 0, 0, tokens, layer=N - 1, L=N - 1, top=16)
    assert abs(back) < 1e-5


def test_scores_are_the_scorings(run):
    tokens = run.decode(STEPS + 1)[1]
    a = X.attribute(run, 0, 0, tokens, 0, top=16)
    with torch.no_grad():
        logits = X.continuation_logits(run.model, tokens[:-1], list(run.k_clean[0]), list(run.v_clean[0]))
    want = torch.log_softmax(logits.double(), -1).gather(1, tokens[1:, None])[:, 0]
    assert torch.allclose(a.clean_logprobs.double(), want, atol=1e-4)
    assert torch.equal(a.clean_entropy, scoring.token_logprobs(logits).entropy)


def test_command(capsys, tmp_path):
    assert X.main(["--steps", "4", "--prompt-len", "40", "--kinds", "BLANK", "ZERO", "--json", str(tmp_path / "a.json")]) == 0
    said = capsys.readouterr().out
    assert "BLANK: divergence" in said and "ZERO: divergence" in said and (tmp_path / "a.json").exists()
