"""Attribution at the ends of its range."""
import pytest
import torch

from paper_2605_30574_gb300 import attribution as X
from paper_2605_30574_gb300 import build as B
from paper_2605_30574_gb300 import decoder as K
from paper_2605_30574_gb300.model import RandomDecoder, SpliceDecode, tiny_dims
from paper_2605_30574_gb300.synth import workloads as W

pytestmark = pytest.mark.gpu


def test_nothing_spliced():
    """L past the last layer is the clean run: no divergence, nothing attributed."""
    B.build()
    dims = tiny_dims()
    model = RandomDecoder(dims, seed=3)
    prompts = torch.arange(40, device="cuda")[None] % dims.vocab
    run = SpliceDecode(model, prompts, [W.BLANK], [W.Seq(0, 0, dims.num_layers, 0)], 7, 4, 2, filler=64)
    tokens = run.decode(7)[0]
    a = X.attribute(run, 0, 0, tokens, L=dims.num_layers, top=16)
    assert a.attribution.shape == (dims.num_layers, 40) and not a.attribution.any()
    assert float(a.divergence.abs().max()) < 1e-6
    assert torch.equal(a.clean_logprobs, a.spliced_logprobs) and torch.equal(a.clean_entropy, a.spliced_entropy)
    K.check_device_error()
    run.close()
