"""Argument checks of the scoring and attention entry points that need no GPU."""
import pytest
import torch

from paper_2605_30574_gb300 import build as B
from paper_2605_30574_gb300 import decoder as K
from paper_2605_30574_gb300.decoder import attention as A
from paper_2605_30574_gb300.decoder import scoring


@pytest.fixture(scope="module", autouse=True)
def _built():
    B.build()


def test_tensors_of_the_cpu_are_refused():
    x, ids, t = torch.zeros(2, 9), torch.zeros(2, 3, dtype=torch.long), torch.zeros(2, 3)
    for call in (lambda: scoring.token_logprobs(x), lambda: scoring.distill_loss(x, ids, t),
                 lambda: scoring.distill_loss_and_grad(x, ids, t)):
        with pytest.raises(ValueError, match="CUDA"):
            call()
    q, k = torch.zeros(3, 4, 64, dtype=torch.bfloat16), torch.zeros(2, 5, 64, dtype=torch.bfloat16)
    for call in (lambda: A.attention(q, k, k), lambda: A.attention_forward(q, k, k),
                 lambda: A.attention_backward(q, q, k, k, q, torch.zeros(4, 3))):
        with pytest.raises(ValueError, match="CUDA"):
            call()


def test_types_are_refused():
    with pytest.raises(TypeError):
        scoring.token_logprobs([[0.0, 1.0]])
    with pytest.raises(TypeError):
        A.attention(torch.zeros(3, 4, 64), torch.zeros(2, 5, 64), torch.zeros(2, 5, 64))
    with pytest.raises(TypeError):
        A.attention([0], [0], [0])


def test_sizes_that_calls_go_by():
    L = K.lib()
    # as many logits as 8 CTAs' shared memory holds, of 4 and of 2 bytes
    assert L.decoder_distill_vocab(0) * 2 == L.decoder_distill_vocab(1) == L.decoder_distill_vocab(2)
    assert L.decoder_distill_vocab(0) >= 1 << 18
    # per row of queries, padded to whole tiles: two floats and 16 bf16
    assert L.decoder_attention_scratch(1, 1, 1) == 128 * 40
    assert L.decoder_attention_scratch(3, 257, 5) == 3 * 5 * 384 * 40
    # bad shapes come back as errors before anything is launched
    assert L.decoder_token_scores(None, 0, 0, 1, 4, None, 5, 1.0, None, None, None, None, None) != 0
    assert L.decoder_token_scores(None, 0, 0, 0, 4, None, 1, 1.0, None, None, None, None, None) != 0
    assert L.decoder_distill(None, 0, 0, 1, 4, None, None, 0, None, 0, 1.0, None, None, None) != 0
    assert L.decoder_distill(None, 0, 0, 1, 4, None, None, 129, None, 0, 1.0, None, None, None) != 0
    assert L.decoder_attention(*[None] * 6, 1, 4, 4, 3, 2, 64, 1.0, None) != 0
    assert L.decoder_attention_backward(*[None] * 11, 1, 4, 4, 2, 0, 64, 1.0, None) != 0


def test_strides_of_views():
    """(row, head, batch) strides, the heads first for k and v."""
    q, k = torch.empty(2, 5, 4, 64, dtype=torch.bfloat16), torch.empty(2, 2, 7, 64, dtype=torch.bfloat16)
    ts, ptrs, strides = A._operands(q, k, k)
    assert strides is None and ptrs == [q.data_ptr(), k.data_ptr(), k.data_ptr()]
    flip = q.transpose(1, 2).contiguous().transpose(1, 2)
    _, _, strides = A._operands(flip, k, k)
    assert list(strides) == [64, 320, 1280, 64, 448, 896, 64, 448, 896]
    _, _, strides = A._operands(flip[0], k[0], k[0])
    assert list(strides)[:2] + list(strides)[3:5] == [64, 320, 64, 448]
    # what the kernels cannot read is copied: an odd start, an odd stride, one over a size of more than one
    wide = torch.empty(2, 5, 4, 65, dtype=torch.bfloat16)
    for t in (wide[..., 1:], wide[..., :64], q[:1].expand(2, -1, -1, -1)):
        ts, ptrs, strides = A._operands(t, k, k)
        assert ts[0].is_contiguous() and ptrs[0] == ts[0].data_ptr() and ts[0].data_ptr() != t.data_ptr()
        assert torch.equal(ts[0], t) or bool(t.isnan().any())
