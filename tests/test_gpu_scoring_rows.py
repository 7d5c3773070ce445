"""Scores and distillations whose CTAs take several rows, or many looks at a row,
against their definitions in fp64, with the tolerances of test_gpu_scoring.py.

On 152 SMs: the distillation's clusters of 1, 2, 8 and 16 CTAs are 608, 304, 76
and some 33 at a time, and rows beyond that come second and third; scores of more
than 304 rows take 4096 fp32 (8192 16-bit) elements to a look and list their
largest by 32 buckets of looks.
"""
import pytest
import torch

from paper_2605_30574_gb300 import build as B
from paper_2605_30574_gb300 import decoder as K
from test_gpu_scoring import check_distill, check_scores, gen, logits_of, teacher_of

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


@pytest.fixture(scope="module", autouse=True)
def _built():
    B.build()
    yield
    K.check_device_error()


@pytest.mark.parametrize("rest", [False, True])
@pytest.mark.parametrize("rows,V,top,dtype", [(2000, 1003, 8, F32), (1999, 1003, 128, BF16), (700, 20011, 40, F32), (1500, 20011, 8, BF16),
                                              (1500, 20008, 128, F16), (200, 100003, 128, F32), (250, 100003, 40, BF16),
                                              (100, 151936, 32, F32), (101, 151937, 8, F32)])
def test_distill_row_after_row(rows, V, top, dtype, rest):
    g = gen(rows + V)
    x = logits_of(g, rows, V + 5, dtype)[:, 3:3 + V]        # rows apart, that start anywhere
    T = 1.3
    ids, teacher = teacher_of(g, x, top, T)
    weight = torch.rand(rows, generator=g, device="cuda") + 0.1
    weight[torch.rand(rows, generator=g, device="cuda") < 0.2] = 0
    none = torch.rand(rows, generator=g, device="cuda") < 0.2
    ids[none, top // 2:] = -1
    ids[torch.rand(rows, generator=g, device="cuda") < 0.05] = -1
    # a row's ends, and a token that comes twice (the teacher's weights stay below 1)
    twice = torch.rand(rows, generator=g, device="cuda") < 0.2
    ids[twice, 1] = ids[twice, 0]
    ends = torch.rand(rows, generator=g, device="cuda") < 0.2
    ids[ends, 2], ids[ends, 3], ids[ends, 4] = 0, V - 1, V - 2
    check_distill(x, ids, teacher, weight, rest, T)
    check_distill(x.contiguous(), ids, teacher, None, rest, T)


def raised(g, rows, V, dtype):
    """Rows whose largest elements stand where a selection could lose them."""
    x = torch.randn(rows, V, generator=g, device="cuda")
    up = torch.zeros(rows, V, dtype=torch.bool, device="cuda")
    kinds = [slice(V - 300, V), slice(0, 300), slice(0, V, 4096), slice(4095, V, 4096), slice(V // 2, V // 2 + 200), slice(3, V, 1024 * 4)]
    for i, at in enumerate(kinds):
        up[i::len(kinds) + 2, at] = True
    up[len(kinds)::len(kinds) + 2, :9] = True
    up[len(kinds)::len(kinds) + 2, V - 9:] = True
    return (x + 6.0 * up).to(dtype)


@pytest.mark.parametrize("rows,V,top,dtype", [(320, 151936, 20, F32), (310, 151937, 128, F32), (320, 262147, 64, BF16), (330, 300001, 5, F16),
                                              (1, 1200001, 5, F32), (1, 1200001, 128, F32), (40, 1000003, 64, BF16), (9, 600011, 15, F32)])
def test_scores_of_many_looks(rows, V, top, dtype):
    g = gen(V + top)
    x = raised(g, max(rows, 8), V, dtype)
    tokens = torch.randint(0, V, (x.shape[0],), generator=g, device="cuda")
    tokens[0], tokens[1], tokens[2] = V - 1, 0, -1
    for i in range(0, x.shape[0], rows):
        check_scores(x[i:i + rows], tokens[i:i + rows], top, 0.9)


@pytest.mark.parametrize("order", ["ascending", "descending", "equal", "few values"])
def test_scores_of_many_looks_in_order(order):
    """More candidates than there is room for: every element is looked at again."""
    rows, V = 306, 140003
    x = torch.linspace(-9, 9, V, device="cuda").repeat(rows, 1)
    if order == "descending":
        x = x.flip(-1).contiguous()
    elif order == "equal":
        x = torch.zeros_like(x)
    elif order == "few values":
        x = torch.randint(0, 3, x.shape, generator=gen(3), device="cuda").float()
    check_scores(x, torch.full((rows,), 17, device="cuda"), 100)
