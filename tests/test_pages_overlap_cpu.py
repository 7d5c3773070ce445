"""Where the rows that are loaded go: keys and values that have a place in common are
refused, those that lie between each other are not."""
import random

import pytest
import torch

from paper_2605_30574_gb300.decoder import pages as P

from page_util import BF
from test_pages_cpu import OnCpu, _built, launched, where  # noqa: F401

SHAPE = (2, 2, 64)


def of(strides, at, size=4096):
    return torch.zeros(size, dtype=BF).as_strided(SHAPE, strides, at)


@pytest.mark.parametrize("k,v", [
    # heads 0 to 1 and 1 to 2 of a joined row; rows 0 to 1 and 1 to 2; a part of a row; between, by part
    (((512, 64, 1), 0), ((512, 64, 1), 64)), (((128, 64, 1), 0), ((128, 64, 1), 128)), (((512, 64, 1), 0), ((512, 64, 1), 32)),
    (((512, 128, 1), 0), ((512, 128, 1), 72)), (((512, 64, 1), 64), ((512, 64, 1), 0)), (((512, 64, 1), 0), ((512, 64, 1), 576)),
    # the heads apart by more than the rows; elements apart; other strides
    (((64, 512, 1), 0), ((64, 512, 1), 64)), (((512, 128, 2), 0), ((512, 128, 2), 2)), (((512, 128, 2), 0), ((512, 128, 2), 130)),
    (((512, 64, 1), 0), ((1024, 64, 1), 512)), (((128, 64, 1), 0), ((64, 128, 1), 0))])
def test_places_in_common(launched, k, v):  # noqa: F811
    flat = torch.zeros(4096, dtype=BF)
    for a, b in ((k, v), (v, k)):
        with pytest.raises(ValueError, match="same place"):
            P.load_pages(OnCpu(), 0, flat.as_strided(SHAPE, *a), flat.as_strided(SHAPE, *b), *where())
    assert not launched


@pytest.mark.parametrize("k,v", [
    # a joined row's; behind each other; each row's keys, then its values, rows apart; the other way round
    (((512, 64, 1), 0), ((512, 64, 1), 128)), (((128, 64, 1), 0), ((128, 64, 1), 256)), (((256, 64, 1), 0), ((256, 64, 1), 128)),
    (((512, 64, 1), 128), ((512, 64, 1), 0)), (((512, 128, 1), 0), ((512, 128, 1), 64)), (((512, 128, 1), 64), ((512, 128, 1), 0)),
    (((64, 512, 1), 0), ((64, 512, 1), 128)), (((512, 128, 2), 0), ((512, 128, 2), 1)), (((512, 64, 1), 0), ((128, 64, 1), 1024)),
    (((512, 64, 1), 0), ((512, 64, 1), 384))])
def test_places_between_each_other(launched, k, v):  # noqa: F811
    flat = torch.zeros(4096, dtype=BF)
    for a, b in ((k, v), (v, k)):
        P.load_pages(OnCpu(), 0, flat.as_strided(SHAPE, *a), flat.as_strided(SHAPE, *b), *where())
    assert len(launched) == 2


@pytest.mark.parametrize("heads,rows,strides", [(1, 1, (0, 0, 1)), (1, 2, (64, 0, 1)), (2, 1, (0, 64, 1)), (1, 1, (8, 8, 1))])
def test_strides_of_one(launched, heads, rows, strides):  # noqa: F811
    """Strides of dimensions of one say nothing of where rows are."""
    flat, cache, w = torch.zeros(4096, dtype=BF), OnCpu(heads=heads), where(rows)
    k, v, apart = (flat.as_strided((rows, heads, 64), strides, at) for at in (0, 32, 64 * rows * heads))
    with pytest.raises(ValueError, match="same place"):
        P.load_pages(cache, 0, k, v, *w)
    P.load_pages(cache, 0, k, apart, *w)
    assert len(launched) == 1


def test_by_all_places():
    """Of any equal strides: as the places say, one by one."""
    rng = random.Random(0)
    flat, seen = torch.zeros(4000, dtype=BF), set()
    while len(seen) < 2 or rng.random() < 0.998:
        shape = [rng.randint(1, 4) for _ in range(3)]
        strides, extent = [0] * 3, 1
        for i in rng.sample(range(3), 3):
            strides[i] = extent + rng.choice((0, 0, 1, 5, 20))
            extent = (shape[i] - 1) * strides[i] + extent if shape[i] > 1 else extent
        k, v = (flat.as_strided(shape, strides, rng.randint(0, 3 * extent)) for _ in range(2))
        places = [{x.storage_offset() + sum(i * s for i, s in zip(at, strides)) for at in torch.cartesian_prod(*map(torch.arange, shape)).tolist()}
                  for x in (k, v)]
        apart = not places[0] & places[1]
        assert P._apart(k, v) == apart, (shape, strides, k.storage_offset(), v.storage_offset())
        seen.add(apart)
