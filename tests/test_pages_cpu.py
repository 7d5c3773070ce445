"""Arguments of the paged cache's calls that are refused, and what the kernels are
handed, without a GPU: the cache's tensors are the CPU's, and no launch is made."""
import random

import pytest
import torch
from torch.fx.experimental.proxy_tensor import make_fx

from paper_2605_30574_gb300 import build as B
from paper_2605_30574_gb300 import decoder as K
from paper_2605_30574_gb300.decoder import pages as P

from page_util import BF, held, ints, nibble_place


class OnCpu(P.PageCache):
    """As a cache that a device holds."""

    def __init__(self, layers=2, pages=5, heads=2, d=64, page=16):
        one = (layers, pages, 2, heads, page)
        self._hold(*(torch.zeros(s, dtype=torch.uint8) for s in ((*one, d // 2), (*one, d // 32), (layers, pages, heads, page, 2))))
        self._scratch = 64


@pytest.fixture(scope="module", autouse=True)
def _built():
    B.build()


@pytest.fixture
def launched(monkeypatch):
    calls = []
    monkeypatch.setattr(P, "_current_device", lambda: None)
    monkeypatch.setattr(P, "_launch", lambda *a: calls.append(a))
    return calls


def where(B_=2, W=2, device="cpu"):
    return [torch.zeros(B_, W, dtype=torch.int32), ints(*range(B_ + 1), device="cpu"), torch.ones(B_, dtype=torch.int32)]


def calls(cache, w, k=None, v=None, q=None):
    k = torch.zeros(2, 2, 64, dtype=BF) if k is None else k
    v = torch.zeros(2, 2, 64, dtype=BF) if v is None else v
    q = torch.zeros(2, 4, 64, dtype=BF) if q is None else q
    return (lambda: P.store_pages(cache, 0, k, v, *w), lambda: P.load_pages(cache, 0, k, v, *w), lambda: P.page_attention(cache, 0, q, *w))


def test_a_cache_is_checked():
    u8 = dict(dtype=torch.uint8)
    good = [torch.zeros(1, 2, 2, 3, 16, 32, **u8), torch.zeros(1, 2, 2, 3, 16, 2, **u8), torch.zeros(1, 2, 3, 16, 2, **u8)]
    with pytest.raises(ValueError, match="CUDA"):
        P.PageCache(*good)
    with pytest.raises(TypeError, match="ratios"):
        # (the first one's device is looked at before the second's type)
        fake = type("T", (), {})
        P.PageCache(*_as_cuda(good[0]), good[1].int(), good[2])
    for d, page in ((96, 16), (64, 48), (64, 512)):
        with pytest.raises(ValueError, match="64, 128 or 256"):
            P.PageCache.empty(1, 1, 1, d, page)


def _as_cuda(t):
    class Cuda(torch.Tensor):
        @property
        def device(self):
            return torch.device("cuda", 0)
    return [t.as_subclass(Cuda)]


def test_what_calls_take(launched):
    cache = OnCpu()
    for call in calls(cache, where()):
        call()
    assert [c[0] for c in launched] == ["decoder_page_rows", "decoder_page_rows", "decoder_page_attention"]
    assert [c[1] for c in launched[:2]] == [0, 1]
    P.page_attention(cache, 1, torch.zeros(2, 4, 64, dtype=BF), *where())
    assert launched[0][2:4] == launched[2][1:3] == (cache._at, 0) and launched[3][1:3] == (cache._at, 1)
    d = cache._described
    assert (d.codes, d.ratios, d.exponents) == tuple(t.data_ptr() for t in (cache.codes, cache.ratios, cache.exponents))
    assert (d.layers, d.pages, d.heads, d.head_dim, d.log_page) == (2, 5, 2, 64, 4)


def test_a_cache_that_was_given_back(launched):
    cache = OnCpu()
    cache.ratios.untyped_storage().resize_(0)
    for call in calls(cache, where()):
        with pytest.raises(ValueError, match="no memory"):
            call()
    with pytest.raises(ValueError, match="no memory"):
        P.copy_pages(cache, [0], [1])
    assert not launched


@pytest.mark.parametrize("name", ["codes", "ratios", "exponents"])
def test_a_cache_whose_tensors_are_others(launched, name):
    cache = OnCpu()
    setattr(cache, name, getattr(cache, name).clone())
    for call in calls(cache, where()) + (lambda: P.copy_pages(cache, [0], [1]),):
        with pytest.raises(ValueError, match="other memory"):
            call()
    assert not launched


def test_tables_of_too_many(launched):
    wide, many = (torch.empty(n, dtype=torch.int32, device="meta") for n in (1 << 31, 1 << 30))
    cache = OnCpu()

    class There(torch.Tensor):
        """As a tensor that has memory."""
        device = cache.device

        def data_ptr(self):
            return 16
    for table, starts, lengths in ((wide.view(1, -1), 2, 1), (many.view(-1, 1), (1 << 30) + 1, 1 << 30)):
        w = [t.as_subclass(There) for t in (table, *(torch.empty(n, dtype=torch.int32, device="meta") for n in (starts, lengths)))]
        for call in calls(cache, w):
            with pytest.raises(ValueError, match="fewer than 2"):
                call()
    assert not launched


def test_nothing_to_do(launched):
    cache = OnCpu()
    none = torch.zeros(0, 2, 64, dtype=BF)
    for call in calls(cache, where(0, 0)) + calls(cache, where(), none, none, torch.zeros(0, 4, 64, dtype=BF)):
        call()
    assert not launched


@pytest.mark.parametrize("i,bad,match", [
    (0, torch.zeros(2, 2), "table"), (0, torch.zeros(2, 2, dtype=torch.int64), "table"), (0, torch.zeros(4, dtype=torch.int32), "table"),
    (0, torch.zeros(2, 0, dtype=torch.int32), "no pages"), (0, torch.zeros(2, 4, dtype=torch.int32)[:, ::2], "table"),
    (1, torch.zeros(2, dtype=torch.int32), "starts"), (1, torch.zeros(3), "starts"), (2, torch.zeros(3, dtype=torch.int32), "lengths"),
    (2, None, "lengths"), (2, torch.zeros(2, dtype=torch.int64), "lengths"), (1, torch._neg_view(torch.zeros(3, dtype=torch.int32)), "starts"),
    (2, torch._efficientzerotensor((2,), dtype=torch.int32), "no memory")])
def test_tables_that_are_refused(launched, i, bad, match):
    w = where()
    w[i] = bad
    for call in calls(OnCpu(), w):
        with pytest.raises((TypeError, ValueError), match=match):
            call()
    assert not launched


def test_tensors_that_are_refused(launched):
    cache, w = OnCpu(), where()
    z = lambda *s, dtype=BF: torch.zeros(*s, dtype=dtype)  # noqa: E731
    for bad in (z(2, 2, 64, dtype=torch.float16), z(2, 2, 32), z(2, 3, 64), z(3, 2, 64), z(2, 128), [0]):
        for call in calls(cache, w, v=bad)[:2]:
            with pytest.raises((TypeError, ValueError), match="v must be"):
                call()
    for bad, match in ((z(2, 4, 64, dtype=torch.float32), "q must be a bf16"), (z(2, 4, 128), "q must be"), (z(4, 64), "q must be"),
                       (z(2, 3, 64), "multiple"), (z(2, 0, 64), "multiple"), (torch._efficientzerotensor((2, 4, 64), dtype=BF), "no memory")):
        with pytest.raises((TypeError, ValueError), match=match):
            P.page_attention(cache, 0, bad, *w)
    for layer in (-1, 2, 0.0, None):
        for call in (lambda: P.store_pages(cache, layer, z(2, 2, 64), z(2, 2, 64), *w), lambda: P.page_attention(cache, layer, z(2, 4, 64), *w)):
            with pytest.raises(ValueError, match="layers 0 to 1"):
                call()
    with pytest.raises(TypeError, match="PageCache"):
        P.page_attention(cache.codes, 0, z(2, 4, 64), *w)
    for window in (-1, 1.0, 1 << 31, None):
        with pytest.raises(ValueError, match="window"):
            P.page_attention(cache, 0, z(2, 4, 64), *w, window=window)
    assert not launched


def test_outputs_that_are_refused(launched):
    cache, w = OnCpu(), where()
    k, q = torch.zeros(2, 2, 64, dtype=BF), torch.zeros(2, 4, 64, dtype=BF)
    with torch.inference_mode():
        inference = torch.zeros(2, 2, 64, dtype=BF)
    for bad, match in ((torch.zeros(1, 2, 64, dtype=BF).expand(2, 2, 64), "overlap"), (torch.zeros(2, 1, 64, dtype=BF).expand(2, 2, 64), "overlap"),
                       (torch.zeros(2, 2, 1, dtype=BF).expand(2, 2, 64), "overlap"), (torch.zeros(300, dtype=BF).as_strided((2, 2, 64), (64, 32, 1)), "overlap"),
                       (k.clone().requires_grad_(), "gradient"), (inference, "inference")):
        with pytest.raises(ValueError, match=match):
            P.load_pages(cache, 0, bad, k, *w)
        with pytest.raises(ValueError, match=match):
            P.load_pages(cache, 0, k, bad, *w)
    for bad, match in ((torch.zeros(2, 4, 65, dtype=BF)[..., :64], "contiguous"), (torch.zeros(513, dtype=BF)[1:].view(2, 4, 64), "16-byte"),
                       (q[:1], "out must be"), (q.float(), "bf16"), (q.clone().requires_grad_(), "gradient"), (torch._neg_view(q.clone()), "contiguous")):
        with pytest.raises((TypeError, ValueError), match=match):
            P.page_attention(cache, 0, q, *w, out=bad)
    flat = torch.zeros(1024, dtype=BF)
    for a, out in ((q, q), (flat[:512].view(2, 4, 64), flat[256:768].view(2, 4, 64))):
        with pytest.raises(ValueError, match="overlap"):
            P.page_attention(cache, 0, a, *w, out=out)
    with pytest.raises(ValueError, match="same place"):
        P.load_pages(cache, 0, k, k, *w)
    assert not launched
    with torch.no_grad():
        P.load_pages(cache, 0, k.requires_grad_(), torch.zeros(2, 2, 64, dtype=BF), *w)
    assert len(launched) == 1


def test_what_is_written_is_another_version(launched):
    cache, w = OnCpu(), where()
    k, v, q, out = (torch.zeros(2, n, 64, dtype=BF) for n in (2, 2, 4, 4))
    before = [t._version for t in (k, v, q, out)]
    P.load_pages(cache, 0, k, v, *w)
    P.page_attention(cache, 0, q, *w, out=out)
    P.store_pages(cache, 0, *(torch.zeros(2, 2, 64, dtype=BF) for _ in range(2)), *w)
    assert [t._version - n for t, n in zip((k, v, q, out), before)] == [1, 1, 0, 1]
    odd = torch.zeros(2, 2, 72, dtype=BF)[..., 1:65]
    before = odd._version, v._version
    P.load_pages(cache, 0, odd, v, *w)
    assert odd._version > before[0] and v._version == before[1] + 1
    with torch.inference_mode():
        P.load_pages(cache, 0, k, torch.zeros(2, 2, 64, dtype=BF), *w)


def test_copies(launched):
    cache = OnCpu()
    for src, dst, match in (([0], [5], "pages 0 to 4"), ([-1], [1], "pages 0 to 4"), ([0, 1], [2], "as many"), ([0, 1], [2, 2], "twice"),
                            ([0, 1], [1, 2], "twice"), ([3], [3], "twice"), ([1 << 40], [0], "pages 0 to 4"), ([0.5], [1], "whole")):
        with pytest.raises((TypeError, ValueError), match=match):
            P.copy_pages(cache, src, dst)
    assert not launched
    P.copy_pages(cache, [0, 0], [2, 4])
    P.copy_pages(cache, torch.tensor([1]), (3,))
    name, at, src, dst, n = launched[0]
    assert (name, at, n) == ("decoder_page_copy", cache._at, 2) and list(src) == [0, 0] and list(dst) == [2, 4]


@pytest.mark.parametrize("n", [1, 30, 256, 257, 3000])
def test_copies_of_many(launched, n):
    """Whatever the order of the pages, the one that is wrong is found."""
    rng = random.Random(n)
    cache = OnCpu(layers=1, pages=2 * n + 5, heads=1)
    pages = rng.sample(range(2 * n + 5), 2 * n)
    src, dst = pages[:n], pages[n:]
    P.copy_pages(cache, src, dst)
    assert len(launched) == 1 and list(launched[0][2]) == src and list(launched[0][3]) == dst
    for i in {0, n // 2, n - 1}:
        for bad, match in ((-1, "pages 0 to"), (2 * n + 5, "pages 0 to"), (1 << 31, "pages 0 to"), (src[(i + 1) % n], "twice")):
            with pytest.raises(ValueError, match=match):
                P.copy_pages(cache, src, dst[:i] + [bad] + dst[i + 1:])
        with pytest.raises(ValueError, match="twice" if n > 1 else "pages 0 to"):
            P.copy_pages(cache, src, dst[:i] + [dst[i - 1] if n > 1 else -5] + dst[i + 1:])
    assert len(launched) == 1
    with pytest.raises(ValueError, match="twice"):
        P.copy_pages(cache, [0] * (2 * n + 6), [1] * (2 * n + 6))


def test_scratch_where_it_is_needed(monkeypatch):
    """Without, where the library may do; with it, when that said so."""
    got = []
    monkeypatch.setattr(P, "_current_device", lambda: None)
    monkeypatch.setattr(P, "_launch", lambda *a: got.append(a[-1]) or (False if answers.pop(0) else None))
    cache, q = OnCpu(), torch.zeros(2, 4, 64, dtype=BF)
    for width, answers, none in ((2, [False], [True]), (2, [True, False], [True, False]), (257, [False], [False])):
        P.page_attention(cache, 0, q, *where(2, width))
        assert [x is None for x in got] == none and not answers
        got.clear()


def test_the_library_refuses_sizes():
    L = K.lib()
    assert L.decoder_page_attention_scratch(96) < 0
    byref = P.ctypes.byref
    good = (1, 1, 1, 64, 4)
    for sizes, layer, width in (((0, 1, 1, 64, 4), 0, 1), ((1, 0, 1, 64, 4), 0, 1), ((1, 1, 0, 64, 4), 0, 1), ((1, 1, 1025, 64, 4), 0, 1),
                                ((1, 1, 1, 32, 4), 0, 1), ((1, 1, 1, 64, 3), 0, 1), ((1, 1, 1, 64, 9), 0, 1), (good, 1, 1), (good, -1, 1), (good, 0, 0)):
        c = P._Described(None, None, None, *sizes)
        assert L.decoder_page_rows(0, byref(c), layer, None, 0, 0, None, 0, 0, None, None, None, width, 1, 1, None) != 0
        assert L.decoder_page_attention(byref(c), layer, None, 0, 0, None, None, None, width, 1, 1, 2, 1.0, 0, None, None, None) != 0
    c = P._Described(None, None, None, 1, 1, 2, 64, 4)
    for rows, hq, window in ((1, 3, 0), (1, 0, 0), (0, 2, 0), (1 << 25, 2, 0), (1, 2, -1)):
        assert L.decoder_page_attention(byref(c), 0, None, 0, 0, None, None, None, 1, 1, rows, hq, 1.0, window, None, None, None) != 0
    for page in (-1, 1):
        ids = (P.ctypes.c_int * 1)(page)
        assert L.decoder_page_copy(byref(c), ids, ids, 1, None) != 0


@pytest.mark.parametrize("mode", ["real", "fake"])
def test_tracers_are_refused(launched, mode):
    cache, w = OnCpu(), where()
    for i in range(3):
        with pytest.raises(RuntimeError, match="tracer"):
            make_fx(lambda x: calls(cache, w, k=x, q=torch.zeros(2, 4, 64, dtype=BF))[i](), tracing_mode=mode)(torch.zeros(2, 2, 64, dtype=BF))
    assert not launched


def test_a_products_rounding_finds_halves():
    """x (1 / s) rounded to multiples of 2^-12, then to whole numbers, is x / s rounded to
    whole numbers, for all 8-bit x and 4-bit s with a quotient below 8."""
    x, s = torch.meshgrid(torch.arange(256.0), torch.arange(8.0, 16.0), indexing="ij")
    for shift in range(-8, 1):
        q = (x.double() * 2.0 ** shift) / s.double()
        keep = q.abs() < 8
        y = (x * 2.0 ** shift).double() * (1 / s).double()        # (exact: 8 by 24 bits)
        twice = torch.round(torch.round(y * 4096) / 4096)
        assert torch.equal(twice[keep], torch.round(q)[keep])


def test_places_of_nibbles():
    for d in (64, 128, 256):
        for value in (0, 1):
            assert sorted(nibble_place(d, value).tolist()) == list(range(d))
    assert nibble_place(128, 0)[:9].tolist() == list(range(8)) + [32] and nibble_place(128, 1)[:5].tolist() == list(range(4)) + [16]
    values, s = held(torch.tensor([[7.0] * 31 + [-7.0] + [1.0] * 32]))
    assert values[0, 0] == 7 and values[0, 31] == -7 and s[0].tolist() == [1.0, 0.140625]
