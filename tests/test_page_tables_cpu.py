"""What a cache's pages are given to, against a plain model of it: every sequence a list of
its tokens' values, every page a list that copies copy."""
import random

import pytest
import torch

from paper_2605_30574_gb300.decoder import pages as P

from test_pages_cpu import OnCpu, _built, launched  # noqa: F401


class Model:
    """Tables over pages whose content is written and copied here, in the order of the
    calls."""

    def __init__(self, monkeypatch, pages=12, page=16):
        self.cache = OnCpu(pages=pages, page=page)
        self.tables = P.PageTables(self.cache)
        self.content = [[None] * page for _ in range(pages)]
        self.tokens, self.stamp = {}, 0
        monkeypatch.setattr(P, "copy_pages", self.copy)

    def copy(self, cache, src, dst):
        assert cache is self.cache and len(set(dst)) == len(dst) == len(src) and not set(src) & set(dst)
        for s, d in zip(src, dst):
            self.content[d] = list(self.content[s])

    def write(self, i, n):
        """The n newest tokens of sequence i, as store_pages writes them."""
        held, page = self.tables.pages(i), self.cache.page
        for at in range(len(self.tokens[i]), len(self.tokens[i]) + n):
            self.stamp += 1
            self.tokens[i].append(self.stamp)
            self.content[held[at // page]][at % page] = self.stamp

    def check(self):
        page = self.cache.page
        for i, want in self.tokens.items():
            held = self.tables.pages(i)
            assert self.tables.length(i) == len(want) and len(held) == -(-len(want) // page)
            assert [self.content[held[at // page]][at % page] for at in range(len(want))] == want
        used = {p for i in self.tokens for p in self.tables.pages(i)}
        assert self.tables.free == self.cache.pages - len(used)


@pytest.mark.parametrize("seed", range(8))
def test_any_order_of_calls(monkeypatch, seed):
    rng = random.Random(seed)
    m = Model(monkeypatch, pages=rng.choice((5, 12, 40)))
    page = m.cache.page
    for _ in range(400):
        ids = list(m.tokens)
        what = rng.choice(("add", "extend", "extend", "extend", "fork", "splice", "drop", "compact"))
        try:
            if what == "add":
                n = rng.choice((0, 1, page, rng.randint(0, 3 * page)))
                i = m.tables.add(n)
                m.tokens[i] = []
                m.write(i, n)
            elif what == "extend" and ids:
                some = rng.sample(ids, rng.randint(1, len(ids)))
                n = [rng.choice((0, 1, 1, 1, page, 2 * page + 3)) for _ in some] if rng.random() < 0.5 else 1
                m.tables.extend(some, n)
                for i, k in zip(some, [n] * len(some) if n == 1 else n):
                    m.write(i, k)
            elif what == "fork" and ids:
                i = rng.choice(ids)
                for j in m.tables.fork(i, rng.randint(0, 3)):
                    m.tokens[j] = list(m.tokens[i])
            elif what == "splice" and ids:
                i, j = rng.choice(ids), rng.choice(ids)
                n = rng.randint(0, min(len(m.tokens[i]), len(m.tokens[j])) // page) * page
                m.tables.splice(i, j, n)
                m.tokens[i][:n] = m.tokens[j][:n]
            elif what == "drop" and ids:
                some = rng.sample(ids, rng.randint(0, min(3, len(ids))))
                m.tables.drop(some)
                for i in some:
                    del m.tokens[i]
            elif what == "compact":
                k = m.tables.compact()
                assert all(p < k for i in m.tokens for p in m.tables.pages(i))
        except RuntimeError as e:
            assert "free" in str(e)
        m.check()


def test_the_last_holder_keeps_a_begun_page(monkeypatch):
    m = Model(monkeypatch)
    a = m.tables.add(20)
    m.tokens[a] = []
    m.write(a, 20)
    b, c = m.tables.fork(a, 2)
    m.tokens[b], m.tokens[c] = list(m.tokens[a]), list(m.tokens[a])
    was = m.tables.pages(a)
    m.tables.extend([a, b, c])
    for i in (a, b, c):
        m.write(i, 1)
    m.check()
    assert m.tables.pages(c) == was and len({m.tables.pages(i)[1] for i in (a, b, c)}) == 3
    assert {m.tables.pages(i)[0] for i in (a, b, c)} == {was[0]}


def test_too_few_pages_change_nothing(monkeypatch):
    m = Model(monkeypatch, pages=3)
    a = m.tables.add(20)
    m.tokens[a] = []
    m.write(a, 20)
    (b,) = m.tables.fork(a)
    before = (m.tables.pages(a), m.tables.pages(b), m.tables.free, m.tables.length(a))
    for call in (lambda: m.tables.extend([a, b], 13), lambda: m.tables.extend([a], 100), lambda: m.tables.add(17)):
        with pytest.raises(RuntimeError, match="1 are free|are free"):
            call()
        assert (m.tables.pages(a), m.tables.pages(b), m.tables.free, m.tables.length(a)) == before


def test_a_copy_that_fails_changes_nothing(monkeypatch):
    m = Model(monkeypatch, pages=6)
    a = m.tables.add(20)
    m.tokens[a] = []
    m.write(a, 20)
    m.tables.fork(a)

    def fails(*_):
        raise RuntimeError("CUDA error 1")
    before = (m.tables.pages(a), m.tables.free, m.tables.length(a))
    with monkeypatch.context() as patch:
        patch.setattr(P, "copy_pages", fails)
        for call in (lambda: m.tables.extend([a], 20), m.tables.compact):
            with pytest.raises(RuntimeError, match="CUDA error 1"):
                call()
            assert (m.tables.pages(a), m.tables.free, m.tables.length(a)) == before
    m.tables.extend([a], 20)
    assert m.tables.free == 6 - 2 - 2 and m.tables.length(a) == 40


def test_tensors(launched):  # noqa: F811
    t = P.PageTables(OnCpu(pages=12))
    a, b = t.add(33), t.add(0)
    c = t.add(1)
    table, starts, lengths = t.tensors([a, c, b], [2, 1, 0])
    assert table.dtype is starts.dtype is lengths.dtype is torch.int32
    assert table.tolist() == [list(t.pages(a)), [t.pages(c)[0], -1, -1], [-1] * 3]
    assert starts.tolist() == [0, 2, 3, 3] and lengths.tolist() == [33, 1, 0]
    assert t.tensors([a, c], None)[1].tolist() == [0, 33, 34] and t.tensors([a], width=5)[0].shape == (1, 5)
    P.store_pages(t.cache, 0, *[torch.zeros(3, 2, 64, dtype=torch.bfloat16)] * 2, table, starts, lengths)
    assert len(launched) == 1


def test_calls_that_are_refused(launched):  # noqa: F811
    t = P.PageTables(OnCpu())
    a, b = t.add(16), t.add(40)
    for call in (lambda: t.fork(99), lambda: t.drop([a, 99]), lambda: t.length(0), lambda: t.pages(None), lambda: t.extend([99]),
                 lambda: t.extend([a, a]), lambda: t.drop([b, b]), lambda: t.extend([a, b], [1]), lambda: t.extend([a], -1),
                 lambda: t.extend([a], [0.5]), lambda: t.add(-1), lambda: t.add(1.0), lambda: t.fork(a, -1), lambda: t.splice(b, a, 8),
                 lambda: t.splice(b, a, 32), lambda: t.splice(a, b, -16), lambda: t.tensors([a], 17), lambda: t.tensors([a], [1, 1]),
                 lambda: t.tensors([a], -1)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        P.PageTables(None)
    assert not launched and t.length(a) == 16 and t.length(b) == 40 and t.free == 1
