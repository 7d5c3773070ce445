"""Tables for calls that store: no page that two sequences hold is written to."""
import pytest
import torch

from paper_2605_30574_gb300.decoder import pages as P

from test_page_tables_cpu import Model
from test_pages_cpu import OnCpu, _built, launched  # noqa: F401


def refused(t, *args):
    with pytest.raises(ValueError, match="another sequence holds too|each sequence once"):
        t.tensors(*args, store=True)
    t.tensors(*args)                                     # (what only reads may)


def test_after_a_fork(launched):  # noqa: F811
    t = P.PageTables(OnCpu(pages=12))
    a = t.add(40)
    (b,) = t.fork(a)
    for ids, new in (([a, b], 40), ([a, b], None), ([a], 1), ([b], 9), ([a, b], [0, 1])):
        refused(t, ids, new)
    t.tensors([a, b], 0, store=True)
    # tokens that ``extend`` gave since then: its copies, and new pages
    t.extend([a, b], [1, 30])
    got = t.tensors([a, b], [1, 30], store=True)
    assert torch.equal(got[0], t.tensors([a, b], [1, 30])[0]) and not set(t.pages(a)[2:]) & set(t.pages(b)[2:])
    for ids, new in (([a], 41), ([b], 39), ([a, b], [1, 70])):
        refused(t, ids, new)
    # the begun page is each one's own by now, as far as its first token
    t.tensors([a, b], [9, 38], store=True)
    refused(t, [a], 10)
    # one that is left by itself
    t.drop([a])
    t.tensors([b], None, store=True)


def test_after_a_splice(launched):  # noqa: F811
    t = P.PageTables(OnCpu(pages=12))
    a, b = t.add(40), t.add(48)
    t.tensors([a, b], None, store=True)
    t.splice(a, b, 32)
    for ids, new in (([a], None), ([b], None), ([a], 9), ([b], 17)):
        refused(t, ids, new)
    t.tensors([a, b], [8, 16], store=True)


def test_a_sequence_twice(launched):  # noqa: F811
    t = P.PageTables(OnCpu(pages=12))
    a, b = t.add(40), t.add(3)
    refused(t, [a, b, a], 1)


@pytest.mark.parametrize("seed", range(4))
def test_what_is_stored_by_such_tables(monkeypatch, seed):
    """Of all sequences of a random history: those that are given tables for a store change
    nobody else's tokens by it."""
    import random
    rng = random.Random(seed)
    m = Model(monkeypatch, pages=40)
    page, given = m.cache.page, 0
    for _ in range(300):
        ids = list(m.tokens)
        what = rng.choice(("add", "extend", "fork", "splice", "drop", "store", "store"))
        try:
            if what == "add":
                i = m.tables.add(rng.randint(0, 60))
                m.tokens[i] = []
                m.write(i, m.tables.length(i))
            elif what == "extend" and ids:
                i, n = rng.choice(ids), rng.randint(0, 20)
                m.tables.extend([i], n)
                m.write(i, n)
            elif what == "fork" and ids:
                i = rng.choice(ids)
                for j in m.tables.fork(i):
                    m.tokens[j] = list(m.tokens[i])
            elif what == "splice" and ids:
                i, j = rng.choice(ids), rng.choice(ids)
                n = min(len(m.tokens[i]), len(m.tokens[j])) // page * page
                m.tables.splice(i, j, n)
                m.tokens[i][:n] = m.tokens[j][:n]
            elif what == "drop" and len(ids) > 3:
                m.tables.drop([ids[0]])
                del m.tokens[ids[0]]
            elif what == "store" and ids:
                some = rng.sample(ids, rng.randint(1, min(3, len(ids))))
                new = [rng.randint(0, len(m.tokens[i])) for i in some]
                try:
                    m.tables.tensors(some, new, store=True)
                except ValueError:
                    continue
                given += any(new)
                for i, n in zip(some, new):
                    del m.tokens[i][len(m.tokens[i]) - n:]
                    m.write(i, n)
        except RuntimeError as e:
            assert "free" in str(e)
        m.check()
    assert given > 5
