"""What the pages of ``PagedDecode`` hold, against a record of it that knows nothing of
pages: the prefills' keys and values as ``SpliceDecode`` stores them, and each step's as
they were given to be stored, rounded by the format's definition.  Exact.  Each step's
logits against the fp64 oracle's attention over that record."""
import numpy as np
import pytest
import torch

import oracle
from paper_2605_30574_gb300 import build as B
from paper_2605_30574_gb300 import decoder as K
from paper_2605_30574_gb300.decoder import pages as P
from paper_2605_30574_gb300.model import SpliceDecode
from paper_2605_30574_gb300.synth import workloads as WL

from page_util import held, values
from test_gpu_paged import KINDS, LOGIT_TOL, started

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    B.build()
    yield
    K.check_device_error()


def rounded(k, v):
    """[2][heads][tokens][d] of k and v [heads][tokens][d], fp64."""
    return torch.stack([held(x.cpu())[0] for x in (k, v)]).numpy()


def in_pages(cache, layer, ids, tokens):
    got = values(cache, layer)[torch.as_tensor(ids).long()]              # [pages][2][heads][page][d]
    return got.permute(1, 2, 0, 3, 4).flatten(2, 3)[:, :, :tokens].numpy()


@pytest.mark.parametrize("page,Tp", [(16, 48), (32, 32)])
def test_the_record_of_a_decode(monkeypatch, page, Tp):
    args, run = started(20, (0, 2, 5, 17), page=page, Tp=Tp)
    model, N = run.model, run.model.dims.num_layers
    other = SpliceDecode(*args)
    # the spans, by prompt, and by prompt and donor
    clean = [[rounded(other.k_clean[p, l], other.v_clean[p, l]) for l in range(N)] for p in range(2)]
    donors = {(p, k): [rounded(other.k_donor[p, i, l], other.v_donor[p, i, l]) for l in range(N)]
              for p in range(2) for i, k in enumerate(other.stored)}
    other.close()
    for p, i in enumerate(run.runs):
        for l in range(N):
            assert np.array_equal(in_pages(run.cache, l, run.tables.pages(i), Tp), clean[p][l])
    for c, cell in enumerate(run.seqs):
        for l in range(N):
            got = in_pages(run.cache, l, run._spans[c].tolist(), Tp)
            assert np.array_equal(got, donors[cell.prompt, cell.slot][l]) if KINDS[cell.slot] != WL.ZERO else not got.any()

    given = {}
    store = P.store_pages

    def recorded(cache, layer, k, v, *where):
        given[layer] = rounded(k.transpose(0, 1), v.transpose(0, 1))
        return store(cache, layer, k, v, *where)
    monkeypatch.setattr(P, "store_pages", recorded)

    rows, cells, toks = [list(x) for x in clean], [None] * 2, run.first_token
    for t in range(1, 19):
        parents = run.fork(t)
        rows += [list(rows[p]) for p in parents]
        cells += [run.seqs[c] for c in run.cells[len(cells) - 2:]]
        toks = torch.cat([toks, toks[torch.tensor(parents, device="cuda", dtype=torch.long)]])
        got = run.step(t, toks)
        for r, row in enumerate(rows):
            for l in range(N):
                row[l] = np.concatenate([row[l], given[l][:, :, r:r + 1]], axis=2)
        if t in (1, 2, 5, 16, 17, 18):
            for r, i in enumerate(run._ids):
                for l in range(N):
                    assert np.array_equal(in_pages(run.cache, l, run.tables.pages(i), Tp + t), rows[r][l]), (t, r, l)
            want = logits_over(model, Tp, t, toks, rows, cells, donors)
            err = (got - want).abs().amax(-1) / want.abs().amax(-1)
            assert float(err.max()) <= LOGIT_TOL, (t, float(err.max()))
        toks = got.argmax(-1)
    # (cells without a spliced layer among them, each from its run's tokens on)
    assert sum(c is not None and c.L == N for c in cells) == len(cells[2:]) // 3
    run.check()


def logits_over(model, Tp, t, tokens, rows, cells, donors):
    """Logits of step t whose attention is the oracle's over the record, spliced physically."""
    pos = torch.full((len(tokens),), Tp + t - 1, device="cuda")
    h = model.embed[tokens].float()
    for l in range(model.dims.num_layers):
        q = model.qkv(l, h, pos)[0].double().cpu().numpy()
        out = np.zeros(q.shape)
        for r, (row, cell) in enumerate(zip(rows, cells)):
            kv = row[l]
            src = oracle.SRC_CLEAN if cell is None else oracle.splice_source(cell.L, cell.W, cell.slot, KINDS[cell.slot], l, t)
            if src == oracle.SRC_ZERO:
                kv = np.concatenate([np.zeros_like(kv[:, :, :Tp]), kv[:, :, Tp:]], axis=2)
            elif src != oracle.SRC_CLEAN:
                kv = np.concatenate([donors[cell.prompt, cell.slot][l], kv[:, :, Tp:]], axis=2)
            out[r] = oracle.attend(q[r], kv[0], kv[1], 0, model.sm_scale)
        h = model.block_out(l, h, torch.from_numpy(out).to("cuda", torch.float32))
    return model.logits(h)
