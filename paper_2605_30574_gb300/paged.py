"""Algorithm 1 over a cache of pages in 4 bits: cells start as forks of the clean run.

``model.SpliceDecode`` decodes every cell of a sweep from step 1 on, over bf16 stores
that all cells' prompt spans and generated tokens have to fit in.  Two facts of the
method (§3 "Splice intervention") leave less to hold and to compute:

* up to its onset W a cell is the clean run of its prompt, token for token.  So one clean
  run per prompt is decoded, and a cell is forked from it at step W: it shares all pages
  but the one that is begun, which is copied when it is written to;
* from step W on, its layers l >= L read the donor's span where the others read the clean
  one's.  Pages hold all layers, and every layer has a table of its own: for those layers
  the span's entries are the donor's pages (ZERO: one page of zeros, again and again).

Keys and values take 4.3 bits each at 128 dims for bf16's 16 (``decoder.pages``), so logits
differ from bf16's by what that rounding makes of them; the prefills' own attention is in
bf16.  The attention reads a span once for each cell: for speed, where the stores fit,
``SpliceDecode`` reads it once for all.

``python -m paper_2605_30574_gb300.paged`` times steps of a Qwen3-8B-shaped random decoder
on the ladder's cells and prints what the cache takes.
"""
from __future__ import annotations

import argparse
import json
import sys
from typing import Dict, List, Optional, Sequence

import torch

from . import decoder as K
from .decoder import pages as P
from .model import RandomDecoder, donor_tokens, ladder_batch_cells, qwen3_8b_dims
from .synth import workloads as W


class PagedDecode:
    """Algorithm 1 for a batch of sweep cells (prompt, donor slot, L, W), as
    ``model.SpliceDecode`` takes them, with ``max_steps`` tokens to a run.  A prompt's length
    is a multiple of ``page``."""

    def __init__(self, model: RandomDecoder, prompts: torch.Tensor, slot_kinds: Sequence[int], seqs: Sequence[W.Seq], max_steps: int,
                 scaffold_head: int = 0, scaffold_tail: int = 0, filler: int = 0, seed: int = 0, page: int = 64):
        dims, dev = model.dims, model.device
        count, Tp = prompts.shape
        if Tp % page:
            raise ValueError(f"PagedDecode: prompts of {Tp} tokens are no whole pages of {page}")
        self.model, self.seqs, self.Tp, self.T, self.page = model, list(seqs), Tp, max_steps, page
        kinds = tuple(slot_kinds)
        N, Hkv, d = dims.num_layers, dims.num_kv_heads, dims.head_dim
        stored = [k for k, kind in enumerate(kinds) if kind != W.ZERO]
        spans, each = Tp // page, -(-max_steps // page) + 1            # (pages of a span; of a run's own tokens)
        self.cache = P.PageCache.empty(N, count * (1 + len(stored)) * spans + 1 + (count + len(self.seqs)) * each, Hkv, d, page, dev)
        self.tables = P.PageTables(self.cache)
        gen = torch.Generator(device=dev)
        gen.manual_seed(seed + 1)
        k, v = (torch.empty((N, Hkv, Tp, d), dtype=torch.bfloat16, device=dev) for _ in range(2))
        with torch.cuda.device(dev):
            self._errors = K.ErrorReader()

        def held(tokens):
            """The sequence of a prefill, and its last logits."""
            logits = model.prefill(tokens, k, v)
            i = self.tables.add(Tp)
            where = self.tables.tensors([i], None, store=True)
            for l in range(N):
                P.store_pages(self.cache, l, k[l].transpose(0, 1), v[l].transpose(0, 1), *where)
            return i, logits

        self.runs: List[int] = []                                      # the clean run of each prompt
        donors: Dict[tuple, torch.Tensor] = {}
        y0 = torch.empty(count, dtype=torch.long, device=dev)
        for p in range(count):
            i, logits = held(prompts[p])
            self.runs.append(i)
            y0[p] = logits.argmax()
            for s in stored:
                toks = donor_tokens(prompts[p], kinds[s], gen, dims.vocab, scaffold_head, scaffold_tail, filler)
                donors[p, s] = torch.tensor(self.tables.pages(held(toks)[0]), dtype=torch.int32)
        zero = self.tables.add(page)
        nothing = torch.zeros((page, Hkv, d), dtype=torch.bfloat16, device=dev)
        for l in range(N):
            P.store_pages(self.cache, l, nothing, nothing, *self.tables.tensors([zero], None, store=True))
        zeros = torch.full((spans,), self.tables.pages(zero)[0], dtype=torch.int32)
        # a cell's pages of the span, at its layers l >= L
        self._spans = [zeros if kinds[c.slot] == W.ZERO else donors[c.prompt, c.slot] for c in self.seqs]
        self.first_token = y0
        # the rows of a step: the clean runs, then the cells, as they are forked
        self.cells: List[int] = []
        self._ids: List[int] = list(self.runs)
        self.check()

    def check(self):
        """As ``SpliceDecode.check``."""
        with torch.cuda.device(self.model.device):
            self._errors.check()

    def fork(self, t: int) -> List[int]:
        """Starts the cells whose onset is step t, behind the rows that there are; returns
        the rows of their prompts' clean runs, which they continue."""
        new = [c for c, cell in enumerate(self.seqs) if max(cell.W, 1) == t]
        for c in new:
            self._ids += self.tables.fork(self.runs[self.seqs[c].prompt])
        self.cells += new
        return [self.seqs[c].prompt for c in new]

    def _tables(self):
        """Every layer's table, starts and lengths for the rows, each with one new token."""
        self.tables.extend(self._ids)
        table, starts, lengths = self.tables.tensors(self._ids, store=True)
        dev, clean, spans = self.model.device, len(self.runs), self.Tp // self.page
        spliced = table.clone()
        if self.cells:
            spliced[clean:, :spans] = torch.stack([self._spans[c] for c in self.cells]).to(dev)
        L = torch.tensor([self.model.dims.num_layers] * clean + [self.seqs[c].L for c in self.cells], device=dev)[:, None]
        return [torch.where(L <= l, spliced, table) for l in range(self.model.dims.num_layers)], starts, lengths

    @torch.no_grad()
    def step(self, t: int, tokens: torch.Tensor) -> torch.Tensor:
        """Forward pass of step t (1 <= t < T) for all rows: tokens are their y_{t-1}; returns
        the logits whose argmax is y_t.  Its tables come from the host's memory, so it begins
        when the GPU has done what was given to it before, and does not wait for what it gives
        it: see ``check``."""
        model, cache = self.model, self.cache
        tables, starts, lengths = self._tables()
        pos = torch.full((len(self._ids),), self.Tp + t - 1, device=model.device)
        h = model.embed[tokens].float()
        for l in range(model.dims.num_layers):
            q, k, v = model.qkv(l, h, pos)
            P.store_pages(cache, l, k, v, tables[l], starts, lengths)
            h = model.block_out(l, h, P.page_attention(cache, l, q, tables[l], starts, lengths, scale=model.sm_scale))
        return model.logits(h)

    @torch.no_grad()
    def decode(self, steps: Optional[int] = None) -> torch.Tensor:
        """Greedy splice-intervention decode; returns the cells' tokens [B][steps], as
        ``SpliceDecode.decode`` does.  Once for an object."""
        steps = self.T if steps is None else steps
        if self.cells or not 1 <= steps <= self.T:
            raise ValueError(f"PagedDecode.decode: once, and 1 to {self.T} steps")
        eos, toks = self.model.dims.eos, self.first_token[:, None]
        for t in range(1, steps):
            parents = self.fork(t)
            if parents:
                toks = torch.cat([toks, toks[torch.tensor(parents, device=toks.device)]])
            y = self.step(t, toks[:, -1]).argmax(-1)
            if eos is not None:
                y = torch.where((toks == eos).any(1), torch.full_like(y, eos), y)
            toks = torch.cat([toks, y[:, None]], dim=1)
        self.check()
        # (a cell whose onset was not reached is its prompt's clean run)
        row = {c: len(self.runs) + i for i, c in enumerate(self.cells)}
        return toks[torch.tensor([row.get(c, cell.prompt) for c, cell in enumerate(self.seqs)], device=toks.device)]


def main(argv=None):
    """Times steps of Algorithm 1 over 4-bit pages for a Qwen3-8B-shaped random decoder on
    batch 0 of the ladder sweep: its cells from their onsets on."""
    ap = argparse.ArgumentParser(description=main.__doc__)
    ap.add_argument("--steps", type=int, default=16, help="decode steps timed (after the warm-up)")
    ap.add_argument("--warmup", type=int, default=3)
    ap.add_argument("--page", type=int, default=64)
    args = ap.parse_args(argv)
    from . import build as B
    B.build()
    wl, dims = W.get("qwen3-8b-ladder"), qwen3_8b_dims()
    seqs = ladder_batch_cells(wl, 0)
    p0 = min(q.prompt for q in seqs)
    seqs = [W.Seq(q.prompt - p0, q.slot, q.L, q.W) for q in seqs]
    count, T = max(q.prompt for q in seqs) + 1, args.warmup + args.steps + 1
    model = RandomDecoder(dims, seed=0)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(7)
    prompts = torch.randint(0, dims.vocab, (count, wl.prompt_len), generator=gen, device="cuda")
    run = PagedDecode(model, prompts, wl.slot_kinds, seqs, T, wl.scaffold_head, wl.scaffold_tail, filler=64, page=args.page)
    toks, ms, rows = run.first_token, [], []
    for t in range(1, T):
        parents = run.fork(t)
        toks = torch.cat([toks, toks[torch.tensor(parents, device=toks.device, dtype=torch.long)]])
        ev = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
        ev[0].record()
        toks = run.step(t, toks).argmax(-1)
        ev[1].record()
        torch.cuda.synchronize()
        if t > args.warmup:
            ms.append(ev[0].elapsed_time(ev[1]))
            rows.append(len(toks))
    run.check()
    tokens = run.cache.pages - run.tables.free
    print(json.dumps({
        "what": "Algorithm 1 over 4-bit pages, random-init Qwen3-8B-shaped decoder, ladder batch 0",
        "cells": len(seqs), "rows_of_a_step": [rows[0], rows[-1]], "ms_per_step_median": round(sorted(ms)[len(ms) // 2], 3),
        "cache_bytes_in_use": round(run.cache.nbytes * tokens / run.cache.pages),
        "bf16_bytes_of_the_same_pages": tokens * args.page * dims.num_layers * dims.num_kv_heads * dims.head_dim * 4}))
    return 0


if __name__ == "__main__":
    sys.exit(main())
