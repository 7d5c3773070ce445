"""Where in the prompt span a splice takes effect, by gradients.

A sweep measures what happens when a donor's K and V stand in for the prompt
span from layer L on.  This module asks how much of that each layer and position
accounts for, to first order and with one backward pass (attribution patching):
the clean run's continuation is fed to the spliced model, the loss is
the divergence of its next-token distributions from the clean run's top
alternatives, and

    attribution[l, j] = (clean - donor)[l, j] . d loss / d (K, V)[l, j]

is, to first order, what the loss changes by when position j of layer l gets its
clean K and V back (§3 "Splice intervention"; Table 1's donors).

The continuation's attention over span and own keys and its gradients are
``decoder.attention``'s, the clean run's alternatives and both runs' token
scores ``decoder.scoring.token_logprobs``', the loss ``distill_loss``'.  Where a
gradient is asked for, the decoder's other pieces are its torch expressions.

Nothing here waits for the GPU but ``restored``: a kernel's bounded wait that ran
out shows in ``decoder.check_device_error``.

``python -m paper_2605_30574_gb300.attribution`` prints the attribution of every
layer for each donor kind, beside what restoring the whole layer really does.
"""
from __future__ import annotations

import argparse
import json
import sys
from dataclasses import dataclass
from typing import Sequence

import torch

from .decoder import attention as A
from .decoder import scoring
from .synth import workloads as W


def continuation_logits(model, tokens: torch.Tensor, k_span: Sequence[torch.Tensor], v_span: Sequence[torch.Tensor]) -> torch.Tensor:
    """Logits [T, vocab] of ``tokens`` [T] that follow a prompt span whose K and V
    are ``k_span``, ``v_span``, a [Hkv, T_p, d] tensor per layer: token t sits at
    position T_p + t, sees the span and the tokens up to itself, and its row
    scores the next one.  Differentiable with respect to the spans."""
    Tp = k_span[0].shape[1]
    pos = torch.arange(Tp, Tp + tokens.shape[0], device=tokens.device)
    h = model.embed[tokens].float()
    for l in range(model.dims.num_layers):
        q, k, v = model.qkv(l, h, pos)
        keys, values = (torch.cat([span[l], own.transpose(0, 1)], dim=1) for span, own in ((k_span, k), (v_span, v)))
        h = model.block_out(l, h, A.attention(q, keys, values, model.sm_scale))
    return model.logits(h)


@dataclass
class Attribution:
    """Of one (prompt, donor, L): the divergence of each step [T], the clean
    tokens' log probabilities in the clean and the spliced run [T], the entropies
    of both, and the attribution [N, T_p] (of the steps' mean divergence)."""
    divergence: torch.Tensor
    clean_logprobs: torch.Tensor
    spliced_logprobs: torch.Tensor
    clean_entropy: torch.Tensor
    spliced_entropy: torch.Tensor
    attribution: torch.Tensor


def spliced_spans(run, prompt: int, slot: int, L: int):
    """Per layer, the K and V that a cell (prompt, slot, L) reads after its onset
    in a ``model.SpliceDecode``: the donor's from layer L on."""
    k, v = list(run.k_clean[prompt]), list(run.v_clean[prompt])
    zero = run.slot_kinds[slot] == W.ZERO
    at = None if zero else run.stored.index(slot)
    for l in range(L, len(k)):
        k[l], v[l] = (torch.zeros_like(k[l]), torch.zeros_like(v[l])) if zero else (run.k_donor[prompt, at, l], run.v_donor[prompt, at, l])
    return k, v


def attribute(run, prompt: int, slot: int, tokens: torch.Tensor, L: int = 0, top: int = 32) -> Attribution:
    """Attribution of the splice (prompt, slot, L, onset 0) of a
    ``model.SpliceDecode`` over the clean continuation ``tokens`` [T + 1] (y_0 ..
    y_T): T rows, each scoring the next token."""
    model = run.model
    tokens, after = tokens[:-1], tokens[1:]
    clean_k, clean_v = list(run.k_clean[prompt]), list(run.v_clean[prompt])
    with torch.no_grad():
        clean = scoring.token_logprobs(continuation_logits(model, tokens, clean_k, clean_v), after, top=min(top, model.dims.vocab))
    spans = [[t.detach().clone().requires_grad_(l >= L) for l, t in enumerate(span)] for span in spliced_spans(run, prompt, slot, L)]
    with torch.enable_grad():
        logits = continuation_logits(model, tokens, *spans)
        loss = scoring.distill_loss(logits, clean.top_ids, clean.top_logprobs, rest=True)
        if loss.requires_grad:          # (L past the last layer: nothing is spliced)
            loss.mean().backward()
    spliced = scoring.token_logprobs(logits.detach(), after)
    attribution = torch.zeros(model.dims.num_layers, clean_k[0].shape[1], device=tokens.device)
    for clean_span, span in zip((clean_k, clean_v), spans):
        for l in range(L, model.dims.num_layers):
            attribution[l] += ((clean_span[l].float() - span[l].detach().float()) * span[l].grad.float()).sum((0, 2))
    return Attribution(loss.detach(), clean.logprobs, spliced.logprobs, clean.entropy, spliced.entropy, attribution)


@torch.no_grad()
def restored(run, prompt: int, slot: int, tokens: torch.Tensor, layer: int, L: int = 0, top: int = 32) -> float:
    """The mean divergence of ``attribute`` with one layer's span restored."""
    model = run.model
    tokens = tokens[:-1]
    k, v = spliced_spans(run, prompt, slot, L)
    clean = continuation_logits(model, tokens, list(run.k_clean[prompt]), list(run.v_clean[prompt]))
    teacher = scoring.token_logprobs(clean, top=min(top, model.dims.vocab))
    k[layer], v[layer] = run.k_clean[prompt, layer], run.v_clean[prompt, layer]
    return float(scoring.distill_loss(continuation_logits(model, tokens, k, v), teacher.top_ids, teacher.top_logprobs, rest=True).mean())


def main(argv=None) -> int:
    """Attributes each donor kind's splice of one prompt to the layers."""
    ap = argparse.ArgumentParser(description=main.__doc__)
    ap.add_argument("--dims", choices=("tiny", "qwen3-8b"), default="tiny")
    ap.add_argument("--prompt-len", type=int, default=128)
    ap.add_argument("--steps", type=int, default=32, help="tokens of the clean continuation")
    ap.add_argument("--L", type=int, default=0, help="first spliced layer")
    ap.add_argument("--top", type=int, default=32, help="alternatives of the clean run that the divergence goes by")
    ap.add_argument("--kinds", nargs="+", default=["BLANK", "ZERO", "SAME_ALGO", "DIFF_ALGO", "DIFF_FAMILY"])
    ap.add_argument("--seed", type=int, default=0)
    ap.add_argument("--json", default=None, help="also write the attributions here")
    args = ap.parse_args(argv)
    from . import build as B
    from .decoder import check_device_error
    from .model import RandomDecoder, SpliceDecode, qwen3_8b_dims, tiny_dims
    B.build()
    dims = qwen3_8b_dims() if args.dims == "qwen3-8b" else tiny_dims()
    names = {v: k for k, v in W.KIND_NAMES.items()}
    kinds = [names[k] for k in args.kinds]
    model = RandomDecoder(dims, seed=args.seed)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(args.seed + 7)
    prompts = torch.randint(0, dims.vocab, (1, args.prompt_len), generator=gen, device="cuda")
    head, tail = (24, 12) if args.dims == "qwen3-8b" else (4, 2)
    run = SpliceDecode(model, prompts, kinds, [W.Seq(0, 0, dims.num_layers, 0)], args.steps + 1, head, tail, filler=64, seed=args.seed)
    out = {}
    try:
        tokens = run.decode(args.steps + 1)[0]
        for slot, kind in enumerate(kinds):
            a = attribute(run, 0, slot, tokens, args.L, args.top)
            by_layer = a.attribution.sum(1).tolist()
            base = float(a.divergence.mean())
            print(f"{W.KIND_NAMES[kind]}: divergence {base:.4g}, clean tokens' log probability {float(a.clean_logprobs.mean()):.3f} "
                  f"clean, {float(a.spliced_logprobs.mean()):.3f} spliced")
            print(" layer   attributed     restored  largest at position")
            for l in range(args.L, dims.num_layers):
                print(f"{l:6d} {by_layer[l]:12.4g} {restored(run, 0, slot, tokens, l, args.L, args.top) - base:12.4g} {int(a.attribution[l].abs().argmax()):20d}")
            out[W.KIND_NAMES[kind]] = {"divergence": base, "by_layer": by_layer, "by_position": a.attribution.sum(0).tolist()}
        check_device_error()
    finally:
        run.close()
    if args.json:
        with open(args.json, "w") as f:
            json.dump(out, f)
    return 0


if __name__ == "__main__":
    sys.exit(main())
