"""Train a draft head on a target's stored top logits.

    python examples/train_on_top_logits.py [--steps 30] [--vocab 32000] [--top 64]

What a training set of a large target keeps of every position is its top logits,
taken after the penalties and grammars that the server applies:

  once      target logits -> aal_logits_process -> aal_topk_logits -> the data set
  a step    draft logits  -> aal_logits_process -> aal_topk_loss_fwd_bwd (KL + 0.1 EAL, windows
            sliding over the sequences) -> aal_logits_process_bwd -> the head's gradient

Target and draft are linear heads over random features (synthetic data); the draft's
features are the target's with noise, so that it can learn most of the distribution.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2609_24150_amd as aal  # noqa: E402


def make_rules(B: int, S: int, V: int, tokens: torch.Tensor, g: torch.Generator) -> dict:
    """Rules of B sequences of S positions: a position's history is its sequence before it,
    the first quarter of it the prompt; every other sequence is generated under a grammar."""
    dev = tokens.device
    place = torch.arange(S, device=dev).repeat(B)
    start = torch.arange(B, device=dev).repeat_interleave(S) * S
    ones = torch.ones(B * S, device=dev)
    words = (V + 31) // 32
    # grammars that allow about three quarters of the vocabulary
    mask = torch.randint(-2 ** 31, 2 ** 31, (B, words), generator=g, device=dev) | \
        torch.randint(-2 ** 31, 2 ** 31, (B, words), generator=g, device=dev)
    which = torch.arange(B, device=dev).repeat_interleave(S)
    return dict(tokens=tokens.reshape(-1), hist_start=start, hist_len=place.int(),
                prompt_len=place.clamp(max=S // 4).int(), repetition=1.1 * ones, frequency=0.05 * ones,
                presence=0.1 * ones, mask=mask.int(), mask_row=torch.where(which % 2 == 0, -1, which).int())


def main(argv=None) -> list[float]:
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--steps", type=int, default=30)
    ap.add_argument("--batch", type=int, default=4)
    ap.add_argument("--positions", type=int, default=64)
    ap.add_argument("--vocab", type=int, default=32000)
    ap.add_argument("--width", type=int, default=256)
    ap.add_argument("--top", type=int, default=64)
    ap.add_argument("--window", type=int, default=7)
    ap.add_argument("--lr", type=float, default=2.0)
    a = ap.parse_args(argv)
    dev, B, S, V, D, K = "cuda", a.batch, a.positions, a.vocab, a.width, a.window
    g = torch.Generator(dev).manual_seed(0)

    target_head = torch.randn(V, D, generator=g, device=dev) * (3.0 / D ** 0.5)
    features = torch.randn(B * S, D, generator=g, device=dev)
    tokens = torch.randint(0, V, (B, S), generator=g, device=dev, dtype=torch.int32)
    rules = make_rules(B, S, V, tokens, g)

    # the data set: 6 bytes for each of the top logits instead of 2 V a position
    target = aal.aal_logits_process((features @ target_head.t()).bfloat16(), **rules)
    data = aal.aal_topk_logits(target, a.top)
    shape = lambda t: t.view(B, S, *t.shape[1:])  # noqa: E731
    top, ids, rest = shape(data["logits"]), shape(data["ids"]), shape(data["rest"])

    seen = features + 0.3 * torch.randn(B * S, D, generator=g, device=dev)
    head = torch.zeros(V, D, device=dev)
    losses = []
    for step in range(a.steps):
        raw = (seen @ head.t()).bfloat16()
        z = aal.aal_logits_process(raw, **rules)
        out = aal.aal_topk_loss_fwd_bwd(z.view(B, S, V), top, ids, K, rest=rest, weights=(0.0, 0.1, 1.0, 0.0),
                                        layout=aal.AAL_LAYOUT_SEQUENCES)
        grad = aal.aal_logits_process_bwd(out["grad"].view(B * S, V), raw, **rules)
        head -= a.lr * (grad.float().t() @ seen)
        losses.append(out["loss"].item())
        if step % 5 == 0 or step == a.steps - 1:
            kl, accept = out["terms"][2].item(), out["accept_tv"].mean().item()
            print(f"step {step:3d}  loss {losses[-1]:.4f}  KL {kl:.4f}  acceptance {accept:.3f}", flush=True)
    return losses


if __name__ == "__main__":
    main()
