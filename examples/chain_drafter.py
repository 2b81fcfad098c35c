"""A chain that drafts for a larger model: the calls on rows of token logits next to the chain's own.

The target is a model over bytes (here a stand-in of fixed random weights: its logits depend on the
last two bytes).  The drafter is a linear chain of 256 labels whose transition scores are one
256 x 256 matrix.
  1. The target reads a corpus; `top_logits` keeps the 32 largest logits of every row and its
     log-sum-exp.
  2. The chain's rows (its matrix, gathered at the corpus' bytes) are distilled from them:
     `distill_grad`, summed over the rows of each byte, is the gradient of the matrix.
  3. `sample` draws a draft of each sequence from the chain, `verify` answers with the target's
     distribution: the drafts that stand, and one more byte.

    python examples/chain_drafter.py
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2002_00876_amd import binding  # noqa: E402

V, K, DRAFTS = 256, 32, 5


class Target:
    """Logits [B, N, 256] of the byte after each of a sequence's bytes [B, N]."""

    def __init__(self, generator):
        dev = generator.device
        self.first = 2.5 * torch.randn((V, V), generator=generator, device=dev)
        self.second = 0.7 * torch.randn((V, V), generator=generator, device=dev)

    def __call__(self, text):
        before = torch.cat([text[:, :1], text[:, :-1]], 1)
        return (self.first[text] + self.second[before]).bfloat16()


def read(target, generator, B, N):
    """A corpus: bytes [B, N] sampled from the target."""
    text = torch.randint(0, V, (B, 1), generator=generator, device=generator.device)
    while text.shape[1] < N:
        p = torch.softmax(target(text[:, -2:])[:, -1].float(), 1)
        text = torch.cat([text, torch.multinomial(p, 1, generator=generator)], 1)
    return text


def answer(chain, target, text, generator):
    """One round: drafts of every sequence, verified.  (emitted, accepted)"""
    B, dev = text.shape[0], text.device
    # the chain's normalised rows, the first clamped to follow the text: its samples are then those
    # of the rows one after the other, whose log-probabilities are what the drafts were drawn from
    rows = torch.log_softmax(chain, 1)
    pot = rows.expand(B, DRAFTS, V, V).clone()
    pot[:, 0] = pot[:, 0].masked_fill(torch.arange(V, device=dev)[None, :, None]
                                      != text[:, -1, None, None], -float("inf"))
    u = torch.rand((1, B, DRAFTS + 1), generator=generator, device=dev)
    path = binding.sample(pot, u)[0]                          # the text's last byte, the drafts
    drafts = path[:, 1:].contiguous()
    logits = target(torch.cat([text[:, -2:], drafts.long()], 1))[:, 1:]
    return binding.verify(
        logits, rows[path[:, :-1].long()], drafts,
        torch.rand((B, DRAFTS), generator=generator, device=dev),
        torch.empty((B, V), device=dev).exponential_(generator=generator).clamp_(min=1e-30),
        draft_lse=torch.zeros((B, DRAFTS), device=dev))[:2]


def main(steps=200, quiet=False):
    g = torch.Generator(device="cuda:0")
    g.manual_seed(0)
    target = Target(g)
    text = read(target, g, 64, 256)
    lengths = torch.full((64,), 256, dtype=torch.int32, device=text.device)
    lengths[::3] = 180                                        # sequences of two lengths
    kept = binding.top_logits(target(text), K, lengths)
    weights = torch.full(text.shape, 1.0 / int(lengths.sum()), device=text.device)
    chain = torch.zeros((V, V), device=text.device)
    drawn = text[:, -2:].repeat(8, 1)
    before = answer(chain, target, drawn, g)[1].float().mean().item()
    losses, speed = [], torch.zeros_like(chain)
    for step in range(steps):
        loss, grad = binding.distill_grad(chain[text], *kept, lengths, weights)
        losses.append((loss * weights).sum().item())
        by_byte = torch.zeros_like(chain).index_add_(0, text.reshape(-1), grad.reshape(-1, V))
        speed = 0.9 * speed + by_byte
        chain = chain - 60.0 * speed
        if not quiet and step % 20 == 0:
            print(f"step {step:4d}  divergence {losses[-1]:.4f}", flush=True)
    emitted, accepted = answer(chain, target, drawn, g)
    after = accepted.float().mean().item()
    if not quiet:
        print(f"divergence {losses[0]:.4f} -> {losses[-1]:.4f}; of {DRAFTS} drafts "
              f"{before:.2f} stood before, {after:.2f} after; emitted {emitted[0].tolist()}")
    return losses, before, after


if __name__ == "__main__":
    main()
