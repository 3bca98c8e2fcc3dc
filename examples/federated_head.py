"""Federated training of a small language model on libfls, from the loss to the averaged weights.

    python examples/federated_head.py

Two groups of two replicas train a next-token model (an embedding, a layer norm and an untied head) on different text.  Per
step and replica, `Embedding.lookup` and `Norm.forward` give the hidden states, `Head.xent_step` computes the loss without
kept logits and writes the head's gradient straight into its unit of the replica's gradient buffer, and `Norm.backward` and
`Embedding.grad` fill the other units; `Session.step` reduces, clips and applies AdamW; every H steps the groups are averaged.  Then a
third group joins that has no text of its own with labels: it is taught by the trained ones on public text, of which only
the teachers' top logits travel (`TopLogits`, then `Head.distill_step`).
"""
from __future__ import annotations

import math
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

from paper_2609_20359_b200.embed import Embedding
from paper_2609_20359_b200.head import Head, TopLogits
from paper_2609_20359_b200.norm import Norm
from paper_2609_20359_b200.session import Session

VOCAB, DIM, BATCH, GROUPS, REPLICAS, PERIOD, TOP = 1031, 128, 384, 2, 2, 4, 16
DEV = "cuda:0"


class Text:
    """Synthetic text: each token has a few likely successors; the groups share half of them."""

    def __init__(self, group: int):
        g = torch.Generator(device=DEV).manual_seed(7)
        shared = torch.randint(0, VOCAB, (VOCAB, 2), generator=g, device=DEV)
        self.gen = torch.Generator(device=DEV).manual_seed(100 + group)
        own = torch.randint(0, VOCAB, (VOCAB, 2), generator=self.gen, device=DEV)
        self.next = torch.cat([shared, own], 1)

    def batch(self):
        """(tokens, next tokens); one in ten has no label, as padding has none."""
        tok = torch.randint(0, VOCAB, (BATCH,), generator=self.gen, device=DEV)
        pick = torch.randint(0, 4, (BATCH,), generator=self.gen, device=DEV)
        label = self.next[tok, pick]
        hidden = torch.rand(BATCH, generator=self.gen, device=DEV) < 0.1
        return tok, torch.where(hidden, -100, label)


SHAPES = [(VOCAB, DIM), (VOCAB, DIM), (DIM,), (DIM,)]       # head, embedding, the norm's weight and bias
UNITS = [math.prod(shape) for shape in SHAPES]


def unit(s: Session, flat: torch.Tensor, u: int) -> torch.Tensor:
    """Unit u of a flat buffer in parameter order (gradients, bf16 parameters) in its own shape."""
    off = s.layout["unit_offset"][u]
    return flat[off: off + UNITS[u]].view(SHAPES[u])


def new_session(groups: int, seed: int) -> Session:
    """A plan whose groups start from the same random parameters; the fp32 copy is held shard by shard."""
    s = Session(sum(UNITS), UNITS, groups=groups, shard_dim=REPLICAS, sync_period=PERIOD, lr=1e-2, weight_decay=0.0)
    lay, g = s.layout, torch.Generator(device=DEV).manual_seed(seed)
    for u, (mean, scale) in enumerate(((0.0, 0.1), (0.0, 1.0), (1.0, 0.0), (0.0, 0.0))):
        x = mean + scale * torch.randn(UNITS[u], generator=g, device=DEV)
        m = lay["unit_shard_numel"][u]
        padded = torch.zeros(REPLICAS * m, device=DEV)
        padded[:UNITS[u]] = x
        for c in range(groups):
            unit(s, s.param_bf16[c], u).copy_(x.view(SHAPES[u]))
            for r in range(REPLICAS):
                at = r * lay["shard_numel"] + lay["unit_shard_offset"][u]
                s.master[c][at: at + m].copy_(padded[r * m: (r + 1) * m])
    return s


def main(steps: int = 48, distill_steps: int = 40, quiet: bool = False):
    s, student = new_session(GROUPS, 1), new_session(1, 2)
    head = Head(BATCH, VOCAB, DIM, top=TOP, device=DEV)
    top_logits = TopLogits(BATCH, VOCAB, TOP, device=DEV)
    embedding, norm = Embedding(BATCH, VOCAB, DIM, device=DEV), Norm(BATCH, DIM, device=DEV)
    text = [Text(c) for c in range(GROUPS)]
    grad_hidden = torch.empty(BATCH, DIM, dtype=torch.bfloat16, device=DEV)

    def forward(sess, p, tok):
        """Hidden states, and what the backward pass takes: embedded rows and their statistics."""
        x = embedding.lookup(tok, unit(sess, p, 1))
        hidden, mean, rstd = norm.forward(x, unit(sess, p, 2), unit(sess, p, 3))
        return hidden, (x, mean, rstd)

    def backward(sess, p, flat, tok, kept):
        """From grad_hidden to the other units of the gradient buffer."""
        x, mean, rstd = kept
        grad_x = norm.backward(x, unit(sess, p, 2), mean, rstd, grad_hidden, unit(sess, flat, 2), unit(sess, flat, 3))
        embedding.grad(tok, grad_x, unit(sess, flat, 1))

    history = []
    for t in range(steps):
        losses = []
        for c in range(GROUPS):
            p = s.param_bf16[c]
            for flat in s.grads[c]:
                tok, label = text[c].batch()
                hidden, kept = forward(s, p, tok)
                loss, _ = head.xent_step(hidden, unit(s, p, 0), label, grad_hidden, unit(s, flat, 0))
                backward(s, p, flat, tok, kept)
                losses.append(loss.sum() / head.rows_taking_part())
        if (t + 1) % PERIOD == 0:
            s.step_fedavg(sample_counts=[1] * GROUPS)
        else:
            s.step()
        history.append(torch.stack(losses).mean())

    taught = []
    p = student.param_bf16[0]
    for t in range(distill_steps):
        for k, flat in enumerate(student.grads[0]):           # replica k listens to group k
            public, _ = text[k].batch()
            q = s.param_bf16[k]
            # what a group sends: TOP values and indices and one number per token
            value, index, lse = top_logits(forward(s, q, public)[0].float() @ unit(s, q, 0).float().t(), temperature=2.0)
            hidden, kept = forward(student, p, public)
            loss, _ = head.distill_step(hidden, unit(student, p, 0), index, value, grad_hidden, unit(student, flat, 0), teacher_lse=lse,
                                        temperature=2.0)
            backward(student, p, flat, public, kept)
            taught.append(loss.mean())
        student.step()

    history = [float(x) for x in history]
    taught = [float(x) for x in taught]
    assert head.status() == 0 and s.status() == 0 and student.status() == 0
    if not quiet:
        print("loss   ", " ".join(f"{x:.3f}" for x in history[::8]), "->", f"{history[-1]:.3f}")
        print("distill", " ".join(f"{x:.3f}" for x in taught[::16]), "->", f"{taught[-1]:.3f}")
    for x in (head, embedding, norm, s, student):
        x.close()
    return history, taught


if __name__ == "__main__":
    main()
