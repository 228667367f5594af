"""One training step's two ends on this library's kernels, and the schedule of the gradient that they share.

    python -m paper_2503_16815_amd.tied_ends [--rows 4096 --vocab 50257 --hidden 768 --k 2 --link-gbs 50]

A language model that ties its head to its token table has one gradient that is far larger than the others:
the table's.  The loss begins it (a piece of the vocabulary after the other), a teacher's top logits add to
it where positions are distilled, and the embedding, the last thing of the backward pass, completes it.  This
program runs those parts of a step around a stand-in for the model's layers (one dense layer in torch),
measures the forward and the backward window, cuts the table's gradient into buckets by pieces of the
vocabulary, and lets the exact solver place them in the windows of k iterations (Sec. III.A, III.B
of the paper).  No row of a shared table is final before the embedding's part has been added, so all buckets
are ready at the end of the backward pass, and the windows are those that follow it; the events of the head's
pieces tell when its part of them is written (of a head with a table of its own: when the bucket is ready).  Inputs
are synthetic.
"""
from __future__ import annotations

import argparse
import json
import sys
from dataclasses import dataclass

import numpy as np
import torch

from . import binding, ends as _ends, workloads as W


@dataclass
class Step:
    """What a program keeps from step to step: the handle, the parameters and the gradients' buffers."""
    ends: _ends.DeftEnds
    table: torch.Tensor       # [vocab][hidden], embedding and head
    mix: torch.Tensor         # [hidden][hidden], the stand-in for the layers
    grad_table: torch.Tensor
    scale: float

    @classmethod
    def create(cls, rows, vocab, hidden, dtype=torch.bfloat16, seed=1, top_k=32):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        table = (torch.randn((vocab, hidden), generator=g, device="cuda") * 0.5).to(dtype)
        mix = (torch.randn((hidden, hidden), generator=g, device="cuda") / hidden ** 0.5).to(dtype)
        ends = _ends.DeftEnds(_ends.OPERATORS, dtype, rows, vocab, hidden, top_k)
        return cls(ends, table, mix, torch.empty_like(table), float(hidden) ** 0.5)

    def forward(self, tokens, labels):
        x = self.ends.embed(tokens, self.table, scale=self.scale)
        hidden = torch.tanh(x @ self.mix)
        loss, lse = self.ends.head_loss(hidden, self.table, labels)
        return x, hidden, loss, lse

    def backward(self, tokens, labels, x, hidden, lse, row_grad, distilled=None, merge=False, piece_events=None):
        """Gradients of sum(row_grad * loss), and of the distilled positions' losses where `distilled` is (positions,
        teacher_index, teacher_logit, row_grad, temperature).  merge: the table's gradient of an earlier iteration,
        whose update is delayed, is added to.  piece_events: recorded as the head's part of each piece of the table's
        gradient is written; the distilled positions' part and the embedding's are added to all pieces after that."""
        grad_hidden, grad_table = self.ends.head_grad(hidden, self.table, labels, lse, row_grad, grad_weight=self.grad_table,
                                                      accumulate=merge, piece_events=piece_events)
        extra = None
        if distilled is not None:
            at, index, value, by, temperature = distilled
            picked = hidden[at]
            logits = picked @ self.table.T
            extra, d = self.ends.distill_grad(logits, index, value, by, temperature, grad_logits=logits)
            grad_hidden.index_add_(0, at, d @ self.table)
            grad_table.addmm_(d.T, picked)
        d = grad_hidden * (1 - hidden * hidden)
        grad_mix = x.T @ d
        self.ends.embed_grad(tokens, d @ self.mix.T, grad_table=grad_table, scale=self.scale, accumulate=True)
        return grad_table, grad_mix, extra


def schedule(step: Step, forward_us: float, backward_us: float, k: int, link_gbs: float):
    """The table's gradient placed by the exact solver in the forward and backward windows of the k iterations after
    the one that computed it, at whose end it is ready; times in 10 us units, value = communication time (Sec. III.B,
    Problem 1).  A piece of the vocabulary is a bucket, cut further where it would take more than a quarter of the
    smaller window (Sec. III.D: a bucket has to fit)."""
    vocab, hidden = step.table.shape
    unit = 10.0
    row_us = hidden * step.table.element_size() / (link_gbs * 1e3)
    piece = min(step.ends.info().vocab_piece, vocab, max(1, int(min(forward_us, backward_us) / 4 / row_us)))
    rows = [min(piece, vocab - at) for at in range(0, vocab, piece)]
    item = np.array([[max(1, round(r * row_us / unit)) for r in rows]], np.int32)
    caps = np.array([[max(1, int(t / unit)) for t in (forward_us, backward_us)] * k], np.int32)
    kb = W.KnapsackBatch("tied_ends", W.MODE_SEQUENTIAL, 1, item.shape[1], 2 * k, np.array([item.shape[1]], np.int32),
                         np.array([2 * k], np.int32), item, item.copy(), caps)
    return kb, binding.solve(kb)


def main(argv=None) -> int:
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, value in (("rows", 4096), ("vocab", 50257), ("hidden", 768), ("k", 2), ("top-k", 32), ("steps", 5)):
        ap.add_argument("--" + name, type=int, default=value)
    ap.add_argument("--link-gbs", type=float, default=50.0, help="rate of the link that the buckets take")
    a = ap.parse_args(argv)
    if not torch.cuda.is_available():
        print("tied_ends: no GPU visible", file=sys.stderr)
        return 1
    step = Step.create(a.rows, a.vocab, a.hidden, top_k=a.top_k)
    g = torch.Generator(device="cuda")
    g.manual_seed(7)
    tokens = torch.randint(0, a.vocab, (a.rows,), generator=g, device="cuda", dtype=torch.int32)
    labels = torch.roll(tokens, -1)
    labels[-1] = -1
    row_grad = torch.full((a.rows,), 1.0 / (a.rows - 1), device="cuda")
    at = torch.arange(0, a.rows, 16, device="cuda")
    top = torch.topk(torch.randn((len(at), a.vocab), generator=g, device="cuda"), a.top_k, dim=1)
    distilled = (at, top.indices.int(), top.values, torch.full((len(at),), 0.5 / len(at), device="cuda"), 2.0)
    pieces = -(-a.vocab // step.ends.info().vocab_piece)
    for n in range(a.steps):
        marks = [torch.cuda.Event(enable_timing=True) for _ in range(3)]
        head_part = [torch.cuda.Event(enable_timing=True) for _ in range(pieces)]
        marks[0].record()
        x, hidden, loss, lse = step.forward(tokens, labels)
        marks[1].record()
        step.backward(tokens, labels, x, hidden, lse, row_grad, distilled, merge=n % a.k != 0, piece_events=head_part)
        marks[2].record()   # (every piece of the table's gradient is final)
    torch.cuda.synchronize()
    forward_us, backward_us = (1e3 * marks[i].elapsed_time(marks[i + 1]) for i in range(2))
    kb, out = schedule(step, forward_us, backward_us, a.k, a.link_gbs)
    print(json.dumps({
        "loss": float(loss.sum() / (a.rows - 1)), "forward_us": forward_us, "backward_us": backward_us,
        "head_part_us": [1e3 * marks[1].elapsed_time(e) for e in head_part], "pieces_ready_us": [backward_us] * pieces,
        "unit_us": 10,
        "bucket_times": kb.weights[0].tolist(), "windows": kb.capacities[0].tolist(),
        "window_of_bucket": out.assignment[0].tolist(), "time_hidden": int(out.total_value[0])}))
    return 0


if __name__ == "__main__":
    sys.exit(main())
