"""A language model's head trained by distillation over a thin link: every step in 4 bits.

A student's head (a matrix of `vocab` rows and `hidden` columns) learns from a teacher's top logits.  One round of the worker:

    logits    = X W^T                          X and W quantised to 4 bits along `hidden`
    loss, dZ  = distillation from the teacher's top entries (the gradient takes the place of the logits)
    dX        = dZ W, dW = dZ^T X              dZ, W and X quantised along the axes that are summed over
    update    = 4 bits of dW - h, h += update  (error feedback)

and of the server: its copy of h takes the same update, and the model's weights one step along it.

    python examples/distilled_head.py [--tokens 4096 --hidden 768 --vocab 50257 --entries 32 --rounds 10 --step 200]
"""
from __future__ import annotations

import argparse
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import torch  # noqa: E402

import paper_2312_08053_amd as kimad  # noqa: E402


def both_forms(x):
    """x in 4 bits along its rows and along its columns, from one read."""
    rows, cols = x.shape
    along_rows, along_columns = kimad.mx4_empty(rows, cols, x.device), kimad.mx4_empty(cols, rows, x.device)
    kimad.kimad_mx4_quantise(x, *along_rows, *along_columns)
    return along_rows, along_columns


class Head:
    """The worker's weights and estimator, the server's copy of the estimator, and the buffers between them."""

    def __init__(self, vocab: int, hidden: int, temperature: float = 2.0, step: float = 1.0):
        self.vocab, self.hidden, self.temperature, self.step = vocab, hidden, temperature, step
        d = vocab * hidden
        self.weights = 0.02 * torch.randn(vocab, hidden, device="cuda")
        self.h = torch.zeros(d, device="cuda")
        self.server_h = torch.zeros(d, device="cuda")
        self.layer_start = torch.tensor([0, d], dtype=torch.int64, device="cuda")
        words = kimad.kimad_mx4_update_words(1, d)
        self.codes = torch.empty(words, 64, dtype=torch.uint8, device="cuda")
        self.scales = torch.empty(words, dtype=torch.int32, device="cuda")
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def gradients(self, x, t_idx, t_val, row_weight):
        """Loss of every token, and the gradients for the hidden states and the weights."""
        tokens = x.shape[0]
        x_rows, x_cols = both_forms(x)
        w_rows, w_cols = both_forms(self.weights)
        z = torch.empty(tokens, self.vocab, dtype=torch.bfloat16, device="cuda")
        kimad.kimad_mx4_matmul(*x_rows, *w_rows, self.hidden, z)
        loss = torch.empty(tokens, device="cuda")
        kimad.kimad_distill(z, t_idx, t_val, self.temperature, loss=loss, grad=z, row_weight=row_weight)
        z_rows, z_cols = both_forms(z)
        dx = torch.empty(tokens, self.hidden, dtype=torch.bfloat16, device="cuda")
        kimad.kimad_mx4_matmul(*z_rows, *w_cols, self.vocab, dx)
        dw = torch.empty(self.vocab, self.hidden, device="cuda")
        kimad.kimad_mx4_matmul(*z_cols, *x_cols, tokens, dw)
        return loss, dx, dw

    def round(self, x, t_idx, t_val, row_weight):
        """One round; returns the tokens' losses and the gradient for the hidden states."""
        loss, dx, dw = self.gradients(x, t_idx, t_val, row_weight)
        kimad.kimad_mx4_compress_ef(dw.view(-1), self.h, self.layer_start, self.codes, self.scales, self.status)
        kimad.kimad_mx4_server_apply([(self.codes, self.scales)], [self.server_h], [1.0], self.layer_start, self.h.numel(),
                                     self.weights.view(-1), self.step)
        return loss, dx


def teacher_batch(tokens: int, hidden: int, vocab: int, entries: int, seed: int = 0):
    """Hidden states, the top entries of a teacher that is a head of its own, and the rows' weights (a few rows do not count)."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    x = torch.randn(tokens, hidden, generator=gen, device="cuda")
    teacher = torch.randn(vocab, hidden, generator=gen, device="cuda") * (3.0 / hidden ** 0.5)
    val, idx = (x @ teacher.t()).topk(entries, dim=1)
    weight = torch.where(torch.rand(tokens, generator=gen, device="cuda") < 0.05, 0.0, 1.0 / tokens)
    return x.to(torch.bfloat16), idx.to(torch.int32), val.contiguous(), weight


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, default in (("tokens", 4096), ("hidden", 768), ("vocab", 50257), ("entries", 32), ("rounds", 10)):
        ap.add_argument("--" + name, type=int, default=default)
    ap.add_argument("--step", type=float, default=200.0)
    a = ap.parse_args(argv)
    torch.manual_seed(0)
    head = Head(a.vocab, a.hidden, step=a.step)
    batch = teacher_batch(a.tokens, a.hidden, a.vocab, a.entries)
    losses = []
    for r in range(a.rounds):
        loss, _ = head.round(*batch)
        losses.append(float(loss.sum()))
        print(f"round {r}: loss {losses[-1]:.4f}", flush=True)
    bits = 8 * (head.codes.numel() + 4 * head.scales.numel()) / head.h.numel()
    print(f"{bits:.2f} bits an entry sent; worker and server hold the same estimator: {torch.equal(head.h, head.server_h)}")
    return losses


if __name__ == "__main__":
    main()
