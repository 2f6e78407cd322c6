"""A factorization machine that answers with one field of its data (the next item), taught by a larger one.

    python -m paper_2004_13940_amd.next_item

Rows hold one-hot context fields; the items are a field of their own, which the rows leave open.  The teacher's largest
logits come from ``fm_field_logprobs``, the student learns them through ``fm_forward``, ``fm_field_distill`` and
``fm_gradient``, and is evaluated by the log probabilities and best items of held-out rows."""
from __future__ import annotations

import numpy as np
import torch

from . import binding as B


class NextItem:
    """A model of the items given a row: context factors ``V`` [D x K], item factors ``items`` [C x K], item weights ``w``."""

    def __init__(self, D, C, K, seed, std=0.1):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.K = K
        self.V = torch.randn(D, K, generator=g, device="cuda") * std
        self.items = torch.randn(C, K, generator=g, device="cuda") * std
        self.w = torch.randn(C, generator=g, device="cuda") * std
        self.zero = torch.zeros(1, device="cuda")
        self.no_w = torch.zeros(D, device="cuda")
        self.no_V = torch.zeros(D * K, device="cuda")

    def aggregates(self, rows: B.Matrix, out):
        """G = X V: the items' logits of a row are w_j + <G_i, items_j>."""
        p = B.make_params(self.K, B.FM_LOSS_SQUARED, 0.0, 0.0, 0.0)
        rows.fm_forward(p, None, self.zero, self.no_w, self.V.view(-1), G=out)
        return out

    def step(self, rows: B.Matrix, field: B.Field, ids, teacher, scale, eta, state):
        """One step of gradient descent on the mean divergence from the teacher; returns that mean, on the device."""
        N = rows.N
        if not state:
            new = lambda *size: torch.empty(*size, device="cuda")  # noqa: E731
            state.update(G=new(N, self.K), dG=new(N, self.K), dV=new(self.V.numel()), dI=new(*self.items.shape),
                         dw=new(*self.w.shape), loss=new(N), one=torch.ones(N, device="cuda"),
                         weight=torch.full((N,), 1.0 / N, device="cuda"))
        s = state
        self.aggregates(rows, s["G"].view(-1))
        field.fm_field_distill(s["G"], self.items, ids, teacher, w=self.w, scale=scale, weight=s["weight"], loss=s["loss"],
                               grad_G=s["dG"], grad_V=s["dI"], grad_w=s["dw"])
        # the gradient by V is X^T dG: what fm_gradient computes for multipliers of 1, aggregates dG and no factors
        p = B.make_params(self.K, B.FM_LOSS_SQUARED, 0.0, 0.0, 0.0)
        rows.fm_gradient(p, s["one"], s["dG"].view(-1), self.no_w, self.no_V, grad_V=s["dV"])
        self.V.view(-1).add_(s["dV"], alpha=-eta)
        self.items.add_(s["dI"], alpha=-eta)
        self.w.add_(s["dw"], alpha=-eta)
        return s["loss"].mean()

    def best(self, rows: B.Matrix, field: B.Field, top, ids=None, scale=1.0):
        """The `top` best items of every row with their log probabilities, and those of given items."""
        n = rows.N
        G = self.aggregates(rows, torch.empty(n * self.K, device="cuda")).view(n, self.K)
        out = dict(top_ids=torch.empty(n, top, dtype=torch.int32, device="cuda"), top_logprob=torch.empty(n, top, device="cuda"),
                   entropy=torch.empty(n, device="cuda"))
        if ids is not None:
            out["logprob"] = torch.empty(n, ids.shape[1], device="cuda")
        field.fm_field_logprobs(G, self.items, w=self.w, scale=scale, ids=ids, **out)
        return out


def contexts(rng, N, fields, width):
    """One-hot rows of `fields` fields of `width` columns, Zipf(1.1) inside a field."""
    p = np.arange(1, width + 1) ** -1.1
    col = np.stack([f * width + rng.choice(width, N, p=p / p.sum()) for f in range(fields)], 1).astype(np.int32)
    return np.arange(N + 1, dtype=np.int64) * fields, col.ravel(), np.ones(N * fields, np.float32)


def run(N=20_000, held_out=2_000, fields=8, width=500, C=5_000, K=16, T=16, steps=150, eta=12.0, scale=0.5, seed=1, say=print):
    """Trains a student of latent size K on a teacher of twice that; returns (losses, share of held-out rows whose best item
    for the teacher is among the student's ten best)."""
    rng = np.random.default_rng(seed)
    D = fields * width
    train, test = B.Matrix(N, D, *contexts(rng, N, fields, width)), B.Matrix(held_out, D, *contexts(rng, held_out, fields, width))
    train.fm_build_csc()
    teacher, student = NextItem(D, C, 2 * K, seed + 1, std=0.45), NextItem(D, C, K, seed + 2)
    asked = B.Field(C, 2 * K, max_rows=N, max_top=T, max_entries=0)
    field = B.Field(C, K, max_rows=N, max_top=10, max_entries=T)
    told = teacher.best(train, asked, T)
    losses, state = [], {}
    for step in range(steps):
        losses.append(student.step(train, field, told["top_ids"], told["top_logprob"], scale, eta, state))
        if step % 30 == 0 or step == steps - 1:
            say(f"step {step}: divergence from the teacher {losses[-1].item():.4f}")
    want = teacher.best(test, asked, 1)["top_ids"]
    got = student.best(test, field, 10, ids=want)
    hit = (got["top_ids"] == want).any(1).float().mean().item()
    say(f"held-out rows: the teacher's best item has mean log probability {got['logprob'].mean().item():.3f} and is among the "
        f"student's ten best in {100 * hit:.1f}% (entropy {got['entropy'].mean().item():.2f})")
    for h in (train, test, asked, field):
        h.close()
    return [float(x) for x in losses], hit


if __name__ == "__main__":
    run()
