"""A small student with routed experts learns from the top logits that are kept of a teacher: the selection and the operators on rows of logits together.

    python -m paper_2501_14336_amd.distill_example [--steps N]

* once, ``topk`` keeps the k largest logits of each of the teacher's rows, and ``logprobs`` their rows' log-sum;
* each step, ``route`` picks two of the student's experts for a token (and counts them, which moves the bias that balances them), and ``distill_step`` gives
  the loss and the gradient to the student's logits, which goes on to its weights and, through the experts' weights, to the router;
* in the end ``logprobs`` scores the teacher's best token under the student, with the entropy and the student's own best tokens.
"""
from __future__ import annotations

import argparse

import torch

from . import binding as B
from . import operators as O


class RoutedStudent(torch.nn.Module):
    """Token -> logits of the next one: an embedding, two of a few experts, and the output's matrix."""

    def __init__(self, vocab, width, experts, chosen):
        super().__init__()
        self.embedding = torch.nn.Embedding(vocab, width)
        self.router = torch.nn.Linear(width, experts, bias=False)
        self.experts = torch.nn.ModuleList(torch.nn.Sequential(torch.nn.Linear(width, 2 * width), torch.nn.SiLU(), torch.nn.Linear(2 * width, width)) for _ in range(experts))
        self.out = torch.nn.Linear(width, vocab)
        self.chosen = chosen
        self.register_buffer("bias", torch.zeros(experts))
        self.register_buffer("counts", torch.zeros(experts, dtype=torch.int64))

    def forward(self, tokens):
        x = self.embedding(tokens)
        weights, at = O.route(self.router(x), self.chosen, score="sigmoid", bias=self.bias, counts=self.counts)
        y = x
        for e, expert in enumerate(self.experts):     # (every expert on every token: an example's sizes)
            y = y + (weights * (at == e)).sum(1, keepdim=True) * expert(x)
        return self.out(y)

    def balance(self, rate=0.01):
        """Experts with more than their share become less likely to be chosen, without a term in the loss."""
        self.bias += rate * torch.sign(self.counts.double().mean() - self.counts).float()
        self.counts.zero_()


def run(steps=200, vocab=2000, width=64, experts=8, chosen=2, kept=50, batch=512, temperature=1.0, seed=0, device="cuda"):
    """Losses per step, how often each expert was chosen in the last one, and the last scores."""
    torch.manual_seed(seed)
    factors = torch.randn((2, vocab, 16), device=device)
    teacher = factors[0] @ factors[1].T               # logits of the next token, a row per token
    values, indices, _ = B.topk(teacher, kept)
    stats = O.logprobs(teacher, temperature=temperature).row_stats
    lse = stats[:, 0] / temperature + stats[:, 1].log()

    student = RoutedStudent(vocab, width, experts, chosen).to(device)
    optimizer = torch.optim.Adam(student.parameters(), lr=3e-3)
    row_weights = torch.full((batch,), 1.0 / batch, device=device)
    losses = []
    for _ in range(steps):
        tokens = torch.randint(0, vocab, (batch,), device=device)
        logits = student(tokens)
        loss, grad = O.distill_step(logits.detach(), values[tokens], indices[tokens], row_weights, lse[tokens], temperature)
        optimizer.zero_grad()
        logits.backward(grad)
        optimizer.step()
        used = student.counts.clone()
        student.balance()
        losses.append((row_weights * loss).sum())
    with torch.no_grad():
        best = indices.gather(1, values.argmax(1, keepdim=True))
        scores = O.logprobs(student(torch.arange(vocab, device=device)), best, k=5, entropy=True)
    return torch.stack(losses).tolist(), used, best, scores


def main():
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    p.add_argument("--steps", type=int, default=200)
    losses, used, best, scores = run(p.parse_args().steps)
    for i in range(0, len(losses), max(1, len(losses) // 10)):
        print("step %4d  divergence from the teacher %.4f" % (i, losses[i]))
    print("step %4d  divergence from the teacher %.4f" % (len(losses) - 1, losses[-1]))
    print("tokens of the last step per expert:", used.tolist())
    print("the teacher's best token under the student: log probability %.3f on average, among its 5 best in %.1f%% of rows; entropy %.3f" % (
        float(scores.logprobs.mean()), 100 * float((scores.top_indices == best).any(1).float().mean()), float(scores.entropy.mean())))


if __name__ == "__main__":
    main()
