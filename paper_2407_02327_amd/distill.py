"""A quantized head distilled from its full-precision teacher: the operators of `head.py` around a quantized linear.

    python -m paper_2407_02327_amd.distill [--steps 60] [--tokens 1024] [--width 512] [--vocabulary 8192] [--top 64]

The last stretch of a language model, hidden states -> layer norm -> head -> logits, twice: the teacher in half precision, the student
with an INT8 head (forward INT8, backward FP16, the pairing the paper trains with) whose weights start away from the teacher's.  A step:

    teacher   LayerNorm -> QLinear (FP16) -> TokenLogProbs: the top alternatives of every position
    student   LayerNorm, which collects the maximum that the INT8 conversion needs -> QLinear (INT8) -> Distillation: loss and gradient
              -> QLinear.backward -> LayerNorm.backward -> plain gradient descent on the head and the norm

Hidden states are synthetic and the teacher's weights random (there is nothing to download); what is shown is the distance to the teacher
falling: the loss, and how often the student's first alternative is the teacher's.
"""
from __future__ import annotations

import argparse

import torch

from . import qsync as Q
from .head import Distillation, LayerNorm, TokenLogProbs
from .operator import QLinear


class Teacher:
    """Layer norm and half-precision head; answers with the top alternatives of every position."""

    def __init__(self, tokens: int, width: int, vocabulary: int, top: int, generator: torch.Generator):
        self.norm = LayerNorm(tokens, width, training=False)
        self.head = QLinear(Q.FP16, tokens, vocabulary, width, y_dtype=torch.float16, transposed_copies=True)
        self.top = TokenLogProbs(tokens, vocabulary, top_k=top)
        self.w = torch.randn(vocabulary, width, generator=generator, device="cuda") * (3.0 / width ** 0.5)

    def __call__(self, hidden: torch.Tensor):
        logits = self.head.forward(self.norm.forward(hidden), self.w)
        _, _, logp, index = self.top.forward(logits)
        return logp, index


class Student:
    """Layer norm with weights and INT8 head, trained on the teacher's alternatives."""

    def __init__(self, tokens: int, width: int, vocabulary: int, top: int, w: torch.Tensor, loss_scale: float = 1024.0):
        self.norm = LayerNorm(tokens, width, collect_y_amax=True)
        self.head = QLinear(Q.INT8, tokens, vocabulary, width, y_dtype=torch.float16, dy_dtype=torch.float16, bwd_tag=Q.FP16)
        self.loss = Distillation(tokens, vocabulary, top, dlogits_dtype=torch.float16)
        self.first = TokenLogProbs(tokens, vocabulary, top_k=1)
        self.w, self.gamma, self.beta = w, torch.ones(width, device="cuda"), torch.zeros(width, device="cuda")
        # of the mean over the positions, times what keeps its gradient in the range of binary16
        self.weight = torch.full((tokens,), loss_scale / tokens, device="cuda")
        self.loss_scale = loss_scale

    def logits(self, hidden: torch.Tensor) -> torch.Tensor:
        return self.head.forward(self.norm.forward(hidden, self.gamma, self.beta), self.w, x_amax=self.norm.y_amax)

    def step(self, hidden: torch.Tensor, logp: torch.Tensor, index: torch.Tensor, rate: float) -> torch.Tensor:
        losses, dlogits = self.loss.forward_backward(self.logits(hidden), logp, index, self.weight)
        dy, dw, db = self.head.backward(dlogits)
        _, dgamma, dbeta = self.norm.backward(dy)
        for p, g in ((self.w, dw), (self.head.bias, db), (self.gamma, dgamma), (self.beta, dbeta)):
            p.sub_(g, alpha=rate / self.loss_scale)
        return losses

    def agreement(self, hidden: torch.Tensor, index: torch.Tensor) -> torch.Tensor:
        """The share of positions whose first alternative is the teacher's."""
        _, _, _, mine = self.first.forward(self.logits(hidden))
        return (mine[:, 0] == index[:, 0]).float().mean()


def run(steps: int = 60, tokens: int = 1024, width: int = 512, vocabulary: int = 8192, top: int = 64, rate: float = 20.0, seed: int = 0, say=print):
    """Trains on a handful of batches; returns the mean losses of the first and last pass over them and the agreements before and after."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    teacher = Teacher(tokens, width, vocabulary, top, g)
    student = Student(tokens, width, vocabulary, top, teacher.w + torch.randn(vocabulary, width, generator=g, device="cuda") * (2.0 / width ** 0.5))
    batches = [torch.randn(tokens, width, generator=g, device="cuda").half() for _ in range(4)]
    known = [tuple(t.clone() for t in teacher(h)) for h in batches]
    agree = lambda: torch.stack([student.agreement(h, i) for h, (_, i) in zip(batches, known)]).mean().item()
    before, losses = agree(), []
    for n in range(steps):
        hidden, (logp, index) = batches[n % 4], known[n % 4]
        losses.append(student.step(hidden, logp, index, rate).mean())
        if n % 20 == 19 or n == 0:
            say(f"step {n + 1:4d}  loss {losses[-1].item():.4f}")
    after = agree()
    first, last = (torch.stack(part).mean().item() for part in (losses[:4], losses[-4:]))
    say(f"loss {first:.4f} -> {last:.4f}, first alternative as the teacher's {100 * before:.1f} % -> {100 * after:.1f} %")
    return first, last, before, after


def main() -> None:
    parser = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, default in (("steps", 60), ("tokens", 1024), ("width", 512), ("vocabulary", 8192), ("top", 64), ("seed", 0)):
        parser.add_argument(f"--{name}", type=int, default=default)
    parser.add_argument("--rate", type=float, default=20.0)
    run(**vars(parser.parse_args()))


if __name__ == "__main__":
    main()
