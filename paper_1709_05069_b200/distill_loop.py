"""Workers that distil a student from a teacher, under the Server step.

The Worker's side and the Server's side together.  A teacher's logits over a vocabulary are scored once
(``qn_logprobs``: its top tokens with their log probabilities, the entropy, and the log probability of sampled tokens);
after that only those few numbers a row are kept of it.  The student is one matrix W [vocab][dim] on the same features X, and
theta is W as one vector.  Each Worker evaluates its loss and gradient at its own theta_k: logits = X W^T, then

* ``--objective distill``: ``qn_distill`` against the teacher's top tokens, the gradient in the logits' place;
* ``--objective tokens``: the negative log probability of the sampled tokens, ``qn_logprobs`` forward and
  ``qn_logprobs_backward``, less a little entropy;

and g_k = dlogits^T X.  The Server keeps the m latest (theta_k, g_k) and steps as in ``closed_loop`` (``qn_push``,
``qn_update_window``); ``lam > 1`` is SGD on the window's means, beside it.  The step is Newton's on the window's directions
and SGD on all others, both times tau: tau stays near 1 and the loss is scaled to a Hessian of about 1 (``--scale``).

    python -m paper_1709_05069_b200.distill_loop [--vocab 4096] [--dim 16] [--rows 512] [--steps 40] [--workers 8]
"""
from __future__ import annotations

import argparse
from typing import List, Tuple

import torch

from . import qn

ENTROPY_BONUS = 1e-2


class Problem:
    """Features, the teacher's record, and the buffers of one Worker (all of one GPU)."""

    def __init__(self, vocab: int = 4096, dim: int = 16, rows: int = 512, top: int = 32, temperature: float = 1.0,
                 seed: int = 1, dtype: torch.dtype = torch.float32, scale: float = 1.0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.vocab, self.dim, self.rows, self.temperature, self.dtype = vocab, dim, rows, temperature, dtype
        self.x = torch.randn((rows, dim), generator=gen, device="cuda") / dim ** 0.5
        teacher = 3.0 * torch.randn((vocab, dim), generator=gen, device="cuda")
        logits = (self.x @ teacher.t()).to(dtype)
        noise = torch.empty_like(logits, dtype=torch.float32).exponential_(generator=gen).log()
        self.tokens = (logits.float() / temperature - noise).argmax(1)  # an answer sampled from the teacher
        self.top_token = torch.empty((rows, top), dtype=torch.int64, device="cuda")
        self.top_logprob = torch.empty((rows, top), device="cuda")
        self.teacher_logprob, self.lse, self.entropy = (torch.empty(rows, device="cuda") for _ in range(3))
        qn.qn_logprobs(logits, self.tokens, self.teacher_logprob, entropy=self.entropy, top_token=self.top_token,
                       top_logprob=self.top_logprob, temperature=temperature)
        self.teacher_entropy = self.entropy.clone()
        self.loss, self.logprob = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
        self.weight = torch.full((rows,), scale / rows, device="cuda")
        self.n = vocab * dim

    def logits(self, theta: torch.Tensor) -> torch.Tensor:
        return (self.x @ theta.view(self.vocab, self.dim).t().float()).to(self.dtype)

    def worker(self, theta: torch.Tensor, objective: str) -> torch.Tensor:
        """The gradient of ``scale`` times the mean loss at ``theta`` (as one vector)."""
        z = self.logits(theta)
        if objective == "distill":
            qn.qn_distill(z, self.top_token, self.top_logprob, self.loss, dlogits=z, weight=self.weight,
                          temperature=self.temperature)
        else:
            qn.qn_logprobs_backward(z, z, tokens=self.tokens, d_logprob=-self.weight,
                                    d_entropy=-ENTROPY_BONUS * self.weight, temperature=self.temperature)
        return (z.float().t() @ self.x).reshape(-1)

    def value(self, theta: torch.Tensor, objective: str) -> float:
        """The mean loss at ``theta``."""
        z = self.logits(theta)
        if objective == "distill":
            qn.qn_distill(z, self.top_token, self.top_logprob, self.loss, temperature=self.temperature)
            return float(self.loss.mean())
        qn.qn_logprobs(z, self.tokens, self.logprob, entropy=self.entropy, temperature=self.temperature)
        return float(-self.logprob.mean() - ENTROPY_BONUS * self.entropy.mean())


def run(problem: Problem, objective: str, m: int, tau: float, lam: float, steps: int, spread: float = 1e-2,
        seed: int = 7) -> Tuple[float, List[float]]:
    """The loss at the start and after each of ``steps`` Server updates with m Workers."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    n = problem.n

    def near(theta: torch.Tensor) -> torch.Tensor:
        return theta + spread * torch.randn(n, generator=gen, device="cuda")

    theta = torch.zeros(n, device="cuda")
    start, losses = problem.value(theta, objective), []
    with qn.qn_create(n, m, torch.float32) as h:
        for _ in range(m):
            at = near(theta)
            qn.qn_push(h, -1, at, problem.worker(at, objective))
        for _ in range(steps):
            qn.qn_update_window(h, tau, lam, theta)
            losses.append(problem.value(theta, objective))
            at = near(theta)
            qn.qn_push(h, -1, at, problem.worker(at, objective))
    return start, losses


def main(argv=None) -> None:
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    ap.add_argument("--vocab", type=int, default=4096)
    ap.add_argument("--dim", type=int, default=16)
    ap.add_argument("--rows", type=int, default=512)
    ap.add_argument("--top", type=int, default=32)
    ap.add_argument("--steps", type=int, default=40)
    ap.add_argument("--workers", type=int, default=8)
    ap.add_argument("--tau", type=float, default=1.0)
    ap.add_argument("--scale", type=float, default=300.0)
    ap.add_argument("--lam", type=float, default=0.05)
    ap.add_argument("--objective", choices=("distill", "tokens"), default="distill")
    ap.add_argument("--dtype", choices=("f32", "bf16"), default="f32")
    a = ap.parse_args(argv)
    p = Problem(a.vocab, a.dim, a.rows, a.top, dtype=torch.float32 if a.dtype == "f32" else torch.bfloat16,
                scale=a.scale)
    print("teacher: mean entropy %.3f, mean log probability of its tokens %.3f" % (float(p.teacher_entropy.mean()),
                                                                                  float(p.teacher_logprob.mean())))
    marks = [t for t in (1, 2, 5, 10, 20, 40, 80) if t <= a.steps]
    print("%-28s%12s" % ("mean loss after t updates", "t = 0") + "".join("%12s" % ("t = %d" % t) for t in marks))
    for name, lam in (("SGD (j = 0)", 2.0), ("m = %d, lambda = %g" % (a.workers, a.lam), a.lam)):
        start, losses = run(p, a.objective, a.workers, a.tau, lam, a.steps)
        print("%-28s%12.4f" % (name, start) + "".join("%12.4f" % losses[t - 1] for t in marks))


if __name__ == "__main__":
    main()
