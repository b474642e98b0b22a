"""The policy loss, the preference loss and AdamW steps in the loop of Workers (paper_1709_05069_b200.distill_loop)."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def loop():
    from paper_1709_05069_b200 import distill_loop

    return distill_loop


@pytest.mark.parametrize("objective", ["policy", "preference"])
def test_worker_gradient_is_the_derivative_of_its_loss(loop, objective):
    """g against torch's derivative of the same loss in 64 bits: every element within 1e-5 of the largest (fp32 logits
    and one fp32 product over 99 rows).  Rows that are clipped (or not) by less than 1e-4 would be undecided: there are none."""
    p = loop.Problem(vocab=301, dim=8, rows=99, top=16, temperature=1.5)
    theta = 0.5 * torch.randn(p.n, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda")
    g = p.worker(theta, objective)
    w = theta.double().view(p.vocab, p.dim).requires_grad_()
    logp = torch.log_softmax(p.x.double() @ w.t() / p.temperature, 1)
    drawn, taught = logp.gather(1, p.drawn[:, None])[:, 0], logp.gather(1, p.tokens[:, None])[:, 0]
    if objective == "policy":
        x = drawn + math.log(p.vocab)
        r, a = x.exp(), p.advantage.double()
        assert not bool((((r - 0.8).abs() < 1e-4) | ((r - 1.2).abs() < 1e-4)).any())
        loss = torch.maximum(-a * r, -a * r.clamp(0.8, 1.2)) + loop.KL * ((-x).exp() + x - 1) + loop.ENTROPY_BONUS * (logp.exp() * logp).sum(1)
    else:
        edges = list(range(0, p.rows, loop.ANSWER)) + [p.rows]
        d = (taught - drawn)
        loss = -torch.nn.functional.logsigmoid(loop.BETA * torch.stack([d[a:b].sum() for a, b in zip(edges, edges[1:])]))
    want, = torch.autograd.grad(loss.mean(), w)
    assert float((g.double() - want.reshape(-1)).abs().max()) <= 1e-5 * float(want.abs().max())
    assert abs(p.value(theta, objective) - float(loss.detach().mean())) <= 1e-5 * (1 + abs(float(loss.detach().mean())))


@pytest.mark.parametrize("objective", ["distill", "tokens", "policy", "preference"])
def test_every_objective_runs_under_the_server_and_under_adamw(loop, objective):
    p = loop.Problem(vocab=515, dim=5, rows=130, top=8)
    start, losses = loop.run(p, objective, m=4, tau=1.0, lam=0.05, steps=3)
    assert len(losses) == 3 and all(x == x for x in losses)
    for bits in (32, 8):
        again, by_adam = loop.run_adam(p, objective, 1e-2, 4, bits)
        assert again == start and len(by_adam) == 4 and all(math.isfinite(x) for x in by_adam)


def test_first_step_of_the_loop_moves_by_the_learning_rate(loop):
    """From zero states, clipped or not, m' / sqrt(v') is the gradient's sign; in the loop theta starts at 0."""
    p = loop.Problem(vocab=300, dim=7, rows=64, top=8)
    g = p.worker(torch.zeros(p.n, device="cuda"), "preference")
    seen = []
    keep, p.value = p.value, lambda theta, objective: (seen.append(theta.clone()), 0.0)[1]
    loop.run_adam(p, "preference", 0.125, 1, 8)
    p.value = keep
    sure = g.abs() > 1e-3 * g.abs().max()
    assert torch.allclose(seen[1][sure], -0.125 * torch.sign(g[sure]), atol=2e-3)


def test_command_line(loop, capsys):
    loop.main(["--vocab", "256", "--dim", "4", "--rows", "40", "--steps", "2", "--workers", "3", "--objective", "policy", "--adam", "0.01",
               "--bits", "8"])
    out = capsys.readouterr().out
    assert "SGD" in out and "AdamW" in out
