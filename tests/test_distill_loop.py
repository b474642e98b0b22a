"""The operators over a vocabulary and the Server step together (paper_1709_05069_b200.distill_loop)."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def loop():
    from paper_1709_05069_b200 import distill_loop

    return distill_loop


@pytest.mark.parametrize("objective", ["distill", "tokens"])
def test_worker_gradient_is_the_derivative_of_its_loss(loop, objective):
    """g against torch's derivative of the same loss in 64 bits: every element within 1e-5 of the largest (fp32 logits
    and one fp32 product over 96 rows)."""
    p = loop.Problem(vocab=301, dim=8, rows=96, top=16, temperature=1.5)
    theta = 0.5 * torch.randn(p.n, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda")
    g = p.worker(theta, objective)
    w = theta.double().view(p.vocab, p.dim).requires_grad_()
    logp = torch.log_softmax(p.x.double() @ w.t() / p.temperature, 1)
    if objective == "distill":
        q = p.top_logprob.double().exp()
        rest = 1 - q.sum(1)
        on = torch.zeros_like(logp).scatter_(1, p.top_token, 1.0)
        p_rest = (logp.exp() * (1 - on)).sum(1)
        loss = (q * (p.top_logprob.double() - logp.gather(1, p.top_token))).sum(1) + rest * (rest.log() - p_rest.log())
    else:
        loss = -logp.gather(1, p.tokens[:, None])[:, 0] + loop.ENTROPY_BONUS * (logp.exp() * logp).sum(1)
    want, = torch.autograd.grad(loss.mean(), w)
    assert float((g.double() - want.reshape(-1)).abs().max()) <= 1e-5 * float(want.abs().max())
    assert abs(p.value(theta, objective) - float(loss.detach().mean())) <= 1e-5 * (1 + abs(float(loss.detach().mean())))


@pytest.mark.parametrize("objective", ["distill", "tokens"])
def test_server_steps_on_distilled_gradients_lower_the_loss(loop, objective):
    # tau = 1: the step is Newton's on the window's directions, so the SGD rate of 40 is a scale of the loss
    p = loop.Problem(vocab=1024, dim=8, rows=256, top=32, scale=40.0)
    start, losses = loop.run(p, objective, m=8, tau=1.0, lam=0.05, steps=20)
    sgd_start, sgd = loop.run(p, objective, m=8, tau=1.0, lam=2.0, steps=20)
    assert start == sgd_start and sgd[-1] < start and losses[-1] < start
    assert all(x == x for x in losses)
