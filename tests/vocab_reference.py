"""Plain 64-bit forms of the operators over a vocabulary, and inputs for their tests."""
import math

import torch

INF = math.inf


def softmax64(logits, temperature):
    """(u - m, p, ln S, m) of u = z / T in float64, with an empty row's p = 0."""
    z = logits.double()
    m = z.amax(1, keepdim=True)
    m = torch.where(m == -INF, torch.zeros_like(m), m)
    d = (z - m) / temperature
    total = d.exp().sum(1, keepdim=True)
    return d, torch.where(total == 0, torch.zeros_like(d), d.exp() / total), total.log(), m / temperature


def xlogy(a, b):
    return torch.special.xlogy(a, b)


def logprobs64(logits, tokens, k, temperature):
    """logprob, lse, entropy, top_token, top_logprob by definition."""
    rows, vocab = logits.shape
    d, p, log_s, m = softmax64(logits, temperature)
    bad = ~torch.isfinite(log_s) & (log_s != -INF)  # a NaN or +inf in the row
    bad = bad[:, 0]
    empty = (logits == -INF).all(1)
    nan = torch.full((rows,), math.nan, dtype=torch.float64, device=logits.device)
    lse = torch.where(bad, nan, (m + log_s)[:, 0])
    entropy = torch.where(bad, nan, -xlogy(p, p).sum(1))
    inside = tokens.clamp(0, vocab - 1)[:, None]
    lp = (d - log_s).gather(1, inside)[:, 0]
    lp = torch.where(empty, torch.full_like(lp, -INF), lp)
    lp = torch.where(bad | (tokens >= vocab), nan, lp)
    lp = torch.where(tokens < 0, torch.zeros_like(lp), lp)
    kept = min(k, vocab)
    order = torch.sort(torch.where(bad[:, None], torch.zeros_like(d), logits.double() + 0.0), dim=1, descending=True,
                       stable=True).indices[:, :kept]
    masked = logits.gather(1, order) == -INF
    top_lp = torch.where(masked, torch.full((), -INF, dtype=torch.float64, device=d.device), (d - log_s).gather(1, order))
    top = torch.where(masked, -1, order)
    top_lp[bad] = math.nan
    top[bad] = -1
    fill = (rows, k - kept)
    top = torch.cat([top, torch.full(fill, -1, dtype=top.dtype, device=d.device)], 1)
    last = torch.where(bad, nan, torch.full_like(nan, -INF))[:, None].expand(fill)
    return lp, lse, entropy, top, torch.cat([top_lp, last], 1)


def backward64(logits, tokens, temperature, d_logprob, d_lse, d_entropy, top_token, d_top):
    """(gradient, sum of the magnitudes of its terms)."""
    rows, vocab = logits.shape
    d, p, log_s, _ = softmax64(logits, temperature)
    entropy = -xlogy(p, p).sum(1, keepdim=True)
    logp = torch.where(p > 0, d - log_s, torch.zeros_like(d))
    zero = torch.zeros((rows, 1), dtype=torch.float64, device=p.device)
    dlp = zero if d_logprob is None else torch.where(tokens >= 0, d_logprob.double(), 0.0)[:, None]
    dl = zero if d_lse is None else d_lse.double()[:, None]
    dh = zero if d_entropy is None else d_entropy.double()[:, None]
    sparse, size = torch.zeros_like(p), torch.zeros_like(p)
    if d_logprob is not None:
        sparse.scatter_add_(1, tokens.clamp(min=0)[:, None], dlp)
        size.scatter_add_(1, tokens.clamp(min=0)[:, None], dlp.abs())
    dt = zero
    if d_top is not None:
        dt = torch.where(top_token >= 0, d_top.double(), 0.0)
        sparse.scatter_add_(1, top_token.clamp(min=0), dt)
        size.scatter_add_(1, top_token.clamp(min=0), dt.abs())
    grad = (sparse + p * (dl - dlp - dt.sum(1, keepdim=True)) - dh * p * (logp + entropy)) / temperature
    size = (size + p * (dl.abs() + dlp.abs() + dt.abs().sum(1, keepdim=True))
            + dh.abs() * p * (logp.abs() + entropy)) / temperature
    none = (dlp == 0) & (dl == 0) & (dh == 0) & (dt == 0).all(1, keepdim=True)
    return torch.where(none, torch.zeros_like(grad), grad), size


def distill64(logits, token, value, logprobs, temperature, weight):
    """loss, gradient, and bounds on the sizes of the terms that each of them adds up."""
    rows, vocab = logits.shape
    d, p, log_s, _ = softmax64(logits, temperature)
    logp = d - log_s
    here = token >= 0
    at = token.clamp(min=0)
    v = torch.where(here, value.double(), -INF)
    if logprobs:
        logq, q = v, v.exp()
        rest = (1.0 - q.sum(1)).clamp(min=0.0)
        rest = torch.where(here.sum(1) == vocab, torch.zeros_like(rest), rest)
    else:
        top = v.amax(1, keepdim=True)
        top = torch.where(top == -INF, torch.zeros_like(top), top)
        logq = torch.log_softmax((v - top) / temperature, 1)
        q = torch.where(v > -INF, logq.exp(), 0.0)
        rest = torch.zeros(rows, dtype=torch.float64, device=p.device)
    on = torch.zeros_like(p).scatter_add_(1, at, here.double())
    q_all = torch.zeros_like(p).scatter_add_(1, at, torch.where(here, q, 0.0))
    lp = logp.gather(1, at)
    terms = torch.where(q > 0, q * (logq - lp), 0.0)
    empty = (logits == -INF).all(1)
    terms = torch.where((q > 0) & empty[:, None], INF, terms)
    p_rest = (p * (1.0 - on)).sum(1)
    tail = torch.where(rest > 0, xlogy(rest, rest) - rest * p_rest.log(), 0.0)
    loss = terms.sum(1) + tail
    mass = (q.sum(1) + rest)[:, None]
    ratio = torch.where((rest > 0) & (p_rest > 0), rest / p_rest, 0.0)[:, None]
    unit = (torch.ones(rows, dtype=torch.float64, device=p.device) if weight is None else weight.double())[:, None]
    grad = unit / temperature * (mass * p - q_all - (1.0 - on) * p * ratio)
    size = unit.abs() / temperature * (mass * p + q_all + (1.0 - on) * p * ratio)
    # 1 - sum q is known to a few 1e-7, whatever is left of it
    slack = unit.abs() / temperature * torch.where((rest > 0) & (p_rest > 0), 1.0 / p_rest, 0.0)[:, None] * p * (1 - on)
    loss_size = torch.where(q > 0, q * (logq.abs() + lp.abs()), 0.0).sum(1) \
        + (rest + 0.2) * (torch.where(rest > 0, rest.log().abs() + p_rest.log().abs(), 0.0))
    if logprobs:
        none = here.sum(1) == 0
    else:
        none = (v == -INF).all(1)
    skip = none | (unit[:, 0] == 0)
    grad = torch.where(empty[:, None] | skip[:, None], 0.0, grad)
    return torch.where(skip, 0.0, loss), grad, loss_size, size, slack


def make_logits(rows, vocab, dtype, seed, pad=0, offset=0, spread=3.0, device="cuda"):
    """Random logits whose rows start ``pad`` elements apart from each other's ends and ``offset`` elements into their
    storage."""
    gen = torch.Generator(device=device).manual_seed(seed)
    store = torch.randn(offset + rows * (vocab + pad), generator=gen, device=device).mul_(spread).to(dtype)
    return store.as_strided((rows, vocab), (vocab + pad, 1), offset)
