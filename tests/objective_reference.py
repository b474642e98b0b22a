"""Plain 64-bit forms of the policy loss and of the preference loss, for the tests.  Independent of the library."""
import math

import torch

from vocab_reference import softmax64

INF = math.inf


def policy64(logits, tokens, old, ref, advantage, weight, temperature, low, high, dual, kl, bonus):
    """loss, log probability, entropy, gradient; and how much of each an error of 1 in the log probability makes, the
    sizes of the gradient's terms, and the ratio."""
    d, p, log_s, _ = softmax64(logits, temperature)
    vocab = logits.shape[1]
    logp = torch.where(p > 0, d - log_s, -INF)
    at = tokens.clamp(0, vocab - 1)[:, None]
    l = logp.gather(1, at)[:, 0]  # noqa: E741
    entropy = -torch.special.xlogy(p, p).sum(1)
    gone = l == -INF
    a = advantage.double()
    r = torch.where(gone, 0.0, (l - old.double()).exp())
    free, held = -a * r, -a * r.clamp(1.0 - low, 1.0 + high)
    loss, slope = torch.maximum(free, held), torch.where(free >= held, free, 0.0)
    if dual:
        beyond = (a < 0) & (loss > -a * dual)
        loss, slope = torch.where(beyond, -a * dual, loss), torch.where(beyond, 0.0, slope)
    loss, slope = torch.where(a == 0, 0.0, loss), torch.where(a == 0, 0.0, slope)
    per, per_slope = (a * r).abs(), (a * r).abs()
    if kl:
        y = torch.where(gone & (ref.double() == -INF), 0.0, ref.double() - l)
        loss = loss + kl * torch.where(y == INF, INF, torch.expm1(y) - y)
        slope = slope - kl * torch.expm1(y)
        per, per_slope = per + kl * torch.expm1(y).abs(), per_slope + kl * y.exp()
    loss = loss - bonus * entropy
    slope = torch.where(gone, 0.0, slope)
    w = (torch.ones_like(a) if weight is None else weight.double()) / temperature
    one = torch.zeros_like(p).scatter_(1, at, 1.0)
    spread = torch.where(p > 0, p * (logp + entropy[:, None]), 0.0)
    grad = w[:, None] * (slope[:, None] * (one - p) + bonus * spread)
    size = w.abs()[:, None] * (slope.abs()[:, None] * (one + p) + abs(bonus) * torch.where(p > 0, p * (logp.abs() + entropy[:, None]), 0.0))
    per_grad = w.abs()[:, None] * torch.where(slope != 0, per_slope, 0.0)[:, None] * (one + p)
    empty = (logits == -INF).all(1)
    grad[empty] = 0.0
    bad = (torch.isnan(log_s) | (log_s == INF))[:, 0] | (tokens >= vocab) | torch.isnan(old) | torch.isnan(advantage)
    if kl:
        bad = bad | torch.isnan(ref)
    loss[bad] = math.nan
    no_row = (torch.isnan(log_s) | (log_s == INF))[:, 0]
    l[no_row | (tokens >= vocab)] = math.nan
    entropy[no_row | (tokens >= vocab)] = math.nan
    grad[bad] = math.nan
    skip = tokens < 0 if weight is None else (tokens < 0) | (weight == 0)
    for x in (loss, l, entropy, grad):
        x[skip] = 0.0
    return loss, l, entropy, grad, per, size, per_grad, r


def preference64(logprob, offsets, ref, weight, pair_weight, kind, beta, margin, smoothing, normalise, split):
    """loss, rewards, gradient; and the sizes of what is added up for each reward."""
    tokens, pairs = logprob.numel(), (offsets.numel() - 1) // 2
    device = logprob.device
    l = logprob.double().clone()  # noqa: E741
    r = torch.zeros_like(l) if ref is None else ref.double()
    w = torch.ones_like(l) if weight is None else weight.double().clone()
    if ref is not None:
        w[(l == -INF) & (r == -INF)] = 0.0
    counts = w != 0
    ratio = torch.where(counts, w * (torch.where(counts, l, 0.0) - torch.where(counts, r, 0.0)), 0.0)
    loss, reward = torch.zeros(pairs, dtype=torch.float64, device=device), torch.zeros(2 * pairs, dtype=torch.float64, device=device)
    size, grad = torch.zeros_like(reward), torch.full((tokens,), 7.0, dtype=torch.float64, device=device)
    at = offsets.tolist()
    for k in range(pairs):
        pw = 1.0 if pair_weight is None else float(pair_weight[k])
        both = (k, pairs + k) if split else (2 * k, 2 * k + 1)
        good = [0 <= at[s] <= at[s + 1] <= tokens for s in both]
        rewards, each = [], []
        for s in both:
            a, b = (at[s], at[s + 1]) if good[both.index(s)] else (0, 0)
            n = float(w[a:b].sum()) if normalise else 1.0
            each.append(beta / n if n != 0 else 0.0)
            rewards.append(each[-1] * float(ratio[a:b].sum()) if each[-1] else 0.0)
            size[s] = abs(each[-1]) * float(ratio[a:b].abs().sum())
        h = rewards[0] - rewards[1] - margin
        if not all(good):
            h = math.nan
        if kind == 0:
            keep, x = 1.0 - smoothing, torch.tensor(h, dtype=torch.float64)
            loss[k] = keep * torch.logaddexp(-x, torch.zeros_like(x))
            slope = -keep * torch.sigmoid(-x)
            if smoothing:
                loss[k] += smoothing * torch.logaddexp(x, torch.zeros_like(x))
                slope = slope + smoothing * torch.sigmoid(x)
        elif kind == 1:
            loss[k], slope = (max(0.0, 1.0 - h), -1.0 if h < 1 else 0.0) if h == h else (math.nan, math.nan)
        else:
            loss[k], slope = ((h - 0.5) / beta) ** 2, 2 * (h - 0.5) / beta ** 2
        for s, sign in zip(both, (1.0, -1.0)):
            reward[s] = rewards[both.index(s)] if all(good) else math.nan
            if good[both.index(s)]:
                a, b = at[s], at[s + 1]
                c = pw * float(slope) * sign * each[both.index(s)]
                grad[a:b] = torch.where(counts[a:b], w[a:b] * c, 0.0)
                if pw == 0:
                    grad[a:b] = 0.0
        if pw == 0:
            loss[k] = 0.0
            reward[both[0]] = reward[both[1]] = 0.0
    return loss, reward, grad, size
