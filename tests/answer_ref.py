"""Losses over answers in 64 bits with the bounds that the kernels' results are held to.

A token's log-probability is within LOGP of the exact one: as in test_gpu_forward_loss, (3 + 64 + 4) 2^-24. What is formed
from it in fp32 adds a few roundings of 2^-24 each, counted below.
"""
import math

import torch

import forward_ref as R

E = 2.0 ** -24
LOGP = (3 + 64 + 4) * E


def rows(logits, targets):
    """Targets' log-probabilities (0 where they do not count), rows' log-sums, whether the rows count."""
    x = logits.double()
    lse = torch.logsumexp(x, 1)
    counted = targets >= 0
    logp = x.gather(1, targets.long().clamp(min=0)[:, None])[:, 0] - lse
    return torch.where(counted, logp, 0.0), lse, counted


def gradient(logits, targets, lse, slope, slope_error, scale):
    """slope (1[v = target] - p_v) scale, and its bound. p: exp of x - lse, whose two differences and product with log2 e are
    rounded, beside LOGP; three products and the exponential 8 more. The target's own, -expm1(x - lse), is off by as much
    of p, and two roundings of itself."""
    away = logits.double() - lse[:, None]
    p = torch.exp(away)
    one = torch.zeros_like(p)
    one[torch.arange(len(targets), device=p.device), targets.long().clamp(min=0)] = 1.0
    hit = torch.where(one > 0, -torch.expm1(away), p)                 # |1[v = target] - p|
    sign = 2 * one - 1
    g = torch.where(slope[:, None] == 0, 0.0, scale * slope[:, None] * hit * sign)
    off = abs(scale) * (slope_error[:, None] * hit + slope.abs()[:, None] * p * (LOGP + (3 * away.abs() + 8) * E))
    u, tiny = R.U[logits.dtype], R.TINY[logits.dtype]
    return g, torch.where(slope[:, None] == 0, abs(scale) * slope_error[:, None] * hit, off + (1.0001 * u + 6 * E) * g.abs()) + tiny


def policy(logits, targets, old, advantages, ref, weights, clip, kl, mean, scale=1.0):
    """loss, its bound, grad, its bound, logp."""
    logp, lse, counted = rows(logits, targets)
    a, old = advantages.double(), old.double()
    r = torch.exp(logp - old)
    lo, hi = 1 - clip[0], 1 + clip[1]
    flat = ((a > 0) & (r > hi)) | ((a < 0) & (r < lo))
    value = -a * torch.where(flat, torch.where(a > 0, hi, lo), r)
    slope = torch.where(flat, 0.0, -a * r)
    # r: LOGP, the difference's rounding, the exponential's 2 and a product's
    error = a.abs() * torch.maximum(r, torch.tensor(hi, device=r.device)) * (LOGP + ((logp - old).abs() + 6) * E)
    value_error = error.clone()
    if kl:
        d = ref.double() - logp
        value = value + kl * (torch.expm1(d) - d)
        slope = slope - kl * torch.expm1(d)
        # exp(d) - 1: as r; exp(d) - 1 - d moves by exp(d) - 1 per unit of d and has 8 roundings of its own, or of the
        # two parts that it is the difference of where they are no less than a quarter
        error = error + kl * (torch.exp(d) * (LOGP + (d.abs() + 6) * E) + 4 * torch.expm1(d).abs() * E)
        parts = torch.where(d.abs() >= 0.25, torch.expm1(d).abs() + d.abs(), torch.expm1(d) - d)
        value_error = value_error + kl * (torch.expm1(d).abs() * (LOGP + (d.abs() + 4) * E) + 8 * parts * E) + 3 * value.abs() * E
    w = torch.where(counted, torch.ones_like(a) if weights is None else weights.double(), 0.0)
    if mean:
        w = w / w.sum()
    keep = counted & (w != 0)
    loss = torch.where(keep, w * value, 0.0).sum()
    bound = torch.where(keep, w.abs() * (value_error + 2 * value.abs() * E), 0.0).sum()
    slope, error = (torch.where(keep, x, 0.0) for x in (w * slope, w.abs() * error))
    return (loss, bound, *gradient(logits, targets, lse, slope, error + 4 * slope.abs() * E, scale), logp)


def preference(logits, targets, starts, ref, beta, margin, smoothing, by_length, mean, scale=1.0):
    """loss, its bound, grad, its bound, the answers' sums, their bounds."""
    logp, lse, counted = rows(logits, targets)
    at = torch.arange(len(targets), device=logits.device)
    starts = starts.long()
    member = ((at >= starts[:-1, None]) & (at < starts[1:, None]) & counted).double()
    n = member.sum(1).clamp(min=1)
    share = member / n[:, None] if by_length else member
    sums = share @ logp
    off = share.sum(1) * LOGP
    away = sums - (0 if ref is None else ref.double())
    m = beta * (away[0::2] - away[1::2]) - margin
    m_off = beta * (off[0::2] + off[1::2]) + m.abs() * E
    soft = lambda x: torch.clamp(x, min=0) + torch.log1p(torch.exp(-x.abs()))  # noqa: E731
    each = (1 - smoothing) * soft(-m) + smoothing * soft(m)
    over = 1.0 / len(m) if mean else 1.0
    slope = beta * over * (smoothing * torch.sigmoid(m) - (1 - smoothing) * torch.sigmoid(-m))
    # the logistic function moves by at most its own value (or 1/4) per unit, and has 5 roundings and the exponential's
    part = beta * over * (smoothing * torch.sigmoid(m) + (1 - smoothing) * torch.sigmoid(-m))
    slope_off = part * (m_off + (m.abs() + 8) * E)
    token = torch.stack([slope, -slope], 1).flatten() @ share
    token_off = torch.stack([slope_off, slope_off], 1).flatten() @ share
    loss = each.sum() * over
    bound = (over * (m_off + 6 * each * E + m.abs() * E)).sum()
    return (loss, bound, *gradient(logits, targets, lse, token, token_off + 4 * token.abs() * E, scale), sums, off + sums.abs() * E)


def close(got, want, bound, what=""):
    assert abs(float(got) - float(want)) <= float(bound) + 1e-13 * abs(float(want)), (what, float(got), float(want), float(bound))
