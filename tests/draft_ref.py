"""Attention of trees of drafted tokens in 64 bits, sequence by sequence, with the sizes that forward_ref's bounds need."""
import math

import torch

import forward_ref as R


def masks_of(parents):
    """Bits of each node's ancestors and its own, from lists of parents; -1: the sequence's last token, below it or not
    ahead of the node: no node."""
    got = []
    for i, up in enumerate(parents):
        if up == -1:
            got.append(1 << i)
        elif 0 <= up < i and got[up]:
            got.append(got[up] | 1 << i)
        else:
            got.append(0)
    return got


def signed(m):
    return m - (1 << 64) if m >> 63 else m


def attention(q, k, v, n, masks, scale, softcap, slopes):
    """q (drafts, heads, dim), k and v (n + drafts, kv_heads, dim) of one sequence, masks: its nodes' (numbers without a
    sign). Returns out, lse (drafts, heads), worst and weighted sizes."""
    drafts, hq, d = q.shape
    hk, keys = k.shape[1], k.shape[0]
    masks = [m & ((1 << drafts) - 1) for m in masks]
    seen = torch.tensor([[bool(m) and (j < n or bool(m >> (j - n) & 1)) for j in range(keys)] for m in masks],
                        dtype=torch.bool, device=q.device).view(drafts, keys)
    place = torch.tensor(list(range(n)) + [n + bin(m).count("1") - 1 for m in masks], device=q.device).double()
    qd = q.double()
    kd, vd = (torch.where(seen.any(0)[:, None, None], x.double(), 0.0).repeat_interleave(hq // hk, 1) for x in (k, v))
    s = torch.einsum("thd,jhd->htj", qd, kd) * scale
    size = torch.where(seen, torch.einsum("thd,jhd->htj", qd.abs(), kd.abs()) * abs(scale), 0.0)
    worst = size.amax(-1)
    if softcap:
        s = softcap * torch.tanh(s / softcap)
        worst = worst + 8 * softcap
    if slopes is not None:
        bias = slopes.double()[:, None, None] * (place[n:, None] - place).abs()
        s = s - bias
        worst = worst + torch.where(seen, bias, 0.0).amax(-1)
    s = s.masked_fill(~seen, -math.inf)
    lse = torch.logsumexp(s, -1)
    p = torch.where(seen, torch.exp(s - lse.masked_fill(lse == -math.inf, 0.0)[..., None]), 0.0)
    return torch.einsum("htj,jhd->thd", p, vd), lse, worst, torch.einsum("htj,jhd->thd", p, vd.abs())


def check(out, lse, q, k, v, n, masks, softcap=0.0, slopes=None, scale=None, what=""):
    drafts, _, d = q.shape
    want, want_lse, worst, weighted = attention(q, k, v, n, masks, d ** -0.5 if scale is None else scale, softcap, slopes)
    keys = n + drafts
    R.check(out, want, R.attention_bound(want, weighted, worst, q.dtype, d, keys), f"out {what}")
    R.check(lse.transpose(0, 1), want_lse, R.lse_bound(want_lse, worst, d, keys), f"lse {what}")
