"""Plain 64-bit implementations of the forward point's operators and the bounds that the kernels' results are held to.

Unit roundoffs u: 2^-8 bf16, 2^-11 fp16, 2^-24 fp32. A result that is formed in fp32 and rounded once is within u of the
exact one, relative, plus what fp32 lost on the way; each bound below says what that is. fp16 results below its normal
range are rounded to multiples of 2^-24, half of one of which is added.
"""
import math

import torch

U = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -25}


def rotate(x, weight, table, positions, eps, layout):
    """(result, size of the pair that each element was formed from), fp64; table None: norm alone."""
    y = x.double()
    if weight is not None:
        y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + eps) * weight.double()
    out, size = y.clone(), y.abs()
    if table is not None:
        r = table.shape[1]
        i = torch.arange(r // 2, device=x.device)
        a, b = (i, i + r // 2) if layout == "half" else (2 * i, 2 * i + 1)
        row = table.double()[positions.long()][:, None]
        c, s = row[..., : r // 2], row[..., r // 2:]
        out[..., a], out[..., b] = y[..., a] * c - y[..., b] * s, y[..., b] * c + y[..., a] * s
        pair = (y[..., a].abs() + y[..., b].abs()) * (c.abs() + s.abs())
        size[..., a], size[..., b] = pair, pair
    return out, size


def rotate_bound(exact, size, dtype, dim):
    """The sum of squares has at most dim + 8 roundings on positive terms (halved by the root), the root, the weight, the
    products and the sum of a pair six more: (dim / 2 + 12) 2^-24 of the pair's size."""
    return U[dtype] * exact.abs() * 1.0001 + (dim / 2 + 12) * 2.0 ** -24 * size + TINY[dtype]


def attention(q, k, v, first, end, self_, scale, softcap, slopes):
    """One fp64 result per query row: out, lse, and the sizes that the bounds need."""
    t, hq, d = q.shape
    hk, n = k.shape[1], k.shape[0]
    qd, kd, vd = q.double(), k.double().repeat_interleave(hq // hk, 1), v.double().repeat_interleave(hq // hk, 1)
    s = torch.einsum("thd,jhd->htj", qd, kd) * scale
    at = torch.arange(n, device=q.device)
    seen = (at >= first[:, None]) & (at < end[:, None])
    size = torch.where(seen, torch.einsum("thd,jhd->htj", qd.abs(), kd.abs()) * abs(scale), 0.0)
    worst = size.amax(-1) if n else torch.zeros(hq, t, dtype=torch.float64, device=q.device)
    if softcap:
        s = softcap * torch.tanh(s / softcap)
        worst = worst + 8 * softcap
    if slopes is not None:
        bias = slopes.double()[:, None, None] * (self_[:, None] - at).abs().double()
        s = s - bias
        if n:
            worst = worst + torch.where(seen, bias, 0.0).amax(-1)
    s = s.masked_fill(~seen, -math.inf)
    if not n:
        return (torch.zeros_like(qd), torch.full((hq, t), -math.inf, dtype=torch.float64, device=q.device), worst,
                torch.zeros_like(qd))
    lse = torch.logsumexp(s, -1)
    p = torch.where(seen, torch.exp(s - lse.masked_fill(lse == -math.inf, 0.0)[..., None]), 0.0)
    return torch.einsum("htj,jhd->thd", p, vd), lse, worst, torch.einsum("htj,jhd->thd", p, vd.abs())


def score_error(worst, dim):
    """Of a score in fp32: a sum of dim products, the scale, cap and bias and the exponent's own rounding, each within
    2^-24 of the largest size that the row forms; the exponential's 2^-21 beside them."""
    return (dim + 16) * 2.0 ** -24 * worst + 2.0 ** -21


def attention_bound(exact, weighted, worst, dtype, dim, keys):
    """Weights are off by the score's error, by their rounding to 16 bits, and their sums by 2^-24 per key."""
    e = score_error(worst, dim).transpose(0, 1)[..., None]
    p = U[dtype] if dtype != torch.float32 else 0.0
    return U[dtype] * 1.0001 * exact.abs() + (p + 2.5 * e + (2 * keys + 8) * 2.0 ** -24) * weighted + TINY[dtype]


def lse_bound(lse, worst, dim, keys):
    finite = lse.masked_fill(lse == -math.inf, 0.0).abs()
    return 1.5 * score_error(worst, dim) + (keys + 8) * 2.0 ** -24 + 4 * 2.0 ** -24 * (finite + worst)


def check(got, exact, bound, what=""):
    """Every element within its bound; infinities where the exact one has them."""
    got = got.double()
    inf = torch.isinf(exact)
    assert torch.equal(got[inf], exact[inf]), what
    off = (got - exact).abs()[~inf]
    ok = off <= bound[~inf]
    assert bool(ok.all()), f"{what}: off by up to {float((off / bound[~inf])[~ok].max() if ok.numel() else 0):.3g} of the bound at " \
                           f"{int((~ok).sum())} of {ok.numel()} (nan {int(torch.isnan(off).sum())})"
