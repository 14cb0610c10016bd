"""Operators for learning from a decoder's own answers -- making them over a paged cache, and the losses that are formed
from them -- as cases that can be timed and compared: in their plain form (elementary torch operations in 32 bits), or
through paper_2609_38095_gb300.forward where `own` is true.

  draft       a tree of drafted tokens per sequence over a paged key-value cache: each sees the sequence so far, its
              ancestors and itself
  policy      the clipped policy loss of answers' tokens with a KL term against a reference, and its gradient in the logits
  preference  the loss of pairs of answers, a preferred and a rejected one, by their log-ratios, and its gradient in the
              logits

Head counts and vocabularies are those of the decoders that workloads.py describes (32 query and 8 key-value heads of 128;
32, 40 or 56 heads of 64 or 128; vocabularies 151936 and 50272) or generic.
"""
import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
IGNORE = -1


def listed():
    return [
        # one sequence being answered, eight drafted tokens verified at once
        {"name": "draft one", "op": "draft", "batch": 1, "longest": 2039, "drafts": 8, "split": 1, "heads": 32,
         "kv_heads": 8, "dim": 128, "page": 16, "dtype": "bf16", "softcap": 0.0, "slopes": False},
        # answers of unequal lengths with trees of unequal sizes, a key-value head each, scores capped and biased
        {"name": "draft batch", "op": "draft", "batch": 16, "longest": 4001, "drafts": 26, "split": 2, "heads": 32,
         "kv_heads": 32, "dim": 64, "page": 16, "dtype": "f16", "softcap": 50.0, "slopes": True},
        # long answers, the widest trees
        {"name": "draft long", "op": "draft", "batch": 16, "longest": 16_384, "drafts": 64, "split": 3, "heads": 32,
         "kv_heads": 8, "dim": 128, "page": 64, "dtype": "bf16", "softcap": 0.0, "slopes": False},
        # an evaluation in full precision, odd pages
        {"name": "draft f32", "op": "draft", "batch": 3, "longest": 777, "drafts": 5, "split": 4, "heads": 16,
         "kv_heads": 4, "dim": 80, "page": 24, "dtype": "f32", "softcap": 0.0, "slopes": True},
        # a few answers' tokens, in full precision: one loss of a step's table
        {"name": "policy few", "op": "policy", "tokens": 16, "vocab": 50_272, "every": 0, "kl": 0.0, "weights": False,
         "mean": True, "grad": False, "dtype": "f32"},
        # the same of a micro-batch: one token in four is a prompt's
        {"name": "policy batch", "op": "policy", "tokens": 4091, "vocab": 151_936, "every": 4, "kl": 0.04,
         "weights": True, "mean": False, "grad": False, "dtype": "bf16"},
        # a smaller model's micro-batch, with the gradient
        {"name": "policy grad", "op": "policy", "tokens": 509, "vocab": 50_272, "every": 7, "kl": 0.0, "weights": False,
         "mean": True, "grad": True, "dtype": "f16"},
        # "policy batch" with the gradient
        {"name": "policy grad batch", "op": "policy", "tokens": 4091, "vocab": 151_936, "every": 4, "kl": 0.04,
         "weights": True, "mean": False, "grad": True, "dtype": "bf16"},
        # one pair of short answers in full precision
        {"name": "preference one", "op": "preference", "pairs": 1, "longest": 24, "split": 5, "pad": 0,
         "vocab": 50_272, "smoothing": 0.0, "by_length": False, "mean": False, "grad": False, "dtype": "f32"},
        # a micro-batch of ragged pairs, every answer's log-probability by its length
        {"name": "preference batch", "op": "preference", "pairs": 8, "longest": 384, "split": 6, "pad": 5,
         "vocab": 151_936, "smoothing": 0.0, "by_length": True, "mean": True, "grad": False, "dtype": "bf16"},
        # a smaller model's pairs with the gradient, labels not quite trusted
        {"name": "preference grad", "op": "preference", "pairs": 4, "longest": 96, "split": 7, "pad": 3,
         "vocab": 50_272, "smoothing": 0.1, "by_length": False, "mean": True, "grad": True, "dtype": "f16"},
        # "preference batch" with the gradient
        {"name": "preference grad batch", "op": "preference", "pairs": 8, "longest": 384, "split": 8, "pad": 5,
         "vocab": 151_936, "smoothing": 0.0, "by_length": False, "mean": True, "grad": True, "dtype": "bf16"},
    ]


def _log_uniform(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["draft", "draft", "policy", "preference"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f16", "f32"])
    if op == "draft":
        heads, kv = rng.choice([(32, 8), (32, 32), (40, 40), (16, 4), (8, 1), (12, 4), (7, 7)])
        batch = _log_uniform(rng, 1, 32)
        most = (60_000 if kv <= 8 else 24_000) // (4 if dtype == "f32" else 1)
        return {"op": op, "batch": batch, "longest": _log_uniform(rng, 1, min(16_000, most // batch)),
                "drafts": _log_uniform(rng, 1, 64), "split": rng.randrange(1 << 20), "heads": heads, "kv_heads": kv,
                "dim": rng.choice([64, 80, 96, 128, 128]), "page": rng.choice([1, 16, 24, 64, 256]), "dtype": dtype,
                "softcap": rng.choice([0.0, 0.0, 30.0]), "slopes": rng.random() < 0.3}
    vocab = rng.choice([50_272, 151_936, _log_uniform(rng, 100, 150_000) | 1])
    grad = rng.random() < 0.6
    tokens = _log_uniform(rng, 1, min(8000, 250_000_000 // vocab // (2 if dtype == "f32" else 1)))
    if op == "policy":
        return {"op": op, "tokens": tokens, "vocab": vocab, "every": rng.choice([0, 2, 4, 7]),
                "kl": rng.choice([0.0, 0.02, 0.1]), "weights": rng.random() < 0.5, "mean": rng.random() < 0.5,
                "grad": grad, "dtype": dtype}
    pairs = _log_uniform(rng, 1, 40)
    return {"op": op, "pairs": pairs, "longest": max(2, tokens // pairs // 2), "split": rng.randrange(1 << 20),
            "pad": rng.choice([0, 0, rng.randint(1, 20)]), "vocab": vocab, "smoothing": rng.choice([0.0, 0.0, 0.1]),
            "by_length": rng.random() < 0.4, "mean": rng.random() < 0.5, "grad": grad, "dtype": dtype}


# ---- what a case describes ---------------------------------------------------------------------------------------


def _lengths(case, n):
    """The sequences' lengths: one of the longest, the others anything from one token on."""
    rng = random.Random(case["split"])
    got = [case["longest"]] + [rng.randint(1, case["longest"]) for _ in range(n - 1)]
    rng.shuffle(got)
    return got


def _parents(case):
    """For each sequence, its nodes' parents (-1: the sequence's last token): chains, stars and what lies between; one
    tree has all the nodes there is room for, the others anything from one on."""
    rng = random.Random(case["split"] + 1)
    sizes = [case["drafts"]] + [rng.randint(1, case["drafts"]) for _ in range(case["batch"] - 1)]
    rng.shuffle(sizes)
    got = []
    for n in sizes:
        back = rng.choice([1, 2, 4, 64])
        got.append([rng.randint(max(-1, i - back), i - 1) for i in range(n)])
    return got


def _masks(parents):
    """A node's bits: its ancestors' and its own."""
    masks = []
    for i, up in enumerate(parents):
        masks.append((masks[up] if up >= 0 else 0) | 1 << i)
    return masks


def _counted(case):
    """Per token whether it counts: of policies' tokens all but one in `every`, of a sequence's tokens those behind its
    first quarter (a prompt's)."""
    if case["op"] == "policy":
        return [not case["every"] or (t + 1) % case["every"] > 0 for t in range(case["tokens"])]
    return [i >= n // 4 for n in _lengths(case, 2 * case["pairs"]) for i in range(n)] + [False] * case["pad"]


def work(case):
    size = SIZE[case["dtype"]]
    if case["op"] == "draft":
        d, trees = case["dim"], _parents(case)
        keys = sum(_lengths(case, case["batch"])) + sum(len(t) for t in trees)
        pairs = sum(n * len(t) + sum(bin(m).count("1") for m in _masks(t)) for n, t in zip(_lengths(case, case["batch"]), trees))
        rows = case["batch"] * case["drafts"] * case["heads"]
        return {"bytes": 2 * (keys * case["kv_heads"] + rows) * d * size + 4 * rows + 4 * -(-keys // case["page"]),
                "flops": 4 * pairs * case["heads"] * d}
    counted = _counted(case)
    t, n, vocab = len(counted), sum(counted), case["vocab"]
    return {"bytes": (n + (t if case["grad"] else 0)) * vocab * size + 24 * t, "flops": (6 if case["grad"] else 4) * n * vocab}


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(g, *shape, dtype, scale=1.0):
    x = torch.randn(*shape, generator=g, device="cuda", dtype=dtype if dtype != torch.float16 else torch.float32)
    return x.mul_(scale).to(dtype)


def _slopes(heads):
    return torch.tensor([2.0 ** (-8.0 * (h + 1) / heads) for h in range(heads)], device="cuda")


def _prepare_draft(case, seed):
    g, dtype = _gen(seed), DTYPES[case["dtype"]]
    b, page, hk, d, drafts = case["batch"], case["page"], case["kv_heads"], case["dim"], case["drafts"]
    lens = _lengths(case, b)
    need = [-(-(n + drafts) // page) for n in lens]
    perm = torch.randperm(sum(need) + 3, generator=g, device="cuda").to(torch.int32)
    table = torch.zeros(b, max(need), dtype=torch.int32, device="cuda")
    at = 0
    for i, n in enumerate(need):
        table[i, :n] = perm[at:at + n]
        at += n
    masks = [m + [0] * (drafts - len(m)) for m in map(_masks, _parents(case))]
    signed = [[v - (1 << 64) if v >> 63 else v for v in m] for m in masks]
    return {"case": case, "q": _randn(g, b, drafts, case["heads"], d, dtype=dtype, scale=1.5),
            "k_cache": _randn(g, sum(need) + 3, page, hk, d, dtype=dtype),
            "v_cache": _randn(g, sum(need) + 3, page, hk, d, dtype=dtype), "pages": table,
            "lengths": torch.tensor(lens, dtype=torch.int32, device="cuda"),
            "masks": torch.tensor(signed, dtype=torch.int64, device="cuda"),
            "slopes": _slopes(case["heads"]) if case["slopes"] else None}


def _prepare_logits(case, seed):
    """Logits under which the answers' tokens are likely, as they are where they were sampled, and their log-probabilities."""
    g, dtype = _gen(seed), DTYPES[case["dtype"]]
    counted = torch.tensor(_counted(case), device="cuda")
    t, vocab = len(counted), case["vocab"]
    targets = torch.randint(0, vocab, (t,), generator=g, device="cuda")
    logits = _randn(g, t, vocab, dtype=dtype, scale=2.0)
    rows = torch.arange(t, device="cuda")
    logits[rows, targets] = (logits[rows, targets].float() + 2 + 8 * torch.rand(t, generator=g, device="cuda")).to(dtype)
    total = torch.cat([x.float().logsumexp(1) for x in logits.split(512)])
    logp = (logits[rows, targets].float() - total).masked_fill(~counted, 0.0)
    targets[~counted] = IGNORE
    return g, logits, targets, logp


def _prepare_policy(case, seed):
    g, logits, targets, logp = _prepare_logits(case, seed)
    t = len(targets)
    # the policy that gave the answers is a few updates old; no ratio lies so near a border of the clipping that 32 bits
    # could not tell its side
    ratio = torch.exp(0.15 * torch.randn(t, generator=g, device="cuda"))
    for border in (0.8, 1.28):
        ratio = torch.where((ratio / border - 1).abs() < 1e-3, ratio * 1.01, ratio)
    per = 64  # an answer's tokens share its advantage; that of answers as good as their group's is zero
    advantage = torch.randn(-(-t // per), generator=g, device="cuda")
    advantage[3::7] = 0.0
    state = {"case": case, "logits": logits, "targets": targets, "old": logp - torch.log(ratio),
             "advantages": advantage.repeat_interleave(per)[:t].contiguous(), "ref": None, "weights": None}
    if case["kl"]:
        state["ref"] = logp + 0.2 * torch.randn(t, generator=g, device="cuda")
    if case["weights"]:
        state["weights"] = 1.0 / torch.randint(16, 257, (-(-t // per),), generator=g, device="cuda").repeat_interleave(per)[:t].float()
    return state


def _prepare_preference(case, seed):
    g, logits, targets, logp = _prepare_logits(case, seed)
    lens = _lengths(case, 2 * case["pairs"])
    starts = torch.tensor([0] + lens, device="cuda").cumsum(0).to(torch.int32)
    sums = torch.stack([x.double().sum() for x in logp[:sum(lens)].split(lens)])
    if case["by_length"]:
        sums = sums / torch.tensor([max(1, n - n // 4) for n in lens], device="cuda")
    # the reference is the model before this training: its answers' log-probabilities are some units away
    ref = sums + (0.3 if case["by_length"] else 8.0) * torch.randn(len(lens), generator=g, device="cuda")
    return {"case": case, "logits": logits, "targets": targets, "starts": starts, "ref": ref.float()}


CLIP = (0.2, 0.28)


def _beta(case):
    return 2.0 if case["by_length"] else 0.1


def prepare(case, seed):
    return {"draft": _prepare_draft, "policy": _prepare_policy, "preference": _prepare_preference}[case["op"]](case, seed)


# ---- one pass ----------------------------------------------------------------------------------------------------


def run(state):
    case = state["case"]
    return (_own if own else _plain)[case["op"]](state, case)


def _plain_draft(state, case):
    b, drafts, hq, d = state["q"].shape
    hk, page = case["kv_heads"], case["page"]
    pages = state["pages"].long()
    k, v = (state[n][pages].float().flatten(1, 2).permute(2, 0, 1, 3) for n in ("k_cache", "v_cache"))  # hk, b, keys, d
    keys = k.shape[2]
    q = state["q"].float().permute(2, 0, 1, 3).reshape(hk, hq // hk, b, drafts, d)
    s = torch.matmul(q.permute(0, 2, 1, 3, 4).reshape(hk, b, -1, d) * d ** -0.5, k.transpose(2, 3))
    s = s.view(hk, b, hq // hk, drafts, keys)
    if case["softcap"]:
        s = case["softcap"] * torch.tanh(s / case["softcap"])
    at = torch.arange(keys, device="cuda")
    node = at - state["lengths"].long()[:, None]  # b, keys: a key's node, negative ahead of them
    is_node = (node >= 0) & (node < drafts)
    bits = (state["masks"][:, :, None] >> node.clamp(0, 63)[:, None, :]) & 1  # b, drafts, keys
    seen = ((node < 0)[:, None, :] & (state["masks"] != 0)[:, :, None]) | (is_node[:, None, :] & (bits == 1))
    if state["slopes"] is not None:
        depth = ((state["masks"][:, :, None] >> torch.arange(64, device="cuda")) & 1).sum(-1) - 1  # b, drafts
        own_depth = torch.where(is_node, depth.gather(1, node.clamp(0, drafts - 1)), node)  # from the end of the sequence
        distance = (depth[:, :, None] - own_depth[:, None, :]).abs().float()
        s = s - state["slopes"].view(hk, 1, -1, 1, 1) * distance[None, :, None]
    s = s.masked_fill(~seen[None, :, None], -math.inf)
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s - top.masked_fill(top == -math.inf, 0.0))
    total = p.sum(-1, keepdim=True)
    v = v.masked_fill(~seen.any(1)[None, :, :, None], 0.0)  # rows of the pages that are nobody's
    out = torch.matmul(p.view(hk, b, -1, keys), v).view(hk, b, hq // hk, drafts, d) / total.masked_fill(total == 0, 1.0)
    lse = (top + torch.log(total)).squeeze(-1).masked_fill(top.squeeze(-1) == -math.inf, -math.inf)
    return {"out": out.permute(1, 3, 0, 2, 4).reshape(b, drafts, hq, d).to(state["q"].dtype),
            "lse": lse.permute(1, 3, 0, 2).reshape(b, drafts, hq)}


def _plain_logp(state):
    """Weights exp(x - top) of each row, their sums, and the targets' log-probabilities (0 where they do not count)."""
    x = state["logits"].float()
    counted = state["targets"] != IGNORE
    top = x.amax(1, keepdim=True)
    picked = (x.gather(1, state["targets"].clamp(min=0)[:, None]) - top)[:, 0]
    e = torch.exp(x - top)
    total = e.sum(1, keepdim=True)
    return e, total, (picked - torch.log(total[:, 0])).masked_fill(~counted, 0.0), counted


def _plain_grad(e, total, state, coefficient):
    """coefficient (1[v = target] - p_v) per token."""
    p = e.div_(total).neg_()
    p.scatter_add_(1, state["targets"].clamp(min=0)[:, None], torch.ones_like(total))
    return p.mul_(coefficient[:, None]).to(state["logits"].dtype)


def _plain_policy(state, case):
    e, total, logp, counted = _plain_logp(state)
    a, ratio = state["advantages"], torch.exp(logp - state["old"])
    whole, cut = ratio * a, ratio.clamp(1 - CLIP[0], 1 + CLIP[1]) * a
    value = -torch.minimum(whole, cut)
    slope = torch.where(whole <= cut, -whole, torch.zeros_like(whole))
    if state["ref"] is not None:
        away = state["ref"] - logp
        value = value + case["kl"] * (torch.exp(away) - away - 1)
        slope = slope + case["kl"] * (1 - torch.exp(away))
    weight = torch.ones_like(logp) if state["weights"] is None else state["weights"]
    weight = torch.where(counted, weight, torch.zeros_like(weight)).double()
    if case["mean"]:
        weight = weight / weight.sum()
    loss = (weight * value).sum(0, keepdim=True).float()
    if not case["grad"]:
        return {"loss": loss, "logp": logp}
    return {"loss": loss, "grad": _plain_grad(e, total, state, (weight * slope).float()), "logp": logp}


def _plain_preference(state, case):
    e, total, logp, counted = _plain_logp(state)
    at, starts = torch.arange(len(logp), device="cuda"), state["starts"].long()
    member = ((at >= starts[:-1, None]) & (at < starts[1:, None]) & counted).double()  # sequences, tokens
    sums = member @ logp.double()
    if case["by_length"]:
        share = member / member.sum(1, keepdim=True).clamp(min=1)
        sums = sums / member.sum(1).clamp(min=1)
    else:
        share = member
    ratio = sums - state["ref"]
    m = _beta(case) * (ratio[0::2] - ratio[1::2])
    eps = case["smoothing"]
    over = case["pairs"] if case["mean"] else 1
    loss = ((1 - eps) * torch.log1p(torch.exp(-m)) + eps * torch.log1p(torch.exp(m))).sum(0, keepdim=True) / over
    if not case["grad"]:
        return {"loss": loss.float(), "logp": sums.float()}
    slope = _beta(case) * (eps / (1 + torch.exp(-m)) - (1 - eps) / (1 + torch.exp(m))) / over
    slope = torch.stack([slope, -slope], 1).flatten()
    return {"loss": loss.float(), "grad": _plain_grad(e, total, state, (slope @ share).float()), "logp": sums.float()}


def _own_draft(state, case):
    from paper_2609_38095_gb300 import forward
    out, lse = forward.draft_attention(state["q"], state["k_cache"], state["v_cache"], state["pages"], state["lengths"],
                                       state["masks"], softcap=case["softcap"], slopes=state["slopes"], with_lse=True)
    return {"out": out, "lse": lse}


def _own_policy(state, case):
    from paper_2609_38095_gb300 import forward
    got = forward.policy_loss(state["logits"], state["targets"], state["old"], state["advantages"], ref_logp=state["ref"],
                              weights=state["weights"], clip=CLIP, kl=case["kl"], mean=case["mean"], dtype=torch.float32,
                              with_grad=case["grad"], with_logp=True)
    return dict(zip(("loss", "grad", "logp") if case["grad"] else ("loss", "logp"), got))


def _own_preference(state, case):
    from paper_2609_38095_gb300 import forward
    got = forward.preference_loss(state["logits"], state["targets"], state["starts"], ref_logp=state["ref"],
                                  beta=_beta(case), smoothing=case["smoothing"], by_length=case["by_length"],
                                  mean=case["mean"], dtype=torch.float32, with_grad=case["grad"], with_logp=True)
    return dict(zip(("loss", "grad", "logp") if case["grad"] else ("loss", "logp"), got))


_plain = {"draft": _plain_draft, "policy": _plain_policy, "preference": _plain_preference}
_own = {"draft": _own_draft, "policy": _own_policy, "preference": _own_preference}


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------


def exact(case, seed):
    state = prepare(case, seed)
    return {"draft": _exact_draft, "policy": _exact_policy, "preference": _exact_preference}[case["op"]](state, case)


def _exact_draft(state, case):
    """Sequence by sequence and head by head, the trees from their parents."""
    hq, hk, d, page, drafts = case["heads"], case["kv_heads"], case["dim"], case["page"], case["drafts"]
    out = torch.zeros(state["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(state["q"].shape[:3], -math.inf, dtype=torch.float64, device="cuda")
    for b, (n, parents) in enumerate(zip(_lengths(case, case["batch"]), _parents(case))):
        m = len(parents)
        pages = state["pages"][b, :-(-(n + m) // page)].long()
        k, v = (state[c][pages].double().reshape(-1, hk, d)[:n + m] for c in ("k_cache", "v_cache"))
        hidden, depth = [[1] * m for _ in range(m)], []
        for i, up in enumerate(parents):
            depth.append(0 if up < 0 else depth[up] + 1)
            j = i
            while j >= 0:
                hidden[i][j] = 0
                j = parents[j]
        hide = torch.cat([torch.zeros(m, n, device="cuda"), torch.tensor(hidden, device="cuda").float()], 1) > 0
        place = torch.cat([torch.arange(n, device="cuda"), n + torch.tensor(depth, device="cuda")]).double()
        away = (place[n:, None] - place[None, :]).abs()
        for h in range(hq):
            g = h // (hq // hk)
            s = state["q"][b, :m, h].double() @ k[:, g].T / math.sqrt(d)
            if case["softcap"]:
                s = torch.tanh(s / case["softcap"]) * case["softcap"]
            if state["slopes"] is not None:
                s = s - state["slopes"][h].double() * away
            s[hide] = -math.inf
            total = torch.logsumexp(s, 1)
            lse[b, :m, h] = total
            out[b, :m, h] = torch.exp(s - total[:, None]) @ v[:, g]
    return {"out": out, "lse": lse}


def _exact_rows(state):
    """Log-probabilities of the counted targets, and a function of one factor per token: the gradient of the sum of the
    log-probabilities times their factors."""
    targets = state["targets"]
    rows = torch.arange(len(targets), device="cuda")
    total = torch.cat([torch.logsumexp(x.double(), 1) for x in state["logits"].split(128)])
    logp = state["logits"][rows, targets.clamp(min=0)].double() - total

    def gradient(factor):
        got = torch.zeros(state["logits"].shape, dtype=torch.float64, device="cuda")
        for lo in range(0, len(targets), 128):
            part = slice(lo, lo + 128)
            got[part] = -torch.exp(state["logits"][part].double() - total[part, None]) * factor[part, None]
        got[rows, targets.clamp(min=0)] += factor
        return got

    return torch.where(targets >= 0, logp, torch.zeros_like(logp)), targets >= 0, gradient


def _exact_policy(state, case):
    logp, counted, gradient = _exact_rows(state)
    a, old = state["advantages"].double(), state["old"].double()
    ratio = torch.exp(logp - old)
    lo, hi = 1 - CLIP[0], 1 + CLIP[1]
    # the part of the objective that is cut off: above for what should be likelier, below for what should be less likely
    flat = ((a > 0) & (ratio > hi)) | ((a < 0) & (ratio < lo))
    value = -a * torch.where(flat, torch.where(a > 0, torch.full_like(a, hi), torch.full_like(a, lo)), ratio)
    slope = torch.where(flat, torch.zeros_like(a), -a * ratio)
    if state["ref"] is not None:
        away = state["ref"].double() - logp
        value += case["kl"] * (torch.expm1(away) - away)
        slope -= case["kl"] * torch.expm1(away)
    weight = counted.double() if state["weights"] is None else counted * state["weights"].double()
    if case["mean"]:
        weight = weight / weight.sum()
    got = {"loss": (weight * value)[counted].sum()[None], "logp": logp}
    if case["grad"]:
        got["grad"] = gradient(torch.where(counted, weight * slope, torch.zeros_like(slope)))
    return {n: got[n] for n in ("loss", "grad", "logp") if n in got}


def _exact_preference(state, case):
    logp, counted, gradient = _exact_rows(state)
    starts = state["starts"].tolist()
    counts = [max(1, int(counted[a:b].sum())) if case["by_length"] else 1 for a, b in zip(starts, starts[1:])]
    sums = torch.stack([logp[a:b].sum() / n for a, b, n in zip(starts, starts[1:], counts)])
    ratio = (sums - state["ref"].double()).view(-1, 2)
    m = (_beta(case) * (ratio[:, 0] - ratio[:, 1])).requires_grad_()
    e = case["smoothing"]
    each = -(1 - e) * torch.nn.functional.logsigmoid(m) - e * torch.nn.functional.logsigmoid(-m)
    loss = each.mean() if case["mean"] else each.sum()
    got = {"loss": loss.detach()[None], "logp": sums}
    if case["grad"]:
        slope = torch.autograd.grad(loss, m)[0] * _beta(case)
        factor = torch.zeros_like(logp)
        for j, (a, b, n) in enumerate(zip(starts, starts[1:], counts)):
            factor[a:b] = (slope[j // 2] if j % 2 == 0 else -slope[j // 2]) / n
        got["grad"] = gradient(factor * counted)
    return {n: got[n] for n in ("loss", "grad", "logp") if n in got}
