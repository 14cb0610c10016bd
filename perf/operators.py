"""The operators of a forward point -- what lies between the weights that a step perturbs and the loss that its
preconditioner reads -- as cases that can be timed and compared: in their plain form (elementary torch operations in
32 bits), or through paper_2609_38095_gb300.forward where `own` is true.

  rotate     norms of queries and keys for each head and the rotation by position, in one pass; with `append` the keys
             and values go to their slots of a paged cache
  attention  packed documents: causal, or with a prefix that is seen from everywhere in its document, keys cached ahead
             of the new tokens, scores capped by a tanh, a bias by distance, rows that see nothing
  decode     one new token per sequence over a paged key-value cache
  loss       the tokens' negative log-likelihoods from logits, and their sum: one entry of a step's loss table

Head counts and sizes are those of the decoders that workloads.py describes (32 query and 8 key-value heads of 128;
32, 40 or 56 heads of 64 or 128) or generic; vocabularies 151936 and 50272.
"""
import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-6
IGNORE = -1


def listed():
    return [
        # the next token of eight sequences that are being answered: queries rotated, keys and values put into the cache
        {"name": "rotate step", "op": "rotate", "tokens": 8, "heads": 32, "kv_heads": 8, "dim": 128, "rotary": 128,
         "layout": "half", "norm": True, "append": True, "page": 16, "pages": 64, "dtype": "bf16"},
        # a micro-batch of 16 documents of at most 256 tokens, one layer of one forward point
        {"name": "rotate batch", "op": "rotate", "tokens": 4091, "heads": 32, "kv_heads": 8, "dim": 128, "rotary": 128,
         "layout": "half", "norm": True, "append": False, "page": 0, "pages": 0, "dtype": "bf16"},
        # a long packed batch, half of each head rotated by neighbouring pairs
        {"name": "rotate long", "op": "rotate", "tokens": 50_001, "heads": 40, "kv_heads": 40, "dim": 128, "rotary": 64,
         "layout": "interleaved", "norm": True, "append": False, "page": 0, "pages": 0, "dtype": "f16"},
        # three short prompts of a classification task
        {"name": "attention short", "op": "attention", "docs": 3, "longest": 41, "split": 1, "cached": 0, "pad": 3,
         "heads": 32, "kv_heads": 32, "dim": 64, "dtype": "f16", "prefix": False, "softcap": 0.0, "slopes": False},
        # the micro-batch of "rotate batch": ragged documents, grouped heads
        {"name": "attention batch", "op": "attention", "docs": 24, "longest": 256, "split": 2, "cached": 0, "pad": 0,
         "heads": 32, "kv_heads": 8, "dim": 128, "dtype": "bf16", "prefix": False, "softcap": 0.0, "slopes": False},
        # one long document
        {"name": "attention long", "op": "attention", "docs": 1, "longest": 8192, "split": 3, "cached": 0, "pad": 0,
         "heads": 32, "kv_heads": 8, "dim": 128, "dtype": "bf16", "prefix": False, "softcap": 0.0, "slopes": False},
        # a scoring pass in full precision: prompts seen whole by their own tokens, scores capped, a bias by distance
        {"name": "attention capped f32", "op": "attention", "docs": 5, "longest": 333, "split": 4, "cached": 100,
         "pad": 1, "heads": 16, "kv_heads": 4, "dim": 80, "dtype": "f32", "prefix": True, "softcap": 30.0,
         "slopes": True},
        # one sequence being answered
        {"name": "decode one", "op": "decode", "batch": 1, "longest": 2047, "split": 5, "heads": 32, "kv_heads": 8,
         "dim": 128, "page": 16, "dtype": "bf16", "softcap": 0.0, "slopes": False},
        # a batch of answers of unequal lengths, one head each, scores capped and biased
        {"name": "decode batch", "op": "decode", "batch": 16, "longest": 4001, "split": 6, "heads": 32, "kv_heads": 32,
         "dim": 64, "page": 16, "dtype": "f16", "softcap": 50.0, "slopes": True},
        # many sequences with long caches
        {"name": "decode long", "op": "decode", "batch": 48, "longest": 16_384, "split": 7, "heads": 32, "kv_heads": 8,
         "dim": 128, "page": 64, "dtype": "bf16", "softcap": 0.0, "slopes": False},
        # the label tokens of a small evaluation batch, logits in full precision
        {"name": "loss few", "op": "loss", "tokens": 16, "vocab": 50_272, "every": 0, "dtype": "f32"},
        # every token of a micro-batch, one in four masked
        {"name": "loss batch", "op": "loss", "tokens": 4091, "vocab": 151_936, "every": 4, "dtype": "bf16"},
    ]


def _log_uniform(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["rotate", "attention", "decode", "loss"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f16", "f32"])
    heads, kv = rng.choice([(32, 8), (32, 32), (40, 40), (16, 4), (8, 1), (12, 4), (7, 7)])
    dim = rng.choice([64, 80, 96, 128, 128])
    if op == "rotate":
        append = rng.random() < 0.4
        tokens = _log_uniform(rng, 1, 600 if append else 40_000 // (2 if dtype == "f32" else 1))
        page = rng.choice([1, 16, 24, 64])
        return {"op": op, "tokens": tokens, "heads": heads, "kv_heads": kv, "dim": dim,
                "rotary": rng.choice([dim, dim, dim // 2, 32]), "layout": rng.choice(["half", "interleaved"]),
                "norm": rng.random() < 0.6, "append": append, "page": page if append else 0,
                "pages": -(-tokens // page) + rng.randint(0, 9) if append else 0, "dtype": dtype}
    if op == "attention":
        docs = _log_uniform(rng, 1, 40)
        longest = _log_uniform(rng, 3, max(4, (3000 if dtype == "f32" else 6000) // docs))
        return {"op": op, "docs": docs, "longest": longest, "split": rng.randrange(1 << 20),
                "cached": rng.choice([0, 0, rng.randint(1, 500)]), "pad": rng.choice([0, 0, rng.randint(1, 50)]),
                "heads": heads, "kv_heads": kv, "dim": dim, "dtype": dtype, "prefix": rng.random() < 0.3,
                "softcap": rng.choice([0.0, 0.0, 20.0, 50.0]), "slopes": rng.random() < 0.3}
    if op == "decode":
        batch = _log_uniform(rng, 1, 64)
        longest = _log_uniform(rng, 1, min(16_000, 100_000 // batch))
        return {"op": op, "batch": batch, "longest": longest, "split": rng.randrange(1 << 20), "heads": heads,
                "kv_heads": kv, "dim": dim, "page": rng.choice([1, 16, 24, 64, 256]), "dtype": dtype,
                "softcap": rng.choice([0.0, 0.0, 30.0]), "slopes": rng.random() < 0.3}
    vocab = rng.choice([50_272, 151_936, _log_uniform(rng, 100, 150_000) | 1])
    return {"op": op, "tokens": _log_uniform(rng, 1, 250_000_000 // vocab // 2 if vocab > 30_000 else 4000),
            "vocab": vocab, "every": rng.choice([0, 2, 4, 7]), "dtype": dtype}


# ---- what a case describes ---------------------------------------------------------------------------------------


def _lengths(case, n):
    """The documents' or sequences' lengths: one of the longest, the others anything from one token on."""
    rng = random.Random(case["split"])
    got = [case["longest"]] + [rng.randint(1, case["longest"]) for _ in range(n - 1)]
    rng.shuffle(got)
    return got


def _spans(case):
    """For every query row: the first key it sees, the end of those, and its own place among the keys. Rows past the
    last document see nothing."""
    first, end, self_ = [], [], []
    at = 0
    for n in _lengths(case, case["docs"]):
        stop = at + case["cached"] + n
        seen = at + case["cached"] + n // 4 if case["prefix"] else 0
        for i in range(n):
            me = at + case["cached"] + i
            first.append(at)
            end.append(max(me + 1, seen))
            self_.append(me)
        at = stop
    pad = case["pad"]
    return first + [0] * pad, end + [0] * pad, self_ + [0] * pad, at + pad


def work(case):
    size = SIZE[case["dtype"]]
    if case["op"] == "rotate":
        t, d = case["tokens"], case["dim"]
        made = case["heads"] + case["kv_heads"] * (2 if case["append"] else 1)
        return {"bytes": 2 * t * made * d * size + min(t, _rows(case)) * case["rotary"] * 4 + 8 * t,
                "flops": t * (case["heads"] + case["kv_heads"]) * (3 * case["rotary"] + (4 * d if case["norm"] else 0))}
    if case["op"] == "attention":
        first, end, _, keys = _spans(case)
        pairs, t, d = sum(max(0, b - a) for a, b in zip(first, end)), len(first), case["dim"]
        return {"bytes": 2 * (t * case["heads"] + keys * case["kv_heads"]) * d * size + 4 * t * case["heads"] + 8 * t,
                "flops": 4 * pairs * case["heads"] * d}
    if case["op"] == "decode":
        keys, b, d = sum(_lengths(case, case["batch"])), case["batch"], case["dim"]
        return {"bytes": 2 * keys * case["kv_heads"] * d * size + 2 * b * case["heads"] * d * size
                + 4 * -(-keys // case["page"]),
                "flops": 4 * keys * case["heads"] * d}
    t, every = case["tokens"], case["every"]
    counted = t - (-(-t // every) if every else 0)
    return {"bytes": counted * case["vocab"] * size + 12 * t, "flops": 4 * counted * case["vocab"]}


def _rows(case):
    return 4096


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(g, *shape, dtype, scale=1.0):
    x = torch.randn(*shape, generator=g, device="cuda", dtype=dtype if dtype != torch.float16 else torch.float32)
    return x.mul_(scale).to(dtype)


def _slopes(heads):
    return torch.tensor([2.0 ** (-8.0 * (h + 1) / heads) for h in range(heads)], device="cuda")


def prepare(case, seed):
    g, dtype = _gen(seed), DTYPES[case["dtype"]]
    if case["op"] == "rotate":
        t, hq, hk, d, r = case["tokens"], case["heads"], case["kv_heads"], case["dim"], case["rotary"]
        qkv = _randn(g, t, (hq + 2 * hk) * d, dtype=dtype)  # a fused projection's output: q, k and v are views of it
        rows = _rows(case)
        turn = torch.arange(rows, device="cuda", dtype=torch.float64)[:, None] * (
            1e6 ** (-torch.arange(0, r, 2, device="cuda", dtype=torch.float64) / r))
        state = {"case": case, "table": torch.cat([turn.cos(), turn.sin()], 1).float(),
                 "q": qkv[:, :hq * d].view(t, hq, d), "k": qkv[:, hq * d:(hq + hk) * d].view(t, hk, d),
                 "v": qkv[:, (hq + hk) * d:].view(t, hk, d), "wq": None, "wk": None, "slots": None}
        if case["norm"]:
            state["wq"], state["wk"] = ((1 + _randn(g, d, dtype=torch.float32, scale=0.1)).to(dtype) for _ in range(2))
        if case["append"]:
            state["positions"] = torch.randint(0, rows, (t,), generator=g, device="cuda")
            state["slots"] = torch.randperm(case["pages"] * case["page"], generator=g, device="cuda")[:t]
            state["k_cache"], state["v_cache"] = (_randn(g, case["pages"], case["page"], hk, d, dtype=dtype) for _ in range(2))
        else:
            state["positions"] = (torch.arange(t, device="cuda") + seed % 97) % rows
        return state
    if case["op"] == "attention":
        first, end, self_, keys = _spans(case)
        t, hq, hk, d = len(first), case["heads"], case["kv_heads"], case["dim"]
        return {"case": case, "q": _randn(g, t, hq, d, dtype=dtype, scale=1.5), "k": _randn(g, keys, hk, d, dtype=dtype),
                "v": _randn(g, keys, hk, d, dtype=dtype),
                "spans": torch.tensor([first, end, self_], dtype=torch.int32, device="cuda"),
                "slopes": _slopes(hq) if case["slopes"] else None}
    if case["op"] == "decode":
        lens, page, b, hk, d = _lengths(case, case["batch"]), case["page"], case["batch"], case["kv_heads"], case["dim"]
        need = [-(-n // page) for n in lens]
        perm = torch.randperm(sum(need) + 3, generator=g, device="cuda").to(torch.int32)
        table = torch.zeros(b, max(need), dtype=torch.int32, device="cuda")
        at = 0
        for i, n in enumerate(need):
            table[i, :n] = perm[at:at + n]
            at += n
        return {"case": case, "q": _randn(g, b, case["heads"], d, dtype=dtype, scale=1.5),
                "k_cache": _randn(g, sum(need) + 3, page, hk, d, dtype=dtype),
                "v_cache": _randn(g, sum(need) + 3, page, hk, d, dtype=dtype), "pages": table,
                "lengths": torch.tensor(lens, dtype=torch.int32, device="cuda"),
                "slopes": _slopes(case["heads"]) if case["slopes"] else None}
    t = case["tokens"]
    targets = torch.randint(0, case["vocab"], (t,), generator=g, device="cuda")
    if case["every"]:
        targets[::case["every"]] = IGNORE
    return {"case": case, "logits": _randn(g, t, case["vocab"], dtype=dtype, scale=2.0), "targets": targets}


# ---- one pass ----------------------------------------------------------------------------------------------------


def run(state):
    case = state["case"]
    return (_own if own else _plain)[case["op"]](state, case)


def _plain_heads(x, weight, state, case):
    y, r = x.float(), case["rotary"]
    if weight is not None:
        y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + EPS) * weight.float()
    rows = state["table"][state["positions"]][:, None, :]
    cos, sin = rows[..., :r // 2], rows[..., r // 2:]
    if case["layout"] == "half":
        a, b = y[..., :r // 2], y[..., r // 2:r]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    else:
        a, b = y[..., 0:r:2], y[..., 1:r:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    return torch.cat([turned, y[..., r:]], -1).to(x.dtype)


def _plain_rotate(state, case):
    q = _plain_heads(state["q"], state["wq"], state, case)
    k = _plain_heads(state["k"], state["wk"], state, case)
    if not case["append"]:
        return {"q": q, "k": k}
    kc, vc = state["k_cache"], state["v_cache"]
    kc.view(-1, *kc.shape[2:])[state["slots"]] = k
    vc.view(-1, *vc.shape[2:])[state["slots"]] = state["v"]
    return {"q": q, "k_cache": kc, "v_cache": vc}


def _plain_softmax(s, seen, v):
    """softmax(s) v over the seen keys; rows that see none are zero, and their log-sum -inf."""
    s = s.masked_fill(~seen, -math.inf)
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s - top.masked_fill(top == -math.inf, 0.0))
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p, v) / total.masked_fill(total == 0, 1.0)
    return out, (top + torch.log(total)).squeeze(-1).masked_fill(top.squeeze(-1) == -math.inf, -math.inf)


def _plain_scores(q, k, distance, state, case):
    s = torch.matmul(q * (case["dim"] ** -0.5), k)
    if case["softcap"]:
        s = case["softcap"] * torch.tanh(s / case["softcap"])
    return s if state["slopes"] is None else s - state["slopes"].view(distance.shape[0], -1, 1, 1) * distance


def _plain_attention(state, case):
    q, k, v = (state[n].float().transpose(0, 1) for n in "qkv")
    hk, (keys, d), t = k.shape[0], k.shape[1:], q.shape[1]
    first, end, self_ = (x[:, None] for x in state["spans"])
    at = torch.arange(keys, device="cuda", dtype=torch.int32)
    distance = (self_ - at).abs().float().expand(hk, 1, t, keys)
    s = _plain_scores(q.reshape(hk, -1, t, d), k.transpose(1, 2)[:, None], distance, state, case)
    out, lse = _plain_softmax(s, (at >= first) & (at < end), v[:, None])
    return {"out": out.reshape(-1, t, d).transpose(0, 1).contiguous().to(state["q"].dtype), "lse": lse.reshape(-1, t)}


def _plain_decode(state, case):
    b, hk, d = case["batch"], case["kv_heads"], case["dim"]
    pages = state["pages"].long()
    k, v = (state[n][pages].float().flatten(1, 2).permute(2, 0, 1, 3) for n in ("k_cache", "v_cache"))  # hk, b, keys, d
    q = state["q"].float().view(b, hk, -1, d).permute(1, 2, 0, 3)  # hk, group, b, d
    at = torch.arange(k.shape[2], device="cuda", dtype=torch.int32)
    lengths = state["lengths"][:, None]
    s = torch.matmul(q.transpose(1, 2) * d ** -0.5, k.transpose(2, 3)).transpose(1, 2)  # hk, group, b, keys
    if case["softcap"]:
        s = case["softcap"] * torch.tanh(s / case["softcap"])
    if state["slopes"] is not None:
        s = s - state["slopes"].view(hk, -1, 1, 1) * (lengths - 1 - at).float()
    s = s.masked_fill(at >= lengths, -math.inf)
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s - top)
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p.transpose(1, 2), v).transpose(1, 2) / total
    return {"out": out.permute(2, 0, 1, 3).reshape(b, -1, d).to(state["q"].dtype),
            "lse": (top + torch.log(total)).squeeze(-1).permute(2, 0, 1).reshape(b, -1)}


def _plain_loss(state, case):
    x, targets = state["logits"].float(), state["targets"]
    top = x.amax(1, keepdim=True)
    nll = torch.log(torch.exp(x - top).sum(1)) + top[:, 0] - x.gather(1, targets.clamp(min=0)[:, None])[:, 0]
    nll = nll.masked_fill(targets == IGNORE, 0.0)
    return {"loss": nll.sum(0, keepdim=True), "nll": nll}


def _own_rotate(state, case):
    from paper_2609_38095_gb300 import forward
    common = {"table": state["table"], "positions": state["positions"], "q_weight": state["wq"], "k_weight": state["wk"],
              "eps": EPS, "layout": case["layout"]}
    if not case["append"]:
        q, k = forward.rotate_heads(state["q"], state["k"], **common)
        return {"q": q, "k": k}
    q, kc, vc = forward.rotate_heads(state["q"], state["k"], state["v"], k_out=state["k_cache"], v_out=state["v_cache"],
                                     slots=state["slots"], **common)
    return {"q": q, "k_cache": kc, "v_cache": vc}


def _own_attention(state, case):
    from paper_2609_38095_gb300 import forward
    out, lse = forward.attention(state["q"], state["k"], state["v"], state["spans"], softcap=case["softcap"],
                                 slopes=state["slopes"], with_lse=True)
    return {"out": out, "lse": lse}


def _own_decode(state, case):
    from paper_2609_38095_gb300 import forward
    out, lse = forward.decode_attention(state["q"], state["k_cache"], state["v_cache"], state["pages"], state["lengths"],
                                        softcap=case["softcap"], slopes=state["slopes"], with_lse=True)
    return {"out": out, "lse": lse}


def _own_loss(state, case):
    from paper_2609_38095_gb300 import forward
    loss, nll = forward.token_loss(state["logits"], state["targets"], dtype=torch.float32, with_nll=True)
    return {"loss": loss, "nll": nll}


_plain = {"rotate": _plain_rotate, "attention": _plain_attention, "decode": _plain_decode, "loss": _plain_loss}
_own = {"rotate": _own_rotate, "attention": _own_attention, "decode": _own_decode, "loss": _own_loss}


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------


def exact(case, seed):
    state = prepare(case, seed)
    return {"rotate": _exact_rotate, "attention": _exact_attention, "decode": _exact_decode, "loss": _exact_loss}[case["op"]](state, case)


def _exact_rotate(state, case):
    """Each rotated pair as a complex number times e^(i angle), the table's entries as they are."""
    r = case["rotary"]
    row = state["table"].double()[state["positions"]]
    turn = torch.complex(row[:, :r // 2], row[:, r // 2:])
    got = {}
    for name, weight in (("q", state["wq"]), ("k", state["wk"])):
        x = state[name].double()
        if weight is not None:
            x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / case["dim"] + EPS) * weight.double()
        out = x.clone()
        i = torch.arange(r // 2, device="cuda")
        i, j = (i, i + r // 2) if case["layout"] == "half" else (2 * i, 2 * i + 1)
        z = torch.complex(x[..., i], x[..., j]) * turn[:, None, :]
        out[..., i], out[..., j] = z.real, z.imag
        got[name] = out
    if not case["append"]:
        return got
    page, slots = case["page"], state["slots"]
    for name, new in (("k_cache", got["k"]), ("v_cache", state["v"].double())):
        cache = state[name].double()
        cache[slots // page, slots % page] = new
        got[name] = cache
    return {n: got[n] for n in ("q", "k_cache", "v_cache")}


def _exact_rows(q, k, v, seen, distance, slope, case):
    """Rows of queries of one head (n, d) against keys and values (m, d)."""
    s = q @ k.T / math.sqrt(case["dim"])
    if case["softcap"]:
        s = torch.tanh(s / case["softcap"]) * case["softcap"]
    if slope is not None:
        s = s - slope * distance
    s = torch.where(seen, s, torch.full_like(s, -math.inf))
    lse = torch.logsumexp(s, 1)
    return torch.where(seen, torch.exp(s - lse[:, None]), torch.zeros_like(s)) @ v, lse


def _exact_attention(state, case):
    hq, hk = case["heads"], case["kv_heads"]
    q, k, v = (state[n].double() for n in "qkv")
    first, end, self_ = (x.long()[:, None] for x in state["spans"])
    at = torch.arange(k.shape[0], device="cuda")[None, :]
    seen, distance = (at >= first) & (at < end), (self_ - at).abs().double()
    out, lse = torch.zeros_like(q), torch.zeros(hq, q.shape[0], dtype=torch.float64, device="cuda")
    for h in range(hq):
        g = h // (hq // hk)
        slope = None if state["slopes"] is None else state["slopes"][h].double()
        out[:, h], lse[h] = _exact_rows(q[:, h], k[:, g], v[:, g], seen, distance, slope, case)
    return {"out": out, "lse": lse}


def _exact_decode(state, case):
    hq, hk, d, page = case["heads"], case["kv_heads"], case["dim"], case["page"]
    out = torch.zeros(case["batch"], hq, d, dtype=torch.float64, device="cuda")
    lse = torch.zeros(case["batch"], hq, dtype=torch.float64, device="cuda")
    for b, n in enumerate(_lengths(case, case["batch"])):
        pages = state["pages"][b, :-(-n // page)].long()
        k, v = (state[c][pages].double().reshape(-1, hk, d)[:n] for c in ("k_cache", "v_cache"))
        away = torch.arange(n - 1, -1, -1, device="cuda").double()
        for g in range(hk):
            heads = slice(g * (hq // hk), (g + 1) * (hq // hk))
            slope = None if state["slopes"] is None else state["slopes"][heads].double()[:, None]
            seen = torch.ones(hq // hk, n, dtype=torch.bool, device="cuda")
            out[b, heads], lse[b, heads] = _exact_rows(state["q"][b, heads].double(), k[:, g], v[:, g], seen, away, slope, case)
    return {"out": out, "lse": lse}


def _exact_loss(state, case):
    targets, got = state["targets"], []
    for rows, t in zip(state["logits"].split(256), targets.split(256)):
        logp = rows.double() - torch.logsumexp(rows.double(), 1, keepdim=True)
        one = -logp[torch.arange(len(t), device="cuda"), t.clamp(min=0)]
        got.append(torch.where(t == IGNORE, torch.zeros_like(one), one))
    nll = torch.cat(got)
    return {"loss": nll.sum()[None], "nll": nll}
