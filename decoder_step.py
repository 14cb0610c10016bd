"""1.5-SPSA steps of a small decoder whose losses are its own: the library's step (perturb, losses, precondition,
update) around the library's forward point (head norms and rotation, attention of packed documents, token loss), then
an answer of the trained weights, token by token over a paged cache, or several drafted tokens at once. Judged and
Preferred are batches of a model's own answers, whose losses are those of learning from them; a step takes them as it takes
documents.

The model has the shape of the Qwen3 decoder in workloads.py at a small size: untied embedding and head, per layer
q/k/v/o projections, per-head norms of queries and keys, SwiGLU, two RMSNorms. Its matrix products, root-mean-square
norms and activations are torch's. The task is synthetic: in every document the next token is the last one plus the
document's stride, modulo the vocabulary; documents are packed one after another, their first token is not counted.

The schedule is the fused in-place one (Algorithm 1, bit for bit): +eps of probe 0, per probe the -2 eps pass and the
restore folded into the next probe's +eps, the last restore in the update.

    python decoder_step.py                          # a few steps and an answer, JSON lines
    python decoder_step.py --steps 20 --probes 32
    python decoder_step.py --answers policy         # steps on the model's own answers; or: preference
"""
import argparse
import json
import time

import torch

import paper_2609_38095_gb300 as zo
from paper_2609_38095_gb300 import forward

STEP_SEED_BASE = 0x5DEC0000


class Decoder:
    """The model: its weights as one ordered list, and forward points over them."""

    def __init__(self, layers=2, hidden=256, heads=8, kv_heads=2, head_dim=64, inter=512, vocab=512, context=1024,
                 dtype=torch.bfloat16, seed=0):
        self.layers, self.hidden, self.heads, self.kv_heads, self.head_dim = layers, hidden, heads, kv_heads, head_dim
        self.vocab, self.dtype = vocab, dtype
        g = torch.Generator(device="cuda").manual_seed(seed)

        def matrix(rows, cols):
            return (torch.randn(rows, cols, generator=g, device="cuda") * cols ** -0.5).to(dtype)

        ones = lambda n: torch.ones(n, device="cuda", dtype=dtype)  # noqa: E731
        self.w = {"embed": torch.randn(vocab, hidden, generator=g, device="cuda").to(dtype)}
        for i in range(layers):
            self.w |= {f"{i}.qkv": matrix((heads + 2 * kv_heads) * head_dim, hidden), f"{i}.o": matrix(hidden, heads * head_dim),
                       f"{i}.q_norm": ones(head_dim), f"{i}.k_norm": ones(head_dim), f"{i}.gate": matrix(inter, hidden),
                       f"{i}.up": matrix(inter, hidden), f"{i}.down": matrix(hidden, inter), f"{i}.norm1": ones(hidden),
                       f"{i}.norm2": ones(hidden)}
        self.w |= {"norm": ones(hidden), "head": matrix(vocab, hidden)}
        self.params = zo.ParamList(list(self.w.values()))
        self.table = forward.rotary_table(context, head_dim, base=1e6)

    def _rms(self, x, name):
        y = x.float()
        return (y * torch.rsqrt(y.square().mean(-1, keepdim=True) + 1e-6) * self.w[name].float()).to(self.dtype)

    def logits(self, tokens, positions, attend):
        """Logits (tokens, vocab); attend(layer, q, k, v, positions) rotates the heads and attends."""
        n, hq, hk, d = len(tokens), self.heads, self.kv_heads, self.head_dim
        x = self.w["embed"][tokens]
        for i in range(self.layers):
            qkv = (self._rms(x, f"{i}.norm1") @ self.w[f"{i}.qkv"].T).view(n, hq + 2 * hk, d)
            out = attend(i, qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:], positions)
            x = x + out.reshape(n, hq * d) @ self.w[f"{i}.o"].T
            y = self._rms(x, f"{i}.norm2")
            x = x + (torch.nn.functional.silu(y @ self.w[f"{i}.gate"].T) * (y @ self.w[f"{i}.up"].T)) @ self.w[f"{i}.down"].T
        return self._rms(x, "norm") @ self.w["head"].T

    def heads_of(self, i):
        return {"table": self.table, "q_weight": self.w[f"{i}.q_norm"], "k_weight": self.w[f"{i}.k_norm"]}

    def packed(self, spans):
        """attend() of packed documents."""
        def attend(i, q, k, v, positions):
            q, k = forward.rotate_heads(q, k, positions=positions, **self.heads_of(i))
            return forward.attention(q, k, v, spans)
        return attend


class Packed:
    """Documents packed one after another: tokens, positions, targets and spans. A document's first `given` targets are not
    counted (-1)."""

    def __init__(self, documents, given):
        tokens, positions, targets, starts = [], [], [], [0]
        for doc, skip in zip(documents, given):
            doc = torch.as_tensor(doc)
            tokens.append(doc[:-1])
            targets.append(doc[1:].clone())
            targets[-1][:skip] = -1
            positions.append(torch.arange(len(doc) - 1))
            starts.append(starts[-1] + len(doc) - 1)
        self.tokens, self.positions, self.targets = (torch.cat(x).cuda() for x in (tokens, positions, targets))
        self.starts = torch.tensor(starts, dtype=torch.int32, device="cuda")
        self.spans = forward.document_spans(self.starts, tokens=starts[-1])

    def logits(self, model):
        return model.logits(self.tokens, self.positions, model.packed(self.spans))


class Batch(Packed):
    """Documents of the task."""

    def __init__(self, lengths, vocab, seed):
        g = torch.Generator().manual_seed(seed)
        documents = []
        for n in lengths:
            first, stride = (int(torch.randint(1, 8, (1,), generator=g)) for _ in range(2))
            documents.append((first + stride * torch.arange(n + 1)) % vocab)
        super().__init__(documents, [1] * len(documents))     # the stride is not known at the first token

    def loss_into(self, model, out):
        forward.token_loss(self.logits(model), self.targets, mean=True, out=out)


class Judged(Packed):
    """Answers of the model with an advantage each: the clipped policy loss of their tokens, with a term that keeps the policy
    near the one that gave them."""

    def __init__(self, model, prompts, answers, advantages, kl=0.02):
        super().__init__([p + a for p, a in zip(prompts, answers)], [len(p) - 1 for p in prompts])
        each = torch.tensor(advantages, dtype=torch.float32, device="cuda")
        self.advantages, self.kl = each.repeat_interleave(self.starts.diff().long()), kl
        self.logp = -forward.token_loss(self.logits(model), self.targets, with_nll=True)[1]

    def loss_into(self, model, out):
        forward.policy_loss(self.logits(model), self.targets, self.logp, self.advantages, ref_logp=self.logp, kl=self.kl, mean=True,
                            out=out)


class Preferred(Packed):
    """Pairs of answers to a prompt, the preferred one first: the loss of their log-ratios to the model that gave them."""

    def __init__(self, model, prompts, pairs, beta=0.1):
        super().__init__([p + a for p, pair in zip(prompts, pairs) for a in pair], [len(p) - 1 for p in prompts for _ in range(2)])
        self.beta = beta
        self.ref = forward.preference_loss(self.logits(model), self.targets, self.starts, with_logp=True)[1]

    def loss_into(self, model, out):
        forward.preference_loss(self.logits(model), self.targets, self.starts, ref_logp=self.ref, beta=self.beta, mean=True, out=out)


def step(model, batch, seed, K, eps, lr):
    """One step; returns the loss table (K, 3) and the preconditioner's status. Nothing waits for the device."""
    table = torch.empty(K, 3, dtype=torch.float64, device="cuda")
    batch.loss_into(model, table[0, 2:3])
    table[1:, 2] = table[0, 2]
    zo.perturb(model.params, seed, 0, eps)
    for k in range(K):
        batch.loss_into(model, table[k, 0:1])
        zo.perturb(model.params, seed, k, -2 * eps)
        batch.loss_into(model, table[k, 1:2])
        if k + 1 < K:
            zo.perturb2(model.params, seed, k, eps, k + 1, eps)
    c, status = zo.precondition(table, eps)
    zo.update(model.params, seed, c, lr, status=status, pre=(K - 1, eps))
    return table, status


class Answer:
    """Sequences being answered: a paged cache per layer, prompts put into it, then a token per sequence at a time."""

    def __init__(self, model, prompts, room, page_size=16):
        self.model, lengths = model, [len(p) for p in prompts]
        need = [-(-(n + room) // page_size) for n in lengths]
        shape = (sum(need), page_size, model.kv_heads, model.head_dim)
        self.caches = [tuple(torch.empty(shape, dtype=model.dtype, device="cuda") for _ in range(2)) for _ in range(model.layers)]
        order = torch.randperm(sum(need), generator=torch.Generator().manual_seed(1)).tolist()
        self.pages = torch.full((len(prompts), max(need)), -1, dtype=torch.int32)   # -1: no page
        self.rows_left = [n * page_size - m for n, m in zip(need, lengths)]
        for b, n in enumerate(need):
            self.pages[b, :n] = torch.tensor(order[:n])
            del order[:n]
        self.pages, self.page_size = self.pages.cuda(), page_size
        self.lengths = torch.tensor(lengths, dtype=torch.int32, device="cuda")
        starts = torch.tensor([sum(lengths[:b]) for b in range(len(lengths) + 1)], dtype=torch.int32, device="cuda")
        spans = forward.document_spans(starts, tokens=sum(lengths))
        sequence = torch.repeat_interleave(torch.arange(len(prompts), device="cuda"), self.lengths.long())
        positions = torch.arange(sum(lengths), device="cuda") - starts[sequence].long()
        slots = self._slots(sequence, positions)

        def attend(i, q, k, v, pos):     # rotated keys both into the cache and, in a row, for the prompt's own attention
            q, k = forward.rotate_heads(q, k, positions=pos, **model.heads_of(i))
            for cache, x in zip(self.caches[i], (k, v)):
                cache.view(-1, model.kv_heads, model.head_dim)[slots] = x
            return forward.attention(q, k, v, spans)

        self.logits = model.logits(torch.cat([torch.as_tensor(p) for p in prompts]).cuda(), positions, attend)[starts[1:].long() - 1]

    def _slots(self, sequence, positions):
        page = self.pages[sequence, positions // self.page_size].long()
        return torch.where(page < 0, -1, page * self.page_size + positions % self.page_size)

    def next(self, tokens):
        """Appends one token to each sequence; returns the logits after it. ValueError when a sequence's pages are full."""
        if min(self.rows_left) == 0:
            raise ValueError("a sequence's pages are full: there is no room for another token")
        self.rows_left = [n - 1 for n in self.rows_left]
        positions = self.lengths.long()
        slots = self._slots(torch.arange(len(positions), device="cuda"), positions)
        self.lengths += 1

        def attend(i, q, k, v, pos):
            kc, vc = self.caches[i]
            q, _, _ = forward.rotate_heads(q, k, v, positions=pos, k_out=kc, v_out=vc, slots=slots, **self.model.heads_of(i))
            return forward.decode_attention(q, kc, vc, self.pages, self.lengths)

        self.logits = self.model.logits(tokens, positions, attend)
        return self.logits

    def draft(self, tokens, parents, sizes=None):
        """Logits (sequences, nodes, vocabulary) after each node of a tree of drafted tokens per sequence: tokens and parents
        (sequences, nodes), a parent ahead of its children, -1: the sequence's last token, -2: no node. sizes: each tree's
        number of nodes, where they differ; what is behind is no node. Nothing is appended until accept(); ValueError where a
        sequence's pages have no room for its tree."""
        batch, nodes = tokens.shape
        if sizes is not None and (len(sizes) != batch or not all(0 <= n <= nodes for n in sizes)):
            raise ValueError("a tree has a size between none and all of its nodes")
        if any(n > left for n, left in zip(sizes if sizes is not None else [nodes] * batch, self.rows_left)):
            raise ValueError("a sequence's pages have no room for so many drafted tokens")
        if sizes is not None:
            ends = torch.tensor(sizes, device="cuda")[:, None]
            parents = torch.where(torch.arange(nodes, device="cuda") < ends, parents, torch.full_like(parents, -2))
        model, masks = self.model, forward.draft_masks(parents)
        depth = ((masks[:, :, None] >> torch.arange(nodes, device="cuda")) & 1).sum(2) - 1
        sequence = torch.arange(batch, device="cuda").repeat_interleave(nodes)
        some = masks.flatten() != 0
        places = (self.lengths[:, None] + torch.arange(nodes, device="cuda")).flatten()     # node j's keys are row lengths + j
        slots = torch.where(some, self._slots(sequence, torch.where(some, places.long(), 0)), -1)
        positions = torch.where(some, (self.lengths[:, None] + depth).flatten().long(), 0)

        def attend(i, q, k, v, pos):
            kc, vc = self.caches[i]
            q, _, _ = forward.rotate_heads(q, k, v, positions=pos, k_out=kc, v_out=vc, slots=slots, **model.heads_of(i))
            q = q.view(batch, nodes, model.heads, model.head_dim)
            return forward.draft_attention(q, kc, vc, self.pages, self.lengths, masks).flatten(0, 1)

        self.drafted = model.logits(tokens.flatten().clamp(min=0), positions, attend).view(batch, nodes, -1)
        return self.drafted

    def accept(self, paths):
        """Appends a path of the last draft()'s nodes to each sequence, a list of them from the root on (or none)."""
        batch = len(paths)
        sequence = torch.tensor([b for b, path in enumerate(paths) for _ in path], dtype=torch.long, device="cuda")
        node = torch.tensor([j for path in paths for j in path], dtype=torch.long, device="cuda")
        place = torch.tensor([i for path in paths for i in range(len(path))], dtype=torch.long, device="cuda")
        start = self.lengths.long()[sequence]
        source, target = self._slots(sequence, start + node), self._slots(sequence, start + place)
        for pair in self.caches:
            for cache in pair:
                rows = cache.view(-1, self.model.kv_heads, self.model.head_dim)
                rows[target] = rows[source]
        last = torch.tensor([path[-1] if path else 0 for path in paths], device="cuda")
        some = torch.tensor([bool(path) for path in paths], device="cuda")
        self.logits = torch.where(some[:, None], self.drafted[torch.arange(batch, device="cuda"), last], self.logits)
        self.lengths += torch.tensor([len(path) for path in paths], dtype=torch.int32, device="cuda")
        self.rows_left = [left - len(path) for left, path in zip(self.rows_left, paths)]

    def greedy_drafted(self, n, propose):
        """The tokens of greedy(n) -- up to ties -- in fewer passes: propose(sequences' tokens so far) gives a tree for each,
        lists of tokens and parents; of each the longest path of tokens that greedy() would give is accepted, and the one that
        comes behind it is known then. A sequence goes no further than its n tokens, and its tree no further than its pages."""
        got = [[t] for t in self.logits.argmax(-1).tolist()]     # the last one is not in the cache yet
        while min(map(len, got)) < n:
            trees = [([g[-1]] + list(t), [-1] + [p + 1 for p in up]) for g, (t, up) in zip(got, propose(got))]
            if not all(0 <= x < self.model.vocab for t, _ in trees for x in t):
                raise ValueError("a proposed token is outside the vocabulary")
            for b, left in enumerate(self.rows_left):            # none for a sequence with its n tokens; what there is room for
                if len(got[b]) < n and left == 0:
                    raise ValueError("a sequence's pages are full: there is no room for another token")
                trees[b] = [x[:left if len(got[b]) < n else 0] for x in trees[b]]
            sizes = [len(t) for t, _ in trees]
            tokens, parents = (torch.tensor([x + [fill] * (max(sizes) - len(x)) for x in xs], dtype=kind, device="cuda")
                               for xs, fill, kind in (([t for t, _ in trees], 0, torch.long), ([up for _, up in trees], -2, torch.int32)))
            best, paths = self.draft(tokens, parents, sizes).argmax(-1).tolist(), []
            for b, (t, up) in enumerate(trees):
                path, nexts = [], [0] if t else []
                while nexts and len(got[b]) < n:
                    path.append(nexts[0])
                    got[b].append(best[b][path[-1]])
                    nexts = [j for j in range(len(t)) if up[j] == path[-1] and t[j] == got[b][-1]]
                paths.append(path)
            self.accept(paths)
        return torch.tensor([g[:n] for g in got], device="cuda")

    def greedy(self, n):
        got = []
        for _ in range(n):
            got.append(self.logits.argmax(-1))
            self.next(got[-1])
        return torch.stack(got, 1)


def strides(got, vocab, most=4, deep=3):
    """For each sequence a tree of what may come by the task's rule: up to `most` strides, `deep` tokens of each."""
    trees = []
    for g in got:
        likely = [g[-1] - g[-2]] if len(g) > 1 else []
        steps = (likely + [s for s in range(1, 8) if s not in likely])[:most]
        tokens = [(g[-1] + s * (i + 1)) % vocab for s in steps for i in range(deep)]
        trees.append((tokens, [j - 1 if j % deep else -1 for j in range(len(tokens))]))
    return trees


def answered(model, count, kind):
    """Answers of the model to prompts of the task, judged by how many of their tokens follow the prompt's stride."""
    prompts = [[(1 + i % 5) + (1 + i % 7) * j for j in range(4)] for i in range(count)]
    first = Answer(model, prompts, 8).greedy(8).tolist()
    right = [[p[-1] + (p[1] - p[0]) * (i + 1) for i in range(8)] for p in prompts]
    if kind == "preference":
        return Preferred(model, prompts, list(zip(right, first)))
    score = torch.tensor([[float(x == y) for x, y in zip(a, r)] for a, r in zip(first + right, right + right)]).mean(1)
    return Judged(model, prompts + prompts, first + right, (score - score.mean()).tolist())


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--steps", type=int, default=5)
    ap.add_argument("--probes", type=int, default=16)
    ap.add_argument("--documents", type=int, default=12)
    ap.add_argument("--eps", type=float, default=1e-3)
    ap.add_argument("--lr", type=float, default=1e-3)
    ap.add_argument("--answers", choices=["policy", "preference"], help="steps on the model's own answers in place of documents")
    a = ap.parse_args()
    model = Decoder(dtype=torch.float32)      # at eps = 1e-3 a perturbation of bf16 weights of this size is mostly lost
    for s in range(a.steps):
        lengths = [5 + (37 * s + 53 * i) % 251 for i in range(a.documents)]
        torch.cuda.synchronize()
        t = time.perf_counter()
        batch = answered(model, a.documents, a.answers) if a.answers else Batch(lengths, model.vocab, s)
        table, status = step(model, batch, STEP_SEED_BASE + s, a.probes, a.eps, a.lr)
        loss = float(table[0, 2])
        print(json.dumps({"step": s, "tokens": len(batch.tokens), "loss": loss, "status": int(status),
                          "ms": 1e3 * (time.perf_counter() - t)}), flush=True)
    prompts = [[3, 5, 7, 9], [1, 2, 3, 4, 5, 6]]
    print(json.dumps({"answers": Answer(model, prompts, 24).greedy_drafted(8, lambda got: strides(got, model.vocab)).tolist()}))


if __name__ == "__main__":
    main()
