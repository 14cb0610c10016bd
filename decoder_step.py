"""1.5-SPSA steps of a small decoder whose losses are its own: the library's step (perturb, losses, precondition,
update) around the library's forward point (head norms and rotation, attention of packed documents, token loss), then
an answer of the trained weights, token by token over a paged cache.

The model has the shape of the Qwen3 decoder in workloads.py at a small size: untied embedding and head, per layer
q/k/v/o projections, per-head norms of queries and keys, SwiGLU, two RMSNorms. Its matrix products, root-mean-square
norms and activations are torch's. The task is synthetic: in every document the next token is the last one plus the
document's stride, modulo the vocabulary; documents are packed one after another, their first token is not counted.

The schedule is the fused in-place one (Algorithm 1, bit for bit): +eps of probe 0, per probe the -2 eps pass and the
restore folded into the next probe's +eps, the last restore in the update.

    python decoder_step.py                          # a few steps and an answer, JSON lines
    python decoder_step.py --steps 20 --probes 32
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


class Batch:
    """Packed documents of the task: tokens, positions, targets (-1: not counted) and spans."""

    def __init__(self, lengths, vocab, seed):
        g = torch.Generator().manual_seed(seed)
        tokens, positions, targets, starts = [], [], [], [0]
        for n in lengths:
            first, stride = (int(torch.randint(1, 8, (1,), generator=g)) for _ in range(2))
            doc = (first + stride * torch.arange(n + 1)) % vocab
            tokens.append(doc[:-1])
            targets.append(doc[1:].clone())
            targets[-1][0] = -1                                   # the stride is not known yet
            positions.append(torch.arange(n))
            starts.append(starts[-1] + n)
        self.tokens, self.positions, self.targets = (torch.cat(x).cuda() for x in (tokens, positions, targets))
        self.spans = forward.document_spans(torch.tensor(starts, dtype=torch.int32, device="cuda"), tokens=starts[-1])

    def loss_into(self, model, out):
        logits = model.logits(self.tokens, self.positions, model.packed(self.spans))
        forward.token_loss(logits, self.targets, mean=True, out=out)


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
        self.rows_left = min(n * page_size - m for n, m in zip(need, lengths))
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
        if self.rows_left == 0:
            raise ValueError("a sequence's pages are full: there is no room for another token")
        self.rows_left -= 1
        positions = self.lengths.long()
        slots = self._slots(torch.arange(len(positions), device="cuda"), positions)
        self.lengths += 1

        def attend(i, q, k, v, pos):
            kc, vc = self.caches[i]
            q, _, _ = forward.rotate_heads(q, k, v, positions=pos, k_out=kc, v_out=vc, slots=slots, **self.model.heads_of(i))
            return forward.decode_attention(q, kc, vc, self.pages, self.lengths)

        self.logits = self.model.logits(tokens, positions, attend)
        return self.logits

    def greedy(self, n):
        got = []
        for _ in range(n):
            got.append(self.logits.argmax(-1))
            self.next(got[-1])
        return torch.stack(got, 1)


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--steps", type=int, default=5)
    ap.add_argument("--probes", type=int, default=16)
    ap.add_argument("--documents", type=int, default=12)
    ap.add_argument("--eps", type=float, default=1e-3)
    ap.add_argument("--lr", type=float, default=1e-3)
    a = ap.parse_args()
    model = Decoder(dtype=torch.float32)      # at eps = 1e-3 a perturbation of bf16 weights of this size is mostly lost
    for s in range(a.steps):
        lengths = [5 + (37 * s + 53 * i) % 251 for i in range(a.documents)]
        torch.cuda.synchronize()
        t = time.perf_counter()
        table, status = step(model, Batch(lengths, model.vocab, s), STEP_SEED_BASE + s, a.probes, a.eps, a.lr)
        loss = float(table[0, 2])
        print(json.dumps({"step": s, "tokens": sum(lengths), "loss": loss, "status": int(status),
                          "ms": 1e3 * (time.perf_counter() - t)}), flush=True)
    prompts = [[3, 5, 7, 9], [1, 2, 3, 4, 5, 6]]
    print(json.dumps({"answers": Answer(model, prompts, 8).greedy(8).tolist()}))


if __name__ == "__main__":
    main()
