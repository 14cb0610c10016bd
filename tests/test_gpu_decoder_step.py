"""The decoder example: its forward point against plain torch, a step against Algorithm 1's order, answers over the
paged cache against the packed forward."""
import pytest
import torch

import decoder_step as D
import paper_2609_38095_gb300 as zo
from paper_2609_38095_gb300 import build as zo_build

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    zo_build.build()


def plain_logits(model, tokens, positions, starts):
    """The model in fp64 from its weights."""
    w = {n: t.double() for n, t in model.w.items()}
    rms = lambda x, g: x / torch.sqrt(x.square().mean(-1, keepdim=True) + 1e-6) * g  # noqa: E731
    half = model.head_dim // 2
    angle = positions[:, None].double() * 1e6 ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)
    turn = torch.complex(angle.cos(), angle.sin())[:, None]

    def rotate(x, g):
        x = rms(x, g)
        z = torch.complex(x[..., :half], x[..., half:]) * turn
        return torch.cat([z.real, z.imag], -1)
    n, hq, hk, d = len(tokens), model.heads, model.kv_heads, model.head_dim
    doc = torch.bucketize(torch.arange(n, device="cuda"), starts[1:], right=True)
    seen = (doc[:, None] == doc) & torch.ones(n, n, dtype=torch.bool, device="cuda").tril()
    x = w["embed"][tokens]
    for i in range(model.layers):
        qkv = (rms(x, w[f"{i}.norm1"]) @ w[f"{i}.qkv"].T).view(n, hq + 2 * hk, d)
        q, k = rotate(qkv[:, :hq], w[f"{i}.q_norm"]), rotate(qkv[:, hq:hq + hk], w[f"{i}.k_norm"])
        k, v = (y.repeat_interleave(hq // hk, 1) for y in (k, qkv[:, hq + hk:]))
        s = torch.einsum("thd,jhd->htj", q, k) * d ** -0.5
        p = torch.softmax(s.masked_fill(~seen, -torch.inf), -1)
        x = x + torch.einsum("htj,jhd->thd", p, v).reshape(n, -1) @ w[f"{i}.o"].T
        y = rms(x, w[f"{i}.norm2"])
        x = x + (torch.nn.functional.silu(y @ w[f"{i}.gate"].T) * (y @ w[f"{i}.up"].T)) @ w[f"{i}.down"].T
    return rms(x, w["norm"]) @ w["head"].T


@pytest.mark.parametrize("dtype,tol", [(torch.float32, 2e-4), (torch.bfloat16, 0.25)], ids=["f32", "bf16"])
def test_forward_point(dtype, tol):
    """Logits of about unit size; some 30 roundings of 2^-8 of unit-sized values along the way in bf16, and as many of
    2^-24 and sums of up to 512 products in fp32, with room for their growth through two layers."""
    model = D.Decoder(dtype=dtype, seed=3)
    lengths = [1, 40, 129, 7]
    batch = D.Batch(lengths, model.vocab, 0)
    starts = torch.tensor([sum(lengths[:i]) for i in range(5)], device="cuda")
    got = model.logits(batch.tokens, batch.positions, model.packed(batch.spans))
    want = plain_logits(model, batch.tokens, batch.positions, starts)
    assert float((got.double() - want).abs().max()) <= tol * max(1.0, float(want.abs().max()) / 4)
    table = torch.empty(1, dtype=torch.float64, device="cuda")
    batch.loss_into(model, table)
    counted = batch.targets >= 0
    loss = torch.nn.functional.cross_entropy(want[counted], batch.targets[counted])
    assert abs(float(table) - float(loss)) <= tol * float(loss)


def test_step_is_algorithm_1():
    """The fused schedule's weights and losses, bit for bit those of +eps, -2 eps, +eps per probe and the update."""
    K, eps, lr, seed = 5, 1e-3, 1e-3, 77
    a, b = D.Decoder(dtype=torch.float32, seed=1), D.Decoder(dtype=torch.float32, seed=1)
    batch = D.Batch([30, 100, 11], a.vocab, 5)
    table, status = D.step(a, batch, seed, K, eps, lr)
    want = torch.empty(K, 3, dtype=torch.float64, device="cuda")
    batch.loss_into(b, want[0, 2:3])
    want[1:, 2] = want[0, 2]
    for k in range(K):
        zo.perturb(b.params, seed, k, eps)
        batch.loss_into(b, want[k, 0:1])
        zo.perturb(b.params, seed, k, -2 * eps)
        batch.loss_into(b, want[k, 1:2])
        zo.perturb(b.params, seed, k, eps)
    c, _ = zo.precondition(want, eps)
    zo.update(b.params, seed, c, lr)
    assert int(status) == zo.ZO_OK
    assert torch.equal(table, want)
    assert all(torch.equal(x, y) for x, y in zip(a.params.tensors, b.params.tensors))
    assert float((table[:, 0] - table[:, 1]).abs().max()) > 0


def test_steps_lower_the_loss():
    model = D.Decoder(dtype=torch.float32, seed=2)
    batch = D.Batch([60, 33, 90, 17], model.vocab, 9)
    losses = [float(D.step(model, batch, 1000 + s, 16, 1e-3, 2e-3)[0][0, 2]) for s in range(12)]
    assert losses[-1] < losses[0], losses


@pytest.mark.parametrize("dtype,tol", [(torch.float32, 2e-4), (torch.bfloat16, 0.25)], ids=["f32", "bf16"])
def test_answers(dtype, tol):
    """Logits after each appended token as a packed forward of the whole sequences gives them."""
    model = D.Decoder(dtype=dtype, seed=4)
    prompts = [list(range(1, 20)), [7], list(range(100, 140))]
    answer = D.Answer(model, prompts, room=6, page_size=8)
    whole = [list(p) for p in prompts]
    for step in range(6):
        lengths = [len(p) for p in whole]
        starts = torch.tensor([sum(lengths[:i]) for i in range(4)], device="cuda")
        positions = torch.cat([torch.arange(n, device="cuda") for n in lengths])
        want = plain_logits(model, torch.tensor(sum(whole, []), device="cuda"), positions, starts)[starts[1:] - 1]
        assert float((answer.logits.double() - want).abs().max()) <= tol * max(1.0, float(want.abs().max()) / 4), step
        tokens = torch.tensor([(31 * step + 5 * b) % model.vocab for b in range(3)], device="cuda")
        for p, t in zip(whole, tokens.tolist()):
            p.append(t)
        answer.next(tokens)


def test_no_gradient_is_cut_silently():
    model = D.Decoder(dtype=torch.float32)
    batch = D.Batch([20], model.vocab, 0)
    for t in model.params.tensors:
        t.requires_grad_(True)
    with pytest.raises(RuntimeError):
        batch.loss_into(model, torch.empty(1, dtype=torch.float64, device="cuda"))
    with torch.no_grad():
        batch.loss_into(model, torch.empty(1, dtype=torch.float64, device="cuda"))
