"""Calls of the operators of learning from answers at sizes and strides beyond those of their other tests: more tokens, pairs and
sequences than a CTA has threads for, caches that share or reorder memory, rows of logits that are one row."""
import pytest
import torch

import answer_ref as A
import draft_ref as D
import forward_ref as R
from paper_2609_38095_gb300 import build as zo_build
from paper_2609_38095_gb300 import forward as F
from test_gpu_answer_losses import check_policy, check_preference, policy_inputs, preference_inputs
from test_gpu_draft_attention import compare, padded, paged, randn, trees

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    zo_build.build()


@pytest.mark.parametrize("tokens,vocab", [(4096, 40), (4097, 40), (9001, 33), (5000, 4100)])
@pytest.mark.parametrize("mean", [False, True])
def test_more_tokens_than_a_round_takes(tokens, vocab, mean):
    check_policy(*policy_inputs(7, tokens, vocab, torch.float32), kl=0.05, mean=mean)


@pytest.mark.parametrize("pairs", [17, 511, 1500])
@pytest.mark.parametrize("by_length", [False, True])
def test_more_pairs_than_a_round_takes(pairs, by_length):
    lengths = [(7 * j) % 5 for j in range(2 * pairs)]
    check_preference(*preference_inputs(pairs, lengths, 50, torch.float32, pad=2, by_length=by_length), beta=0.3, smoothing=0.1,
                     by_length=by_length, mean=True)


def test_one_row_for_all():
    """Logits of stride 0: every token has the same row; the gradient's rows are its own."""
    g = torch.Generator(device="cuda").manual_seed(4)
    for vocab in (600, 9000):
        row = torch.randn(1, vocab, generator=g, device="cuda", dtype=torch.float32) * 2
        x = row.expand(12, vocab)
        t = torch.randint(0, vocab, (12,), generator=g, device="cuda")
        old, a = A.rows(x, t)[0].float() - 0.05, torch.randn(12, generator=g, device="cuda")
        got = F.policy_loss(x, t, old, a, with_grad=True)
        want = F.policy_loss(x.contiguous(), t, old, a, with_grad=True)
        loss, bound, grad, grad_bound, _ = A.policy(x, t, old, a, None, None, (0.2, 0.2), 0.0, False)
        for have in (got, want):           # (rows at other alignments are summed in other orders)
            A.close(have[0], loss, bound, "loss")
            R.check(have[1], grad, grad_bound, "grad")
        with pytest.raises(F._zo.ZoError):
            F.policy_loss(x, t, old, a, grad_out=x)


def room(args, columns):
    """The same call with a page table that has room for much more: the kernels for many rows."""
    table = torch.zeros(len(args[3]), columns, dtype=torch.int32, device="cuda")
    table[:, :args[2].shape[1]] = args[2]
    return (*args[:2], table, *args[3:])


def equal_or_near(got, want):
    """As another cut of the same sums: two roundings of 16 bits of values below 4, of out and of the weights, each way."""
    u = 2.0 ** -8 if got.dtype == torch.bfloat16 else 2.0 ** -11
    assert float((got.float() - want.float()).abs().max()) <= 4 * 4 * u


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "f16"])
@pytest.mark.parametrize("drafts", [26, 64])
def test_caches_in_other_orders(dtype, drafts):
    """Heads before rows, pages apart by more than they take, one key-value head for all: with room for long answers and without."""
    lengths = [700, 0, 190]
    masks = padded(trees(drafts, [drafts, drafts, 9]), drafts)
    g = torch.Generator(device="cuda").manual_seed(drafts)
    args, rows = paged(g, lengths, masks, 16, 4, 128, dtype)
    kc, vc = args[:2]
    q = randn(g, 3, drafts, 8, 128, dtype=dtype)
    for columns in (args[2].shape[1], 10_000):
        wide = room(args, columns)
        want, want_lse = compare(q, wide, rows, lengths, masks)
        first = [x.transpose(1, 2).contiguous().transpose(1, 2) for x in (kc, vc)]
        apart = [torch.zeros(x.shape[0], 19, 5, 136, dtype=dtype, device="cuda")[:, :16, :4, :128].copy_(x) for x in (kc, vc)]
        for caches in (first, apart, [first[0], vc], [kc, apart[1]]):
            out, lse = F.draft_attention(q, *caches, *wide[2:], with_lse=True)
            assert torch.equal(out, want) and torch.equal(lse, want_lse)
        one = [x[:, :, 2:3].expand(x.shape) for x in (kc, vc)]
        out = F.draft_attention(q, *one, *wide[2:])
        own = F.draft_attention(q, *(x.contiguous() for x in one), *wide[2:])
        equal_or_near(out, own)


@pytest.mark.parametrize("page", [192, 200, 48])
@pytest.mark.parametrize("drafts", [26, 64])
def test_pages_of_other_sizes(page, drafts):
    """Pages of several steps and of no power of two, with many rows."""
    lengths = [1000, 191, 0, 64]
    masks = padded(trees(page, [drafts, 5, drafts, drafts]), drafts)
    g = torch.Generator(device="cuda").manual_seed(page)
    args, rows = paged(g, lengths, masks, page, 2, 64, torch.bfloat16)
    q = randn(g, 4, drafts, 4, 64, dtype=torch.bfloat16)
    compare(q, room(args, 300_000 // page), rows, lengths, masks)


def test_more_sequences_than_a_round_takes():
    """Sequences of few keys and of none, more than the plan's CTA has threads."""
    batch, drafts = 2500, 20
    g = torch.Generator(device="cuda").manual_seed(9)
    lengths = [(37 * b) % 50 - (b % 7 == 0) * 60 for b in range(batch)]
    masks = padded(trees(3, [drafts - b % 4 for b in range(batch)]), drafts)
    args, rows = paged(g, lengths, masks, 16, 1, 64, torch.bfloat16)
    q = randn(g, batch, drafts, 1, 64, dtype=torch.bfloat16)
    wide = room(args, 64)
    out, lse = F.draft_attention(q, *wide, with_lse=True)
    for b in list(range(0, batch, 61)) + [1023, 1024, 1025, 2047, 2048, batch - 1]:
        if lengths[b] < 0:
            assert not out[b].any()
        else:
            D.check(out[b], lse[b], q[b], *rows[b], lengths[b], masks[b], what=f"of {b}")
    equal_or_near(out, F.draft_attention(q, *args))
