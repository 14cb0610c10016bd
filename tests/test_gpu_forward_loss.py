"""Token losses (zo_token_loss) against 64 bits."""
import math

import pytest
import torch

from paper_2609_38095_gb300 import build as zo_build
from paper_2609_38095_gb300 import forward as F
from paper_2609_38095_gb300 import zo

pytestmark = pytest.mark.gpu

DTYPES = [torch.bfloat16, torch.float16, torch.float32]
IDS = ["bf16", "f16", "f32"]


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    zo_build.build()


def reference(logits, targets):
    x = logits.double()
    nll = torch.logsumexp(x, 1) - x.gather(1, targets.long().clamp(min=0)[:, None])[:, 0]
    return torch.where(targets < 0, 0.0, nll)


def bound(logits):
    """exp(x - max): the difference and its product with log2 e are each rounded once, so the exponent of a logit d below
    the maximum is off by 3 d 2^-24; weighed by exp(-d) d that is at most 3 2^-24 of the sum. A thread adds at most
    1200 values in fp32, which at random signs of rounding stay below 64 of 2^-24; the exponential's own error is 2^-22."""
    return (3 + 64 + 4) * 2.0 ** -24


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("tokens", [1, 2, 5, 76, 77, 150, 700])
@pytest.mark.parametrize("vocab", [1, 7, 511, 4096, 8193, 50272, 65537])
def test_against_64_bits(dtype, tokens, vocab):
    if tokens * vocab > 20_000_000:
        tokens = 20_000_000 // vocab
    g = torch.Generator(device="cuda").manual_seed(vocab + tokens)
    logits = (torch.randn(tokens, vocab, generator=g, device="cuda") * 3).to(dtype)
    targets = torch.randint(0, vocab, (tokens,), generator=g, device="cuda", dtype=torch.int32 if tokens % 2 else torch.int64)
    targets[1::3] = -1
    loss, nll = F.token_loss(logits, targets, with_nll=True)
    want = reference(logits, targets)
    off = bound(logits)
    assert loss.dtype == torch.float64
    assert ((nll.double() - want).abs() <= off + 2.0 ** -24 * want.abs()).all()
    counted = max(1, int((targets >= 0).sum()))
    assert abs(float(loss) - float(want.sum())) <= counted * off
    assert torch.equal(F.token_loss(logits, targets), loss)
    mean = F.token_loss(logits, targets, mean=True)
    assert abs(float(mean) * counted - float(loss)) <= 1e-12 * abs(float(loss))
    assert float(F.token_loss(logits, targets, dtype=torch.float32)) == float(loss.float())


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("tokens,vocab,row,offset", [(3, 1001, 1003, 0), (40, 999, 1001, 1), (6, 30000, 30007, 3), (600, 77, 80, 5)])
def test_rows_off_every_boundary(dtype, tokens, vocab, row, offset):
    """Rows of a wider tensor, each at another alignment, NaN between them."""
    g = torch.Generator(device="cuda").manual_seed(row)
    flat = torch.full((tokens * row + offset,), math.nan, dtype=dtype, device="cuda")
    logits = flat[offset:offset + tokens * row].view(tokens, row)[:, :vocab]
    logits.copy_(torch.randn(tokens, vocab, generator=g, device="cuda"))
    targets = torch.randint(0, vocab, (tokens,), generator=g, device="cuda")
    targets[-1] = vocab - 1
    _, nll = F.token_loss(logits, targets, with_nll=True)
    want = reference(logits, targets)
    assert ((nll.double() - want).abs() <= bound(logits) + 2.0 ** -24 * want.abs()).all()


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
def test_extreme_logits(dtype):
    """Masked logits of -inf and of the type's lowest value, rows of nothing else, large offsets, NaN and +inf."""
    low = torch.finfo(dtype).min
    x = torch.zeros(8, 9000, dtype=dtype, device="cuda")
    x[0, 5:] = -math.inf
    x[1, 5:] = low
    x[2] = low
    x[3] = 60000.0 if dtype == torch.float16 else 1e30
    x[4] = -math.inf
    x[5, 100] = math.nan
    x[6, 200] = math.inf
    x[7] = -math.inf
    x[7, 3] = 1.0
    targets = torch.tensor([1, 2, 8000, 17, 3, 5, 7, 3], device="cuda")
    _, nll = F.token_loss(x, targets, with_nll=True)
    got = nll.double().cpu()
    for i, want in ((0, math.log(5)), (1, math.log(5)), (2, math.log(9000)), (3, math.log(9000)), (7, 0.0)):
        assert abs(float(got[i]) - want) <= 1e-5, i
    assert torch.isnan(got[4:7]).all()
    masked = F.token_loss(x, torch.tensor([7000, -1, -1, -1, -1, -1, -1, -1], device="cuda"))
    assert float(masked) == math.inf        # a target of probability zero


def test_targets_outside_the_vocabulary_nothing_counted_and_no_tokens():
    x = torch.randn(4, 1000, device="cuda")
    _, nll = F.token_loss(x, torch.tensor([1000, 3, -7, 1 << 40], device="cuda"), with_nll=True)
    assert torch.isnan(nll[[0, 3]]).all() and torch.isfinite(nll[1]) and float(nll[2]) == 0.0
    none = torch.full((4,), -1, device="cuda")
    assert float(F.token_loss(x, none)) == 0.0
    assert math.isnan(float(F.token_loss(x, none, mean=True)))
    assert float(F.token_loss(x[:0], none[:0])) == 0.0
    y = x.clone()
    y[2] = math.nan                          # not counted, not read
    t = torch.tensor([1, 2, -1, 3], device="cuda")
    assert torch.equal(F.token_loss(x, t), F.token_loss(y, t))


def test_loss_table():
    """Entries of a step's loss table, micro-batches added up, and the preconditioner on them; a NaN stops the update."""
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(3, 64, 2000, generator=g, device="cuda").bfloat16()
    t = torch.randint(0, 2000, (64,), generator=g, device="cuda")
    table = torch.full((2, 3), math.nan, dtype=torch.float64, device="cuda")
    for k in range(2):
        for i in range(3):
            F.token_loss(x[i, :40], t[:40], out=table[k, i:i + 1])
            F.token_loss(x[i, 40:], t[40:], out=table[k, i:i + 1], add=True)
    whole = torch.stack([reference(x[i], t).sum() for i in range(3)])
    assert (table - whole).abs().max() <= 64 * bound(x)
    _, status = zo.precondition(table, 1e-3)
    assert int(status) == zo.ZO_OK
    F.token_loss(x[0], torch.full_like(t, 5000), out=table[1, 1:2])
    _, status = zo.precondition(table, 1e-3)
    assert int(status) == zo.ZO_ERR_NONFINITE


def test_long_rows_beyond_32_bits():
    """Rows that start past 2^31 elements."""
    vocab, tokens = 151_936, 14_200
    logits = torch.empty(tokens, vocab, dtype=torch.bfloat16, device="cuda")
    logits[-2:] = torch.randn(2, vocab, device="cuda")
    targets = torch.full((tokens,), -1, device="cuda")
    targets[-2:] = torch.tensor([0, vocab - 1], device="cuda")
    _, nll = F.token_loss(logits, targets, with_nll=True)
    want = reference(logits[-2:], targets[-2:])
    assert ((nll[-2:].double() - want).abs() <= bound(logits) + 2.0 ** -24 * want.abs()).all()
    assert not nll[:-2].any()


def test_other_stream_and_graph():
    x = torch.randn(33, 5000, device="cuda").half()
    t = torch.arange(33, device="cuda")
    want = F.token_loss(x, t)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    out = torch.zeros(1, dtype=torch.float64, device="cuda")
    with torch.cuda.stream(s):
        got = F.token_loss(x, t)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            F.token_loss(x, t, out=out)
    s.synchronize()
    assert torch.equal(got, want)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)
