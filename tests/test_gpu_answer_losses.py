"""Losses over answers (zo_policy_loss, zo_preference_loss) and their gradients against 64 bits."""
import math

import pytest
import torch

import answer_ref as A
import forward_ref as R
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


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def answers(seed, tokens, vocab, dtype, ignore=3):
    """Logits, targets of which one in `ignore` does not count, and the targets' log-probabilities."""
    g = gen(seed)
    logits = (torch.randn(tokens, vocab, generator=g, device="cuda") * 2.5).to(dtype)
    targets = torch.randint(0, vocab, (tokens,), generator=g, device="cuda", dtype=torch.int32 if tokens % 2 else torch.int64)
    rows = torch.arange(tokens, device="cuda")
    logits[rows, targets.long()] = (logits[rows, targets.long()].float() + 6).to(dtype)
    if ignore:
        targets[1::ignore] = -1
    return g, logits, targets, A.rows(logits, targets)[0]


def policy_inputs(seed, tokens, vocab, dtype, clip=(0.2, 0.28), **kw):
    g, logits, targets, logp = answers(seed, tokens, vocab, dtype, **kw)
    ratio = torch.exp(0.2 * torch.randn(tokens, generator=g, device="cuda").double())
    for border in (1 - clip[0], 1 + clip[1]):    # none so near a border that fp32 could not tell its side
        ratio = torch.where((ratio / border - 1).abs() < 1e-3, ratio * 1.01, ratio)
    old = (logp - torch.log(ratio)).float()
    advantages = torch.randn(tokens, generator=g, device="cuda")
    advantages[2::5] = 0.0
    ref = (logp + 0.3 * torch.randn(tokens, generator=g, device="cuda")).float()
    weights = torch.rand(tokens, generator=g, device="cuda") + 0.1
    return logits, targets, old, advantages, ref, weights


def check_policy(logits, targets, old, advantages, ref, weights, clip=(0.2, 0.28), kl=0.0, mean=False, scale=1.0, **kw):
    got = F.policy_loss(logits, targets, old, advantages, ref_logp=ref if kl else None, weights=weights, clip=clip, kl=kl, mean=mean,
                        with_grad=True, grad_scale=scale, with_logp=True, **kw)
    loss, bound, grad, grad_bound, logp = A.policy(logits, targets, old, advantages, ref, weights, clip, kl, mean, scale)
    assert got[0].dtype == torch.float64 and got[1].dtype == logits.dtype and got[2].dtype == torch.float32
    A.close(got[0], loss, bound, "loss")
    R.check(got[1], grad, grad_bound, "grad")
    R.check(got[2], logp, A.LOGP + logp.abs() * A.E, "logp")
    assert not got[1][targets < 0].any() and not got[2][targets < 0].any()
    return got


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("tokens", [1, 2, 5, 77, 300])
@pytest.mark.parametrize("vocab", [1, 2, 7, 33, 511, 4096, 4097, 8193, 50272, 65537])
def test_policy(dtype, tokens, vocab):
    tokens = min(tokens, max(1, 6_000_000 // vocab))
    args = policy_inputs(tokens + vocab, tokens, vocab, dtype)
    got = check_policy(*args)
    check_policy(*args[:5], None, kl=0.05, mean=True, scale=16.0)
    kw = {"ref_logp": args[4], "weights": args[5], "clip": (0.2, 0.28), "with_logp": True}
    loss, logp = F.policy_loss(*args[:4], **kw)
    again = F.policy_loss(*args[:4], with_grad=True, **kw)
    want = A.policy(*args[:4], None, args[5], (0.2, 0.28), 0.0, False)       # the rows may be summed in other parts
    A.close(loss, want[0], want[1], "loss alone")
    R.check(logp, want[4], A.LOGP + want[4].abs() * A.E, "logp alone")
    assert all(torch.equal(x, y) for x, y in zip(again, got))
    out = torch.full((1,), 2.5, dtype=torch.float64, device="cuda")
    assert F.policy_loss(*args[:4], weights=args[5], clip=(0.2, 0.28), add=True, out=out) is out
    assert float(out) == 2.5 + float(loss)
    assert float(F.policy_loss(*args[:4], weights=args[5], clip=(0.2, 0.28), dtype=torch.float32)) == float(loss.float())


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("tokens,vocab", [(3, 151_936), (40, 151_936), (2, 500_001), (1, 1_400_003)])
def test_policy_of_large_vocabularies(dtype, tokens, vocab):
    """Rows that one SM cannot hold, nor several."""
    check_policy(*policy_inputs(5, tokens, vocab, dtype), kl=0.1, mean=True, scale=1024.0)


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("tokens,vocab,row,offset,grad_row,grad_offset", [
    (3, 1001, 1003, 0, 1001, 0), (40, 999, 1001, 1, 1001, 1), (6, 30000, 30007, 3, 30000, 0), (60, 77, 80, 5, 77, 2),
    (5, 9001, 9008, 8, 9016, 8), (5, 9001, 9001, 0, 9001, 1), (3, 160_001, 160_001, 1, 160_003, 2)])
def test_rows_off_every_boundary(dtype, tokens, vocab, row, offset, grad_row, grad_offset):
    """Rows of wider tensors, each at another alignment, NaN between them; what lies between the gradient's rows stays."""
    args = policy_inputs(row, tokens, vocab, dtype)

    def wide(x, row, offset):
        flat = torch.full((tokens * row + offset,), math.nan, dtype=dtype, device="cuda")
        rows = flat[offset:].view(tokens, row)[:, :vocab]
        rows.copy_(x)
        return flat, rows
    _, logits = wide(args[0], row, offset)
    flat, grad = wide(args[0], grad_row, grad_offset)
    between = torch.isnan(flat)
    got = check_policy(logits, *args[1:], grad_out=grad)
    assert got[1] is grad and torch.equal(torch.isnan(flat), between)
    want = grad.clone()
    F.policy_loss(logits, *args[1:4], weights=args[5], clip=(0.2, 0.28), grad_out=logits)     # in place
    assert torch.equal(logits, want)


@pytest.mark.parametrize("grad", [False, True])
def test_policy_of_extreme_logits(grad):
    """Masked logits of -inf and of the type's lowest value, targets of probability one and zero, NaN and +inf."""
    for dtype in DTYPES:
        low = torch.finfo(dtype).min
        x = torch.zeros(9, 9000, dtype=dtype, device="cuda")
        x[0, 5:] = -math.inf
        x[1, 5:] = low
        x[2] = low
        x[3] = 60000.0 if dtype == torch.float16 else 1e30
        x[4] = -math.inf
        x[5, 100] = math.nan
        x[6, 200] = math.inf
        x[7] = -math.inf
        x[7, 3] = 1.0
        x[8, 7000:] = -math.inf
        targets = torch.tensor([1, 2, 8000, 17, 3, 5, 7, 3, 8000], device="cuda")
        old, a = torch.zeros(9, device="cuda"), torch.ones(9, device="cuda")
        logp = F.policy_loss(x, targets, old, a, with_logp=True)[1].double().cpu()
        for i, want in ((0, -math.log(5)), (1, -math.log(5)), (2, -math.log(9000)), (3, -math.log(9000)), (7, 0.0)):
            assert abs(float(logp[i]) - want) <= 1e-5, i
        assert torch.isnan(logp[4:7]).all() and logp[8] == -math.inf
        good = torch.tensor([0, 1, 2, 3, 7, 8], device="cuda")
        loss, g = F.policy_loss(x[good], targets[good], old[good], a[good], with_grad=True)
        # ratios 1/5, 1/5, 1/9000, 1/9000, 1 and 0 of advantage 1: none is cut, the loss is minus their sum
        assert abs(float(loss) + 1.4 + 2 / 9000) <= 1e-5
        ratio = [0.2, 0.2, 1 / 9000, 1 / 9000, 1.0, 0.0]
        for i in range(6):
            want = torch.softmax(x[good[i]].double(), 0) * ratio[i]
            want[targets[good[i]]] -= ratio[i]
            tol = (R.U[dtype] + 1e-5) * want.abs() + R.TINY[dtype]
            assert ((g[i].double() - want).abs() <= tol).all(), i
        every = F.policy_loss(x, targets, old, a, with_grad=True)
        assert torch.isnan(every[0]) and torch.isnan(every[1][4:7]).all() and torch.equal(every[1][good], g)


def test_policy_where_nothing_counts():
    g, x, t, logp = answers(3, 6, 5000, torch.float32, ignore=0)
    nan = torch.full((6,), math.nan, device="cuda")
    none = torch.full_like(t, -1)
    loss, grad, lp = F.policy_loss(x, none, nan, nan, ref_logp=nan, weights=nan, kl=0.1, with_grad=True, with_logp=True)
    assert float(loss) == 0.0 and not grad.any() and not lp.any()
    loss, grad = F.policy_loss(x, none, nan, nan, mean=True, with_grad=True)
    assert math.isnan(float(loss)) and not grad.any()
    empty = F.policy_loss(x[:0], t[:0], nan[:0], nan[:0], with_grad=True, with_logp=True)
    assert float(empty[0]) == 0.0 and empty[1].shape == (0, 5000) and empty[2].shape == (0,)
    assert math.isnan(float(F.policy_loss(x[:0], t[:0], nan[:0], nan[:0], mean=True)))
    # what does not count is not read: neither logits nor what stands beside them
    t = t.clone()
    t[2], t[4] = -1, -(1 << 40)
    old, a, ref, w = (torch.rand(6, generator=g, device="cuda") for _ in range(4))
    want = F.policy_loss(x, t, old, a, ref_logp=ref, weights=w, kl=0.1, mean=True, with_grad=True)
    for v in (x, old, a, ref, w):
        v[2], v[4] = math.nan, math.inf
    got = F.policy_loss(x, t, old, a, ref_logp=ref, weights=w, kl=0.1, mean=True, with_grad=True)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    # targets outside the vocabulary
    t[1], t[3] = 5000, 1 << 40
    loss, grad, lp = F.policy_loss(x, t, old, a, with_grad=True, with_logp=True)
    assert torch.isnan(loss) and torch.isnan(grad[[1, 3]]).all() and torch.isnan(lp[[1, 3]]).all()
    assert torch.isfinite(grad[[0, 2, 4, 5]]).all()


def test_policy_gradient_against_differences():
    """Each logit of a few rows moved by h in fp64; central differences are off by h^2 / 6 of a third derivative, which is
    bounded by the loss's scale here, and by fp32's error of the loss over h."""
    x, t, old, a, ref, w = policy_inputs(9, 6, 12, torch.float32, ignore=4)
    kw = {"ref_logp": ref, "weights": w, "clip": (0.2, 0.28), "kl": 0.2}
    _, grad = F.policy_loss(x, t, old, a, with_grad=True, **kw)
    h = 2.0 ** -6
    for i in range(6):
        for v in range(12):
            sides = []
            for s in (h, -h):
                y = x.clone()
                y[i, v] += s
                sides.append((float(F.policy_loss(y, t, old, a, **kw)), float(y[i, v])))
            want = (sides[0][0] - sides[1][0]) / (sides[0][1] - sides[1][1])
            # borders of the clamp may lie between the two points: those logits' differences are no derivative
            logp = [A.rows(torch.where(torch.arange(12, device="cuda") == v, torch.tensor(s[1], device="cuda"), x[i]).view(1, -1), t[i:i + 1])[0]
                    for s in sides]
            r = [float(torch.exp(z - old[i])) for z in logp]
            if any(min(r) <= b <= max(r) for b in (0.8, 1.28)):
                continue
            assert abs(float(grad[i, v]) - want) <= 8 * h * h + 32 * A.LOGP / h, (i, v)


def test_gradient_through_a_models_weights():
    """The gradient in the logits handed on by torch's backward pass is that of the formula written in torch."""
    g = gen(4)
    weight = torch.randn(700, 32, generator=g, device="cuda", dtype=torch.float32, requires_grad=True)
    x = torch.randn(20, 32, generator=g, device="cuda")
    _, t, old, a, ref, w = policy_inputs(2, 20, 700, torch.float32)
    logits = x @ weight.T
    with pytest.raises(RuntimeError):
        F.policy_loss(logits, t, old, a, with_grad=True)         # the loss itself would have no gradient
    old = (A.rows(logits.detach(), t)[0] + 0.05).float()
    ref = old - 0.2
    loss, grad = F.policy_loss(logits.detach(), t, old, a, ref_logp=ref, kl=0.1, with_grad=True)
    logits.backward(grad)
    double = weight.detach().double().requires_grad_()
    z = x.double() @ double.T
    logp = torch.log_softmax(z, 1).gather(1, t.long().clamp(min=0)[:, None])[:, 0]
    r, d = torch.exp(logp - old), ref - logp
    each = -torch.minimum(r * a, r.clamp(0.8, 1.2) * a) + 0.1 * (torch.exp(d) - d - 1)
    want = torch.where(t >= 0, each, 0.0).sum()
    want.backward()
    assert abs(float(loss) - float(want.detach())) <= 20 * 60 * A.LOGP
    assert float((weight.grad.double() - double.grad).abs().max()) <= 20 * 60 * A.LOGP


def preference_inputs(seed, lengths, vocab, dtype, pad=0, by_length=False, **kw):
    g, logits, targets, logp = answers(seed, sum(lengths) + pad, vocab, dtype, **kw)
    starts = torch.tensor([sum(lengths[:j]) for j in range(len(lengths) + 1)], dtype=torch.int32, device="cuda")
    if pad:
        targets[-pad:] = 0                          # in no sequence: they do not count
    logp = A.rows(logits, targets)[0]
    sums = torch.stack([logp[a:b].sum() / (max(1, int((targets[a:b] >= 0).sum())) if by_length else 1)
                        for a, b in zip(starts.tolist(), starts[1:].tolist())] + [logp.sum() * 0])[:-1]
    ref = (sums + torch.randn(len(lengths), generator=g, device="cuda") * (0.3 if by_length else 4)).float()
    return logits, targets, starts, ref


def check_preference(logits, targets, starts, ref, beta=0.1, margin=0.0, smoothing=0.0, by_length=False, mean=False, scale=1.0, **kw):
    got = F.preference_loss(logits, targets, starts, ref_logp=ref, beta=beta, margin=margin, smoothing=smoothing, by_length=by_length,
                            mean=mean, with_grad=True, grad_scale=scale, with_logp=True, **kw)
    loss, bound, grad, grad_bound, sums, sums_bound = A.preference(logits, targets, starts, ref, beta, margin, smoothing, by_length,
                                                                   mean, scale)
    A.close(got[0], loss, bound, "loss")
    R.check(got[1], grad, grad_bound, "grad")
    R.check(got[2], sums, sums_bound, "logp")
    assert not got[1][targets < 0].any() and not got[1][int(starts[-1]):].any() and not got[1][:int(starts[0])].any()
    return got


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("lengths", [[1, 1], [3, 0], [0, 0, 2, 1], [7, 30, 1, 2, 40, 33], [4] * 70], ids=str)
@pytest.mark.parametrize("vocab", [1, 2, 33, 511, 4097, 50272])
def test_preference(dtype, lengths, vocab):
    if sum(lengths) * vocab > 6_000_000:
        lengths = [min(n, 30) for n in lengths[:4]]
    args = preference_inputs(sum(lengths) + vocab, lengths, vocab, dtype, pad=3)
    got = check_preference(*args)
    check_preference(*args, beta=0.5, margin=0.7, smoothing=0.1, mean=True, scale=64.0)
    check_preference(*args[:3], None, beta=2.0, by_length=True, smoothing=1.0)
    loss, sums = F.preference_loss(*args[:3], ref_logp=args[3], with_logp=True)
    assert torch.equal(loss, got[0]) and torch.equal(sums, got[2])
    out = torch.full((1,), 2.5, dtype=torch.float32, device="cuda")
    F.preference_loss(*args[:3], ref_logp=args[3], add=True, out=out)
    assert float(out) == float((torch.tensor(2.5, dtype=torch.float64) + loss.cpu()).float())


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("lengths,vocab", [([2, 1], 151_936), ([9, 20, 17, 4], 151_936), ([1, 1], 700_001), ([300, 280, 5, 600], 20_000)])
def test_preference_of_large_vocabularies_and_long_answers(dtype, lengths, vocab):
    """Pairs that stay in the caches between their two passes, and pairs that do not."""
    check_preference(*preference_inputs(7, lengths, vocab, dtype, pad=1, by_length=True), beta=2.0, by_length=True, mean=True, scale=4096.0)


def test_preference_starts_elsewhere():
    """Rows ahead of the first answer and behind the last are nobody's: they may hold anything."""
    x, t, starts, ref = preference_inputs(11, [5, 3, 20, 8], 5000, torch.bfloat16)
    want = F.preference_loss(x, t, starts, ref_logp=ref, with_grad=True, with_logp=True)
    wide = torch.full((50, 5000), math.nan, dtype=torch.bfloat16, device="cuda")
    wide[4:40] = x
    targets = torch.full((50,), 7, device="cuda", dtype=t.dtype)
    targets[4:40] = t
    got = F.preference_loss(wide, targets, starts + 4, ref_logp=ref, with_grad=True, with_logp=True)
    assert torch.equal(got[0], want[0]) and torch.equal(got[2], want[2])
    assert torch.equal(got[1][4:40], want[1]) and not got[1][:4].any() and not got[1][40:].any()


@pytest.mark.parametrize("starts", [[0, 5, 3, 20, 30], [0, 3, 5, 20, 37], [-1, 3, 5, 20, 30], [0, 3, 1 << 30, 20, 30], [10, 8, 6, 4, 2],
                                    [-(1 << 31), 3, 5, (1 << 31) - 1, 30]], ids=str)
def test_preference_of_starts_that_are_none(starts):
    x, t, _, ref = preference_inputs(11, [5, 3, 20, 8], 5000, torch.float16)
    loss, grad, logp = F.preference_loss(x, t, torch.tensor(starts, dtype=torch.int32, device="cuda"), ref_logp=ref, with_grad=True,
                                         with_logp=True)
    assert torch.isnan(loss) and torch.isnan(logp).all() and torch.isnan(grad[t >= 0]).all() and not grad[t < 0].any()


def test_preference_of_nothing_and_of_bad_rows():
    x, t, starts, ref = preference_inputs(13, [5, 3, 20, 8], 5000, torch.float32)
    assert float(F.preference_loss(x, t, starts[:1])) == 0.0 and math.isnan(float(F.preference_loss(x, t, starts[:1], mean=True)))
    loss, grad, logp = F.preference_loss(x, t, starts[:1], with_grad=True, with_logp=True)
    assert not grad.any() and logp.shape == (0,)
    nothing = F.preference_loss(x[:0], t[:0], starts * 0, with_grad=True, with_logp=True)
    assert abs(float(nothing[0]) - 2 * math.log(2)) <= 1e-6 and not nothing[2].any() and nothing[1].shape == (0, 5000)
    want = F.preference_loss(x, t, starts, ref_logp=ref, with_grad=True, with_logp=True)
    none = t.clone()
    none[:8] = -1                                    # a pair of answers without a counted token
    got = F.preference_loss(x, none, starts, with_grad=True, with_logp=True)
    assert float(got[2][0]) == 0.0 and float(got[2][1]) == 0.0 and not got[1][:8].any() and torch.isfinite(got[1]).all()
    bad = x.clone()
    bad[6, 17] = math.nan                            # a row of the first pair
    t[6] = 3
    got = F.preference_loss(bad, t, starts, ref_logp=ref, with_grad=True, with_logp=True)
    assert torch.isnan(got[0]) and torch.isnan(got[2][1]) and torch.isfinite(got[2][[0, 2, 3]]).all()
    assert torch.isnan(got[1][:8][t[:8] >= 0]).all() and torch.equal(got[1][8:], want[1][8:])


def test_preference_of_large_margins():
    """Log-ratios of hundreds either way: the loss is their size or nothing, the slope beta or nothing."""
    x, t, starts, _ = preference_inputs(13, [5, 3, 4, 8], 500, torch.float32, ignore=0)
    sums = F.preference_loss(x, t, starts, with_logp=True)[1]
    for away in (3000.0, -3000.0, 150.0, -150.0):
        ref = sums.clone()
        ref[0::2] -= away
        loss, grad = F.preference_loss(x, t, starts, ref_logp=ref, beta=1.0, with_grad=True)
        assert abs(float(loss) - 2 * max(0.0, -away)) <= 1e-2 and torch.isfinite(grad).all()
        check_preference(x, t, starts, ref, beta=1.0, smoothing=0.25)


def test_preference_gradient_against_differences():
    x, t, starts, ref = preference_inputs(21, [2, 3, 1, 2], 9, torch.float32, ignore=5)
    kw = {"ref_logp": ref, "beta": 0.5, "smoothing": 0.1, "margin": 0.2, "by_length": True}
    _, grad = F.preference_loss(x, t, starts, with_grad=True, **kw)
    h = 2.0 ** -6
    for i in range(8):
        for v in range(9):
            y, z = x.clone(), x.clone()
            y[i, v] += h
            z[i, v] -= h
            want = (float(F.preference_loss(y, t, starts, **kw)) - float(F.preference_loss(z, t, starts, **kw))) / float(y[i, v] - z[i, v])
            assert abs(float(grad[i, v]) - want) <= 2 * h * h + 16 * A.LOGP / h, (i, v)


def test_rows_beyond_32_bits():
    """Rows of logits and gradient that start past 2^31 elements, in place."""
    vocab, tokens = 151_936, 14_200
    x = torch.zeros(tokens, vocab, dtype=torch.bfloat16, device="cuda")
    x[-2:] = torch.randn(2, vocab, generator=gen(1), device="cuda") * 3
    t = torch.full((tokens,), -1, device="cuda")
    t[-2:] = torch.tensor([0, vocab - 1], device="cuda")
    last = x[-2:].clone()
    logp = A.rows(last, t[-2:])[0]
    old, a = torch.zeros(tokens, device="cuda"), torch.ones(tokens, device="cuda")
    old[-2:] = logp
    want = A.policy(last, t[-2:], old[-2:], a[-2:], None, None, (0.2, 0.2), 0.0, False)
    _, grad = F.policy_loss(x, t, old, a, grad_out=x)
    assert grad is x
    R.check(x[-2:], want[2], want[3], "grad")
    assert not x[:-2].any()


def test_other_stream_graphs_and_versions():
    """Two captured calls with gradients, replayed side by side with eager calls, each with its own workspace."""
    args = policy_inputs(8, 40, 9000, torch.float16)
    pairs = preference_inputs(9, [9, 11, 6, 14], 9000, torch.float16)

    def calls(outs):
        a, b = outs
        F.policy_loss(*args[:4], ref_logp=args[4], kl=0.1, mean=True, out=a[0], grad_out=a[1])
        F.preference_loss(*pairs[:3], ref_logp=pairs[3], out=b[0], grad_out=b[1])

    def fresh():
        return [(torch.zeros(1, dtype=torch.float64, device="cuda"), torch.full((40, 9000), math.nan, dtype=torch.float16, device="cuda"))
                for _ in range(2)]
    want = fresh()
    version = want[0][1]._version
    calls(want)
    assert want[0][1]._version > version and want[0][0]._version > 0
    streams, graphs, outs = [torch.cuda.Stream() for _ in range(2)], [], [fresh() for _ in range(2)]
    for s, o in zip(streams, outs):
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=s):
                calls(o)
            graphs.append(graph)
    torch.cuda.synchronize()
    eager = fresh()
    for _ in range(3):
        for s, graph in zip(streams, graphs):
            with torch.cuda.stream(s):
                graph.replay()
        calls(eager)
    torch.cuda.synchronize()
    for o in (*outs, eager):
        assert all(torch.equal(x, y) for p, r in zip(o, want) for x, y in zip(p, r))


def test_loss_table():
    """Entries of a step's loss table, micro-batches added up, and the preconditioner on them; a NaN stops the update."""
    x, t, old, a, ref, w = policy_inputs(8, 40, 9000, torch.bfloat16)
    pairs = preference_inputs(9, [9, 11, 6, 14], 9000, torch.bfloat16)
    table = torch.full((2, 3), math.nan, dtype=torch.float64, device="cuda")
    for i in range(3):
        F.policy_loss(x[:25], t[:25], old[:25], a[:25], out=table[0, i:i + 1])
        F.policy_loss(x[25:], t[25:], old[25:], a[25:], out=table[0, i:i + 1], add=True)
        F.preference_loss(*pairs[:3], ref_logp=pairs[3], out=table[1, i:i + 1])
    whole = F.policy_loss(x, t, old, a)
    assert abs(float(table[0, 0]) - float(whole)) <= 1e-12 * abs(float(whole))
    _, status = zo.precondition(table, 1e-3)
    assert int(status) == zo.ZO_OK
    F.policy_loss(x, torch.full_like(t, 9000), old, a, out=table[1, 1:2])
    _, status = zo.precondition(table, 1e-3)
    assert int(status) == zo.ZO_ERR_NONFINITE


def test_refusals():
    x, t, old, a, ref, w = policy_inputs(8, 6, 100, torch.bfloat16)
    starts = torch.tensor([0, 2, 6], dtype=torch.int32, device="cuda")

    def policy(**kw):
        p = dict(logits=x, targets=t, old_logp=old, advantages=a) | kw
        return F.policy_loss(*[p.pop(n) for n in ("logits", "targets", "old_logp", "advantages")], **p)

    def preference(**kw):
        p = dict(logits=x, targets=t, starts=starts) | kw
        return F.preference_loss(*[p.pop(n) for n in ("logits", "targets", "starts")], **p)
    policy(), preference()
    for call in (policy, preference):
        for bad in ({"logits": x[0]}, {"targets": t[:3]}, {"add": True}, {"out": torch.zeros(2, device="cuda")}, {"dtype": torch.float16},
                    {"grad_out": x[:, :50]}, {"grad_out": x.T.contiguous().T}, {"ref_logp": ref[:1]}, {"logits": x.T.contiguous().T}):
            with pytest.raises(ValueError):
                call(**bad)
        for bad in ({"logits": x.cpu()}, {"logits": t}, {"targets": t.short()}, {"targets": t.cpu()}, {"grad_out": x.float()},
                    {"out": torch.zeros(1, device="cuda", dtype=torch.bfloat16)}, {"ref_logp": ref.double()}):
            with pytest.raises(TypeError):
                call(**bad)
        grad = torch.empty(12, 100, dtype=torch.bfloat16, device="cuda")
        for bad in ({"grad_out": x[:1].expand(6, 100)}, {"grad_scale": math.nan}, {"grad_scale": math.inf, "with_grad": True},
                    {"out": x.view(-1)[:4].view(torch.float64), "with_grad": True},
                    {"logits": grad[:6], "grad_out": grad[1:7]}):
            with pytest.raises(zo.ZoError):
                call(**bad)
        with pytest.raises(RuntimeError):
            call(logits=x.clone().requires_grad_())
    for bad in ({"old_logp": old[:2]}, {"advantages": a[:, None]}, {"weights": w[::2]}, {"kl": 0.1}):
        with pytest.raises(ValueError):
            policy(**bad)
    for bad in ({"old_logp": None}, {"advantages": a.double()}, {"weights": w.half()}):
        with pytest.raises(TypeError):
            policy(**bad)
    for bad in ({"clip": 1.5}, {"clip": (-0.1, 0.2)}, {"clip": (0.2, math.inf)}, {"clip": math.nan}, {"kl": math.nan, "ref_logp": ref},
                {"kl": -0.1, "ref_logp": ref}, {"out": old[:1], "dtype": torch.float32}):
        with pytest.raises(zo.ZoError):
            policy(**bad)
    for bad in ({"starts": starts[:2]}, {"starts": starts[None]}, {"ref_logp": ref[:3]}):
        with pytest.raises(ValueError):
            preference(**bad)
    for bad in ({"starts": starts.long()}, {"starts": [0, 2, 6]}):
        with pytest.raises(TypeError):
            preference(**bad)
    for bad in ({"beta": -0.1}, {"beta": math.inf}, {"margin": math.nan}, {"smoothing": 1.1}, {"smoothing": -0.1}):
        with pytest.raises(zo.ZoError):
            preference(**bad)
    inside = x.clone().requires_grad_()
    with torch.no_grad():
        assert policy(logits=inside, with_grad=True)[1].shape == x.shape
