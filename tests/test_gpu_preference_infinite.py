"""The loss of pairs of answers where a part of a loss is infinite, or beyond fp32, and the factor in front of it is 0: the part is left
out, as it is by the formula for every finite value. A NaN stays one."""
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


def pairs(seed, vocab, dtype):
    """Three pairs of answers of 2, 3, 1, 2, 2 and 1 tokens."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    starts = torch.tensor([0, 2, 5, 6, 8, 10, 11], dtype=torch.int32, device="cuda")
    x = (torch.randn(11, vocab, generator=g, device="cuda") * 2).to(dtype)
    t = torch.randint(0, vocab, (11,), generator=g, device="cuda")
    return x, t, starts


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("vocab", [300, 9000])
@pytest.mark.parametrize("side,smoothing", [(1, 0.0), (0, 1.0)], ids=["rejected", "preferred"])
@pytest.mark.parametrize("by_length", [False, True])
def test_answers_of_probability_zero(dtype, vocab, side, smoothing, by_length):
    """A pair whose rejected answer cannot be given has the loss 0 without smoothing, one whose preferred answer cannot has it
    with labels turned round; the other pairs' losses and gradients are theirs alone."""
    x, t, starts = pairs(vocab, vocab, dtype)
    row = int(starts[2 + side])                                  # of the second pair's answer
    x[row, t[row]] = -math.inf
    loss, grad, logp = F.preference_loss(x, t, starts, beta=0.5, margin=0.1, smoothing=smoothing, by_length=by_length, with_grad=True,
                                         with_logp=True)
    assert logp[2 + side] == -math.inf and torch.isfinite(logp[[0, 1, 3 - side, 4, 5]]).all()
    others = torch.tensor([0, 1, 2, 3, 4, 8, 9, 10], device="cuda")
    rest = starts[[0, 1, 2, 5, 6]] - torch.tensor([0, 0, 0, 3, 3], dtype=torch.int32, device="cuda")
    want = A.preference(x[others], t[others], rest, None, 0.5, 0.1, smoothing, by_length, False)
    A.close(loss, want[0], want[1], "loss")
    R.check(grad[others], want[2], want[3], "grad")
    assert not grad[5:8].any()
    table = torch.zeros(1, 3, dtype=torch.float64, device="cuda")
    for i in range(3):
        F.preference_loss(x, t, starts, smoothing=smoothing, by_length=by_length, out=table[0, i:i + 1])
    assert int(zo.precondition(table, 1e-3)[1]) == zo.ZO_OK


def test_what_is_infinite_stays():
    """With some smoothing either side of such a pair is infinite, and without it a preferred answer that cannot be given."""
    x, t, starts = pairs(1, 500, torch.float32)
    x[5, t[5]] = -math.inf
    assert float(F.preference_loss(x, t, starts)) == math.inf
    assert float(F.preference_loss(x, t, starts, smoothing=0.1)) == math.inf
    x[6, t[6]] = -math.inf                                       # both: their difference is none
    assert math.isnan(float(F.preference_loss(x, t, starts)))
    x, t, starts = pairs(1, 500, torch.float32)
    for smoothing in (0.0, 1.0):
        y = x.clone()
        y[6, 3] = math.nan
        assert math.isnan(float(F.preference_loss(y, t, starts, smoothing=smoothing)))


def test_beta_of_zero():
    """Every pair's loss is softplus(margin), whatever the answers' probabilities; no gradient."""
    x, t, starts = pairs(1, 500, torch.float32)
    x[6, t[6]] = -math.inf
    loss, grad = F.preference_loss(x, t, starts, beta=0.0, margin=0.25, with_grad=True)
    want = 3 * math.log1p(math.exp(0.25))
    assert abs(float(loss) - want) <= 8 * A.E * want             # an exponential's 4 of three quarters, a logarithm's 2, a sum's 1
    assert not grad.any()
