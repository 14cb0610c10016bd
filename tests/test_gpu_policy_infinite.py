"""The policy loss where a part of a loss is infinite, or beyond fp32, and the factor in front of it is 0: the part is left
out, as it is by the formula for every finite value. A NaN stays one."""
import math

import pytest
import torch

import answer_ref as A
from paper_2609_38095_gb300 import build as zo_build
from paper_2609_38095_gb300 import forward as F

pytestmark = pytest.mark.gpu

DTYPES = [torch.bfloat16, torch.float16, torch.float32]
IDS = ["bf16", "f16", "f32"]


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    zo_build.build()


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("vocab", [300, 9000])
@pytest.mark.parametrize("mean", [False, True])
def test_ratios_beyond_fp32(dtype, vocab, mean):
    """Tokens whose ratio, or whose ratio to the reference, is beyond fp32: nothing comes of them where the advantage is 0 (the
    ratio's part) or the weight is 0."""
    g = torch.Generator(device="cuda").manual_seed(vocab)
    x = (torch.randn(8, vocab, generator=g, device="cuda") * 2).to(dtype)
    t = torch.randint(0, vocab, (8,), generator=g, device="cuda")
    logp = A.rows(x, t)[0].float()
    old, ref = logp - 0.05, logp + 0.1
    a = torch.tensor([0.0, 1.0, -1.0, 0.5, -2.0, 0.0, 1.5, -1.0], device="cuda")
    w = torch.tensor([1.0, 0.5, 0.0, 1.0, 0.25, 1.0, 0.0, 1.0], device="cuda")
    want = F.policy_loss(x, t, old, a, ref_logp=ref, weights=w, kl=0.1, mean=mean, with_grad=True)
    alone = F.policy_loss(x, t, old, a, ref_logp=ref, weights=w, kl=0.1, mean=mean)
    assert torch.isfinite(want[0]) and torch.isfinite(want[1]).all()
    old[0] -= 200.0                                              # advantage 0
    old[2] -= 200.0                                              # weight 0
    ref[6] += 200.0
    got = F.policy_loss(x, t, old, a, ref_logp=ref, weights=w, kl=0.1, mean=mean, with_grad=True)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and not got[1][[2, 6]].any()
    assert torch.equal(F.policy_loss(x, t, old, a, ref_logp=ref, weights=w, kl=0.1, mean=mean), alone)
    # without a term for the reference the first token has no gradient at all
    grad = F.policy_loss(x, t, old, a, weights=w, mean=mean, with_grad=True)[1]
    assert not grad[0].any() and torch.isfinite(grad).all()


def test_policy_stays_nan_and_infinite():
    g = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn(4, 600, generator=g, device="cuda")
    t = torch.randint(0, 600, (4,), generator=g, device="cuda")
    old = A.rows(x, t)[0].float()
    a = torch.tensor([1.0, 0.0, -1.0, 1.0], device="cuda")
    w = torch.tensor([1.0, 1.0, 1.0, 0.0], device="cuda")
    for row in (1, 3):                                           # of advantage 0, and of weight 0
        y = x.clone()
        y[row, 7] = math.nan
        assert math.isnan(float(F.policy_loss(y, t, old, a, weights=w)))
    far = old.clone()
    far[2] -= 200.0                                              # advantage -1, weight 1: the ratio is not cut on that side
    assert float(F.policy_loss(x, t, far, a, weights=w)) == math.inf
    far = old.clone()
    far[0] -= 200.0                                              # advantage 1: cut
    loss, grad = F.policy_loss(x, t, far, a, weights=w, with_grad=True)
    # -1.2, 0 and a ratio of 1 within fp32's error of its logarithm
    assert abs(float(loss) + 1.2 - 1.0) <= 4 * A.LOGP and not grad[0].any()
