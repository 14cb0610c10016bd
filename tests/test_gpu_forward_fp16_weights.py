"""fp16: keys that together weigh little beside one of their row's, each less than the type's normal range."""
import pytest
import torch

import forward_ref as R
from paper_2609_38095_gb300 import build as zo_build
from paper_2609_38095_gb300 import forward as F

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    zo_build.build()


def inputs(below, keys, dim, heads):
    """A first key whose score is ln(2^below) above the others', with values 0 where theirs are about 1."""
    g = torch.Generator(device="cuda").manual_seed(below)
    q = torch.ones(heads, dim, device="cuda")
    k = torch.zeros(keys, heads, dim, device="cuda")
    k[0] = below * 0.6931471805599453 / dim
    k[1:] += torch.randn(keys - 1, heads, dim, generator=g, device="cuda") * 0.3 / dim ** 0.5 / dim ** 0.5
    v = torch.rand(keys, heads, dim, generator=g, device="cuda") + 0.5
    v[0] = 0
    return q.half(), k.half(), v.half()


def bound(want, weighted, worst, dim, keys, v):
    """The usual bound, and what fp16's smallest numbers leave: with weights of up to 2^15, 2^7 of them for the largest
    seen when the reference was set, a weight is off by at most half a step, 2^-25 2^-7 of the row's sum."""
    return R.attention_bound(want, weighted, worst, torch.float16, dim, keys) + keys * 2.0 ** -32 * float(v.abs().max())


@pytest.mark.parametrize("below", [12, 18, 22, 24, 25, 26, 28])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("keys", [700, 6000])
def test_attention(below, dim, keys):
    heads = 2
    q, k, v = inputs(below, keys, dim, heads)
    rows = q.expand(40, heads, dim).contiguous()
    spans = torch.tensor([[0] * 40, [keys] * 40, [keys - 1] * 40], dtype=torch.int32, device="cuda")
    out, lse = F.attention(rows, k, v, spans, scale=1.0, with_lse=True)
    one = torch.zeros(40, dtype=torch.long, device="cuda")
    want, want_lse, worst, weighted = R.attention(rows, k, v, one, one + keys, one, 1.0, 0.0, None)
    R.check(out, want, bound(want, weighted, worst, dim, keys, v), "out")
    R.check(lse, want_lse, R.lse_bound(want_lse, worst, dim, keys), "lse")


@pytest.mark.parametrize("below", [12, 18, 22, 24, 25, 26, 28])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("keys", [700, 6000])
def test_decode(below, dim, keys):
    heads, page = 2, 16
    q, k, v = inputs(below, keys, dim, heads)
    n = -(-keys // page)
    kc, vc = (torch.zeros(n, page, heads, dim, dtype=torch.float16, device="cuda") for _ in range(2))
    kc.view(-1, heads, dim)[:keys], vc.view(-1, heads, dim)[:keys] = k, v
    pages = torch.arange(n, dtype=torch.int32, device="cuda")[None]
    out, lse = F.decode_attention(q[None], kc, vc, pages, torch.tensor([keys], dtype=torch.int32, device="cuda"), scale=1.0,
                                  with_lse=True)
    one = torch.zeros(1, dtype=torch.long, device="cuda")
    want, want_lse, worst, weighted = R.attention(q[None], k, v, one, one + keys, one, 1.0, 0.0, None)
    R.check(out, want, bound(want, weighted, worst, dim, keys, v), "out")
    R.check(lse.T, want_lse, R.lse_bound(want_lse, worst, dim, keys), "lse")
