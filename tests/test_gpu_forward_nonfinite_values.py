"""Values that are not finite: where a row sees them its columns are not finite, where it does not they do not matter,
and neither takes long."""
import math

import pytest
import torch

import forward_ref as R
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


def randn(seed, *shape, dtype, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype)


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("dim", [128, 64, 80, 33])
@pytest.mark.parametrize("softcap,biased", [(0.0, False), (5.0, False), (0.0, True), (5.0, True)])
@pytest.mark.parametrize("lengths", [[50, 75, 40], [400, 330, 300]], ids=["165", "1030"])
def test_columns(dtype, dim, softcap, biased, lengths):
    """NaN and infinities in single values and in whole keys' values, capped and biased: a row's column is not finite
    where it sees one, and is within the bound of a row without the unseen ones elsewhere."""
    t, hq, hk = sum(lengths), 4, 2
    q, k, v = (randn(i, t, h, dim, dtype=dtype) for i, h in enumerate((hq, hk, hk)))
    starts = torch.tensor([0, lengths[0], lengths[0] + lengths[1], t], dtype=torch.int32, device="cuda")
    spans = F.document_spans(starts, tokens=t)
    slopes = torch.tensor([2.0 ** -(h + 1) for h in range(hq)], device="cuda") if biased else None
    clean = v.clone()
    for key, head, col, value in ((0, 0, 1, math.inf), (lengths[0] + 30, 0, 7, math.nan), (lengths[0] + 31, 0, 1, -math.inf),
                                  (t - 20, 1, slice(None), math.nan), (t - 9, 0, dim - 1, math.inf)):
        v[key, head, col] = value
        clean[key, head, col] = 0
    out, lse = F.attention(q, k, v, spans, softcap=softcap, slopes=slopes, with_lse=True)
    s = spans.long()
    at = torch.arange(t, device="cuda")
    seen = (at >= s[0][:, None]) & (at < s[1][:, None])
    bad = torch.einsum("tj,jhd->thd", seen.double(), (~torch.isfinite(v)).double()) > 0
    bad = bad.repeat_interleave(hq // hk, 1)
    assert torch.equal(~torch.isfinite(out), bad)
    want, want_lse, worst, weighted = R.attention(q, k, clean, s[0], s[1], s[2], dim ** -0.5, softcap, slopes)
    # without the keys whose values were taken out the sums are smaller: only untouched columns are compared
    touched = (clean != v).any(0).repeat_interleave(hq // hk, 0)
    full = torch.where(touched, 0.0, 1.0).bool().expand(t, hq, dim)
    R.check(out[full], want[full], R.attention_bound(want, weighted, worst, dtype, dim, t)[full], "untouched columns")
    near = ~bad & ~full                          # columns that the row does not see touched
    R.check(out[near], want[near], R.attention_bound(want, weighted, worst, dtype, dim, t)[near], "touched columns")
    R.check(lse, want_lse, R.lse_bound(want_lse, worst, dim, t), "lse")


def per_call(f):
    for _ in range(2):
        f()
    a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    a.record()
    for _ in range(3):
        f()
    b.record()
    b.synchronize()
    return a.elapsed_time(b) / 3


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("where", ["first value", "first key", "late key", "NaN query"])
def test_time(dtype, where):
    """A document with such values takes a small multiple of a clean one's time, not one key after another for each row.
    32 times allows for one warp's walk over the keys before a late one."""
    t, heads, dim = 4096, 8, 128
    q, k, v = (randn(i, t, heads, dim, dtype=dtype) for i in range(3))
    starts = torch.tensor([0, t], dtype=torch.int32, device="cuda")
    spans = F.document_spans(starts, tokens=t)
    clean = per_call(lambda: F.attention(q, k, v, spans))
    if where == "first value":
        v[0, :, 3] = math.inf
    elif where == "first key":
        v[0] = math.nan
    elif where == "late key":
        v[3000] = math.inf
    else:
        q[1000] = math.nan
    took = per_call(lambda: F.attention(q, k, v, spans))
    print(f"{dtype} {where}: {1e3 * clean:.0f} us, {1e3 * took:.0f} us")
    assert took <= 32 * clean, (took, clean)
