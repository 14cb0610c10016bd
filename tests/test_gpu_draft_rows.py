"""Attention of trees of drafted tokens where a warp's rows are unlike: some of them none, some at addresses that take vectors and some
not, in blocks that a CTA forms alone and in ones that several share."""
import math

import pytest
import torch

from paper_2609_38095_gb300 import build as zo_build
from paper_2609_38095_gb300 import forward as F

pytestmark = pytest.mark.gpu

DTYPES = [torch.bfloat16, torch.float16]
IDS = ["bf16", "f16"]


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    zo_build.build()


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("heads,kv,drafts", [(4, 4, 26), (8, 4, 21), (4, 1, 26), (8, 1, 23), (5, 1, 53)])   # rows of a head: 26, 42, 104, 184, 265
@pytest.mark.parametrize("dim", [128, 64, 40])
@pytest.mark.parametrize("length", [50, 30_000], ids=["alone", "shared"])
def test_unlike_rows(dtype, heads, kv, drafts, dim, length):
    """Queries and outputs in rows that are off every boundary of 16 bytes in turn: the results of rows in a row, bit for bit, and
    nothing between the rows is written."""
    page, columns = 16, 12_000                                 # room for long answers: the kernels for many rows
    g = torch.Generator(device="cuda").manual_seed(drafts + dim)
    k, v = (torch.randn(300, page, kv, dim, generator=g, device="cuda").to(dtype) for _ in range(2))
    table = (torch.arange(columns, device="cuda") * 7 % 300).to(torch.int32).expand(2, columns).contiguous()
    lengths = torch.tensor([length, 3 * length // 4], dtype=torch.int32, device="cuda")
    masks = F.draft_masks(torch.tensor([[i - 1 if i % 4 else -1 for i in range(drafts)]] * 2, dtype=torch.int32, device="cuda"))
    masks[1, drafts - 3:] = 0                                  # rows at the end that see nothing, and one in between
    masks[0, 5] = 0
    q = torch.randn(2, drafts, heads, dim, generator=g, device="cuda").to(dtype)
    want, want_lse = F.draft_attention(q, k, v, table, lengths, masks, with_lse=True)
    assert torch.isfinite(want.float()).all() and not want[1, drafts - 3:].any() and not want[0, 5].any()

    def wide(fill):                                            # heads dim + 3 apart, nodes 2 more: each row at another alignment
        flat = torch.full((2, drafts, heads * (dim + 3) + 2), fill, dtype=dtype, device="cuda")
        return flat, flat[:, :, 1:1 + heads * (dim + 3)].unflatten(2, (heads, dim + 3))[..., :dim]
    _, qs = wide(math.nan)
    qs.copy_(q)
    flat, out = wide(7.0)
    got, lse = F.draft_attention(qs, k, v, table, lengths, masks, out=out, with_lse=True)
    assert torch.equal(got, want) and torch.equal(lse, want_lse)
    out.fill_(7.0)
    assert (flat == 7.0).all()
