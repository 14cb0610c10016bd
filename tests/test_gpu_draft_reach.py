"""Trees of drafted tokens whose keys the page table does not hold: NaN in the rows that see anything, nothing where none does, and
no look at the table beyond its columns -- of which it may have none."""
import math

import pytest
import torch

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


def inputs(batch, drafts, heads, kv, dim, dtype, pages, page):
    g = torch.Generator(device="cuda").manual_seed(drafts + dim)
    q = torch.randn(batch, drafts, heads, dim, generator=g, device="cuda").to(dtype)
    k, v = (torch.randn(pages, page, kv, dim, generator=g, device="cuda").to(dtype) for _ in range(2))
    masks = F.draft_masks(torch.tensor([[i - 1 if i % 3 else -1 for i in range(drafts)]] * batch, dtype=torch.int32, device="cuda"))
    return q, k, v, masks


def lengths_of(*n):
    return torch.tensor(n, dtype=torch.int32, device="cuda")


BIASES = [None, "slopes"]


def call(q, k, v, table, lengths, masks, bias):
    slopes = torch.tensor([2.0 ** -(h + 1) for h in range(q.shape[2])], device="cuda") if bias else None
    return F.draft_attention(q, k, v, table, lengths, masks, slopes=slopes, with_lse=True)


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("drafts,heads,dim", [(3, 4, 64), (3, 2, 128), (20, 4, 128), (5, 4, 200), (64, 2, 64)])
@pytest.mark.parametrize("bias", BIASES, ids=["plain", "biased"])
def test_no_columns(dtype, drafts, heads, dim, bias):
    """A page table of no columns holds no key."""
    q, k, v, masks = inputs(3, drafts, heads, 2, dim, dtype, 4, 8)
    table = torch.zeros(3, 0, dtype=torch.int32, device="cuda")
    masks[2] = 0
    out, lse = call(q, k, v, table, lengths_of(50, 0, 1000), masks, bias)
    assert torch.isnan(out[:2]).all() and torch.isnan(lse[:2]).all()
    assert not out[2].any() and (lse[2] == -math.inf).all()
    out, lse = call(q, k, v, table, lengths_of(1 << 30, 0, 5), torch.zeros_like(masks), bias)
    assert not out.any() and (lse == -math.inf).all()


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("drafts,heads,dim", [(3, 4, 64), (3, 2, 128), (20, 4, 128), (5, 4, 200), (64, 2, 64)])
@pytest.mark.parametrize("bias", BIASES, ids=["plain", "biased"])
@pytest.mark.parametrize("beyond", [0, 1, 7, 4096, (1 << 31) - 1 - 16])
def test_one_key_too_many(dtype, drafts, heads, dim, bias, beyond):
    """The last sequence of a table of two columns: full with its tree, and from a key more on."""
    q, k, v, masks = inputs(2, drafts, heads, 2, dim, dtype, 6, 40)
    table = torch.tensor([[0, 1], [2, 3]], dtype=torch.int32, device="cuda")
    full = 80 - drafts
    want, want_lse = call(q, k, v, table, lengths_of(20, full), masks, bias)
    assert torch.isfinite(want[1].float()).all() and torch.isfinite(want_lse[1]).all()
    fits = 20 + drafts <= 80                     # the first sequence too; else it is NaN throughout

    def first_stays(out, lse):
        if fits:
            assert torch.isfinite(want[0].float()).all() and torch.equal(out[0], want[0]) and torch.equal(lse[0], want_lse[0])
        else:
            assert all(torch.isnan(x[0]).all() for x in (want, want_lse, out, lse))
    out, lse = call(q, k, v, table, lengths_of(20, min(full + 1 + beyond, (1 << 31) - 1)), masks, bias)
    first_stays(out, lse)
    assert torch.isnan(out[1]).all() and torch.isnan(lse[1]).all()
    # rows without a bit in such a sequence see nothing, and where none has one the length does not matter
    some = masks.clone()
    some[1, 1:] = 0
    out, lse = call(q, k, v, table, lengths_of(20, min(80 + beyond, (1 << 31) - 1)), some, bias)
    assert torch.isnan(out[1, 0]).all() and not out[1, 1:].any() and (lse[1, 1:] == -math.inf).all()
    some[1] = 0
    out, lse = call(q, k, v, table, lengths_of(20, min(80 + beyond, (1 << 31) - 1)), some, bias)
    first_stays(out, lse)
    assert not out[1].any() and (lse[1] == -math.inf).all()


@pytest.mark.parametrize("bias", BIASES, ids=["plain", "biased"])
def test_blocks_of_rows_behind_the_last_that_sees(bias):
    """Rows enough for several blocks, of which only the first see anything, at the table's very end."""
    q, k, v, masks = inputs(2, 60, 4, 1, 128, torch.bfloat16, 6, 40)
    masks[1, 2:] = 0
    table = torch.tensor([[0, 1], [2, 3]], dtype=torch.int32, device="cuda")
    out, lse = call(q, k, v, table, lengths_of(10, 78), masks, bias)
    assert torch.isfinite(out.float()).all() and torch.isfinite(lse[1, :2]).all()
    assert not out[1, 2:].any() and (lse[1, 2:] == -math.inf).all()
    first, first_lse = call(q[:, :2], k, v, table, lengths_of(10, 78), masks[:, :2].contiguous(), bias)
    # the same keys in the order of another cut: two roundings of unit-sized values, of out and of the weights
    assert float((out[1, :2] - first[1]).float().abs().max()) <= 2.0 ** -5 and float((lse[1, :2] - first_lse[1]).abs().max()) <= 2.0 ** -16


def test_many_rows_in_a_table_for_long_answers():
    """The kernels for many rows: sequences beyond a table of much room, beside ones within it."""
    page, columns = 16, 4096
    q, k, v, masks = inputs(4, 64, 8, 2, 64, torch.float16, 40, page)
    table = torch.zeros(4, columns, dtype=torch.int32, device="cuda")
    table[:] = torch.arange(columns, device="cuda") % 40
    within = lengths_of(500, 100, 63, 0)
    want, want_lse = call(q, k, v, table, within, masks, None)
    lengths = lengths_of(500, columns * page - 63, 63, 0)
    out, lse = call(q, k, v, table, lengths, masks, None)

    def others_stay():
        # cut elsewhere: two roundings of fp16 of values below 4, of out and of the weights
        for b in (0, 2, 3):
            assert float((out[b].float() - want[b].float()).abs().max()) <= 4 * 4 * 2.0 ** -11
            assert float((lse[b] - want_lse[b]).abs().max()) <= 2.0 ** -16
    others_stay()
    assert torch.isnan(out[1]).all() and torch.isnan(lse[1]).all()
    masks[1] = 0
    out, lse = call(q, k, v, table, lengths, masks, None)
    others_stay()
    assert not out[1].any() and (lse[1] == -math.inf).all()
