"""Scores that are NaN under a cap: the rows that see them are NaN, whatever their neighbours' scores are, and no others."""
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


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(g, *shape, dtype, scale=1.0):
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype)


def ints(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def exactly(out, lse, rows):
    """NaN in every element and log-sum of the (token or sequence, head) pairs of `rows`, in none of the others."""
    assert torch.equal(torch.isnan(out), rows[..., None].expand(out.shape)), "out"
    assert torch.equal(torch.isnan(lse), rows), "lse"


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("dim", [64, 128, 80, 200])
@pytest.mark.parametrize("softcap,scale", [(5.0, 4.0), (20.0, 4.0), (20.0, 0.05)], ids=["cap 5", "cap 20", "far below"])
@pytest.mark.parametrize("lengths", [[70, 130], [300, 700]], ids=["200", "1000"])
@pytest.mark.parametrize("biased", [False, True], ids=["", "biased"])
def test_attention(dtype, dim, softcap, scale, lengths, biased):
    t, hq, hk = sum(lengths), 4, 2
    g = gen(dim)
    q, k, v = (randn(g, t, h, dim, dtype=dtype, scale=scale if h == hq else 1.0) for h in (hq, hk, hk))
    spans = F.document_spans(ints(0, lengths[0], t), tokens=t)
    slopes = torch.tensor([2.0 ** -(h + 2) for h in range(hq)], device="cuda") if biased else None
    rows = torch.zeros(t, hq, dtype=torch.bool, device="cuda")
    out, lse = F.attention(q, k, v, spans, softcap=softcap, slopes=slopes, with_lse=True)
    exactly(out, lse.T, rows)
    q[11, 1, 5] = math.nan                       # one element of a query
    q[lengths[0] + 3, 2] = math.nan
    rows[11, 1] = rows[lengths[0] + 3, 2] = True
    key = lengths[0] + 20                        # and one of a key, whose values are finite
    k[key, 1, dim - 1] = math.nan
    rows[key:, 2:] = True
    out, lse = F.attention(q, k, v, spans, softcap=softcap, slopes=slopes, with_lse=True)
    exactly(out, lse.T, rows)


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("dim", [64, 128, 80, 256, 33])
@pytest.mark.parametrize("heads,kv", [(6, 2), (32, 2), (2, 2)])
@pytest.mark.parametrize("softcap,scale", [(5.0, 4.0), (20.0, 4.0), (20.0, 0.05)], ids=["cap 5", "cap 20", "far below"])
def test_decode(dtype, dim, heads, kv, softcap, scale):
    lengths, page = [1, 40, 333, 90], 16
    g = gen(dim + heads)
    need = [-(-n // page) for n in lengths]
    pages = torch.full((4, max(need)), -1, dtype=torch.int32, device="cuda")
    order = torch.randperm(sum(need), generator=g, device="cuda").to(torch.int32)
    for b in range(4):
        pages[b, :need[b]] = order[sum(need[:b]):sum(need[:b + 1])]
    kc, vc = (randn(g, sum(need), page, kv, dim, dtype=dtype) for _ in range(2))
    q = randn(g, 4, heads, dim, dtype=dtype, scale=scale)
    rows = torch.zeros(4, heads, dtype=torch.bool, device="cuda")
    out, lse = F.decode_attention(q, kc, vc, pages, ints(*lengths), softcap=softcap, with_lse=True)
    exactly(out, lse, rows)
    q[0, heads - 1, 0] = q[3, 0, dim - 1] = math.nan
    rows[0, heads - 1] = rows[3, 0] = True
    kc[pages[2, 300 // page], 300 % page, 1, 2] = math.nan   # a key of sequence 2
    rows[2, heads // kv:] = True
    kc[pages[1, 40 // page], 40 % page:] = math.nan          # and what lies beyond sequence 1
    out, lse = F.decode_attention(q, kc, vc, pages, ints(*lengths), softcap=softcap, with_lse=True)
    exactly(out, lse, rows)


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
def test_a_position_outside_the_table_stops_the_update(dtype):
    """Through a capped layer to the loss table: the preconditioner sees a loss that is not finite."""
    t, heads, dim = 40, 4, 64
    g = gen(1)
    q, k, v = (randn(g, t, heads, dim, dtype=dtype, scale=3.0) for _ in range(3))
    table = F.rotary_table(64, dim)
    positions = torch.arange(t, device="cuda")
    positions[25] = 64
    q, k = F.rotate_heads(q, k, table=table, positions=positions)
    out, lse = F.attention(q, k, v, F.document_spans(ints(0, 20, t), tokens=t), softcap=20.0, with_lse=True)
    rows = torch.zeros(t, heads, dtype=torch.bool, device="cuda")
    rows[25:] = True                             # its key is seen by those that follow in its document
    exactly(out, lse.T, rows)
    losses = torch.zeros(1, 3, dtype=torch.float64, device="cuda")
    F.token_loss(out.reshape(t, -1), torch.zeros(t, dtype=torch.int64, device="cuda"), out=losses[0, 0:1])
    assert int(zo.precondition(losses, 1e-3)[1]) == zo.ZO_ERR_NONFINITE
