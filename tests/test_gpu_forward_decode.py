"""One-token attention over a paged cache (zo_attention_decode) against 64 bits."""
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


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(g, *shape, dtype, scale=1.0):
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype)


def paged(g, lengths, page, kv, dim, dtype, garbage=math.nan):
    """A cache with the sequences' pages in random order; what no sequence owns is garbage, and so is the page table
    beyond each length."""
    need = [-(-n // page) for n in lengths]
    total = sum(need) + 2
    order = torch.randperm(total, generator=g, device="cuda").to(torch.int32)
    table = torch.full((len(lengths), max(need + [1]) + 1), 1 << 30, dtype=torch.int32, device="cuda")
    caches = [torch.full((total, page, kv, dim), garbage, dtype=dtype, device="cuda") for _ in range(2)]
    rows = []
    at = 0
    for b, n in enumerate(lengths):
        mine = order[at:at + need[b]]
        table[b, :need[b]] = mine
        at += need[b]
        pair = [randn(g, n, kv, dim, dtype=dtype) for _ in range(2)]
        for cache, x in zip(caches, pair):
            for i in range(need[b]):
                part = x[i * page:(i + 1) * page]
                cache[mine[i], :len(part)] = part
        rows.append(pair)
    return caches[0], caches[1], table, torch.tensor(lengths, dtype=torch.int32, device="cuda"), rows


def compare(q, caches, rows, softcap=0.0, slopes=None, **kw):
    kc, vc, table, lengths = caches
    out, lse = F.decode_attention(q, kc, vc, table, lengths, softcap=softcap, slopes=slopes, with_lse=True, **kw)
    d = q.shape[2]
    for b, (k, v) in enumerate(rows):
        n = len(k)
        one = torch.zeros(1, dtype=torch.long, device="cuda")
        want, want_lse, worst, weighted = R.attention(q[b:b + 1], k, v, one, one + n, one + n - 1, d ** -0.5, softcap, slopes)
        R.check(out[b:b + 1], want, R.attention_bound(want, weighted, worst, q.dtype, d, n), f"out {b}")
        R.check(lse[b][:, None], want_lse, R.lse_bound(want_lse, worst, d, n), f"lse {b}")
    return out, lse


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("dim", [128, 64, 80, 96, 8, 33, 200, 256])
@pytest.mark.parametrize("page", [1, 7, 16, 64])
def test_lengths(dtype, dim, page):
    """Lengths from none to several tiles of every warp, pages that end inside a tile, NaN in what is not owned."""
    lengths = [0, 1, 15, 16, 17, 63, 64, 65, 200, 1, 0, 531]
    g = gen(dim + page)
    *caches, rows = paged(g, lengths, page, 2, dim, dtype)
    q = randn(g, len(lengths), 6, dim, dtype=dtype, scale=1.5)
    compare(q, caches, rows)


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("heads,kv", [(1, 1), (2, 1), (8, 1), (9, 1), (16, 1), (17, 1), (24, 2), (40, 2), (5, 5)])
def test_groups(dtype, heads, kv):
    g = gen(heads)
    *caches, rows = paged(g, [70, 300], 16, kv, 128, dtype)
    compare(randn(g, 2, heads, 128, dtype=dtype), caches, rows)


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("batch,kv,length", [(1, 1, 3000), (1, 8, 2500), (3, 8, 1111), (40, 4, 130), (200, 2, 90)])
def test_splits(dtype, batch, kv, length):
    """From a cluster of many CTAs per head to one CTA; capped and biased too."""
    g = gen(batch)
    lengths = [max(1, length - 37 * b) for b in range(batch)]
    *caches, rows = paged(g, lengths, 16, kv, 64, dtype)
    q = randn(g, batch, 2 * kv, 64, dtype=dtype, scale=2.0)
    compare(q, caches, rows)
    slopes = torch.tensor([2.0 ** -(h + 2) for h in range(2 * kv)], device="cuda")
    compare(q, caches, rows, softcap=10.0, slopes=slopes)


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("dim", [128, 40, 33])
def test_strides(dtype, dim):
    """A cache with heads before rows, one off every vector boundary, q and out as parts of wider tensors."""
    g = gen(dim)
    kc, vc, table, lengths, rows = paged(g, [100, 37], 8, 2, dim, dtype)
    wide = randn(g, 2, 7, dim + 8, dtype=dtype)
    q = wide[:, 1:5, :dim]
    out = torch.zeros(2, 6, dim, dtype=dtype, device="cuda")
    want, _ = compare(q, (kc, vc, table, lengths), rows, out=out[:, :4])
    assert not out[:, 4:].any()
    first = [x.transpose(1, 2).contiguous().transpose(1, 2) for x in (kc, vc)]
    assert torch.equal(compare(q, (*first, table, lengths), rows)[0], want)
    off = [torch.empty(x.numel() + 1, dtype=dtype, device="cuda")[1:].view(x.shape).copy_(x) for x in (kc, vc)]
    compare(q, (*off, table, lengths), rows)


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
def test_bad_pages_and_lengths_are_nan(dtype):
    g = gen(8)
    kc, vc, table, lengths, rows = paged(g, [100, 37, 50, 20], 8, 2, 64, dtype)
    q = randn(g, 4, 4, 64, dtype=dtype)
    want, want_lse = F.decode_attention(q, kc, vc, table, lengths, with_lse=True)
    table[1, 2] = -1                       # no page of the cache
    table[2, 0] = kc.shape[0]
    lengths[3] = table.shape[1] * 8 + 1    # more than the page table can hold
    out, lse = F.decode_attention(q, kc, vc, table, lengths, with_lse=True)
    assert torch.equal(out[0], want[0]) and torch.equal(lse[0], want_lse[0])
    assert torch.isnan(out[1:]).all() and torch.isnan(lse[1:]).all()
    lengths[:] = -5
    out, lse = F.decode_attention(q, kc, vc, table, lengths, with_lse=True)
    assert not out.any() and (lse == -math.inf).all()


def test_offsets_beyond_32_bits():
    """Pages whose elements lie past 2^32 in the cache."""
    page, kv, dim = 64, 8, 128
    total = (1 << 32) // (page * kv * dim) + 40
    kc = torch.empty(total, page, kv, dim, dtype=torch.bfloat16, device="cuda")
    vc = torch.empty_like(kc)
    g = gen(2)
    ids = [total - 1, 3, total - 17, total // 2]
    n = 4 * page - 9
    k, v = (randn(g, 4 * page, kv, dim, dtype=torch.bfloat16) for _ in range(2))
    for i, p in enumerate(ids):
        kc[p], vc[p] = k[i * page:(i + 1) * page], v[i * page:(i + 1) * page]
    table = torch.tensor([ids], dtype=torch.int32, device="cuda")
    q = randn(g, 1, 32, dim, dtype=torch.bfloat16)
    compare(q, (kc, vc, table, torch.tensor([n], dtype=torch.int32, device="cuda")), [(k[:n], v[:n])])
    # and rows appended there
    slots = torch.tensor([total * page - 2], device="cuda")
    new = randn(g, 1, kv, dim, dtype=torch.bfloat16)
    pos = torch.zeros(1, dtype=torch.int64, device="cuda")
    F.rotate_heads(q, new, new, table=F.rotary_table(1, dim), positions=pos, k_out=kc, v_out=vc, slots=slots)
    assert torch.equal(kc[total - 1, page - 2], new[0]) and torch.equal(vc[total - 1, page - 2], new[0])


def test_repeatable_stream_and_graph():
    g = gen(6)
    *caches, rows = paged(g, [3000, 17], 16, 8, 128, torch.bfloat16)
    q = randn(g, 2, 32, 128, dtype=torch.bfloat16)
    want = F.decode_attention(q, *caches)
    for _ in range(3):
        assert torch.equal(F.decode_attention(q, *caches), want)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    out = torch.zeros_like(q)
    with torch.cuda.stream(s):
        got = F.decode_attention(q, *caches)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            F.decode_attention(q, *caches, out=out)
    s.synchronize()
    assert torch.equal(got, want)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)
