"""Attention of trees of drafted tokens over a paged cache (zo_draft_masks, zo_attention_draft) against 64 bits."""
import math
import random

import pytest
import torch

import draft_ref as D
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


def trees(seed, counts):
    """Random trees of so many nodes: chains, stars and what lies between."""
    rng = random.Random(seed)
    got = []
    for n in counts:
        back = rng.choice([1, 2, 5, 64])
        got.append([rng.randint(max(-1, i - back), i - 1) for i in range(n)])
    return got


def paged(g, lengths, masks, page, kv, dim, dtype, garbage=math.nan):
    """Caches with the sequences' pages in random order, and each sequence's keys and values in a row. What no node sees is
    garbage, and so is the page table where none of a page's keys is seen."""
    drafts = len(masks[0])
    rows, tables = [], []
    most = max(max(0, n) + drafts for n in lengths)
    table = torch.full((len(lengths), -(-most // page) + 1), 1 << 30, dtype=torch.int32)
    seen = []
    for n, m in zip(lengths, masks):
        union = 0
        for x in m:
            union |= x & ((1 << drafts) - 1)
        seen.append([union != 0] * max(0, n) + [bool(union >> j & 1) for j in range(drafts)] if n >= 0 else [False] * drafts)
    need = sum(-(-len(s) // page) for s in seen) + 2
    order = torch.randperm(need, generator=g, device="cuda").tolist()
    caches = [torch.full((need, page, kv, dim), garbage, dtype=dtype, device="cuda") for _ in range(2)]
    for b, s in enumerate(seen):
        pair = [randn(g, len(s), kv, dim, dtype=dtype) for _ in range(2)]
        s = torch.tensor(s)
        for x in pair:
            x[~s.cuda()] = garbage
        for i in range(-(-len(s) // page)):
            if not bool(s[i * page:(i + 1) * page].any()):
                continue
            table[b, i] = order.pop()
            for cache, x in zip(caches, pair):
                part = x[i * page:(i + 1) * page]
                cache[table[b, i], :len(part)] = part
        rows.append(pair)
    words = torch.tensor([[D.signed(x) for x in m] for m in masks], device="cuda")
    return (caches[0], caches[1], table.cuda(), torch.tensor(lengths, dtype=torch.int32, device="cuda"), words), rows


def compare(q, args, rows, lengths, masks, softcap=0.0, slopes=None, **kw):
    out, lse = F.draft_attention(q, *args, softcap=softcap, slopes=slopes, with_lse=True, **kw)
    for b, (k, v) in enumerate(rows):
        if lengths[b] < 0:
            assert not out[b].any() and (lse[b] == -math.inf).all()
            continue
        D.check(out[b], lse[b], q[b], k, v, lengths[b], masks[b], softcap, slopes, kw.get("scale"), f"of {b}")
    return out, lse


def padded(parents, drafts):
    return [D.masks_of(p) + [0] * (drafts - len(p)) for p in parents]


@pytest.mark.parametrize("drafts", [1, 2, 31, 32, 33, 64])
def test_masks(drafts):
    parents = [[-1 if i == 0 else (i * 7) % i for i in range(drafts)], [i - 1 for i in range(drafts)], [-1] * drafts, [-2] * drafts]
    if drafts > 8:
        broken = [i - 1 for i in range(drafts)]
        broken[3], broken[7] = 5, 7                       # later than the node, and itself
        parents.append(broken)
        parents.append([-1 if i % 3 else -5 for i in range(drafts)])
    parents.append([(-1 << 31) + i for i in range(drafts)])
    parents.append([(1 << 31) - 1] * drafts)
    t = torch.tensor(parents, dtype=torch.int32, device="cuda")
    want = torch.tensor([[D.signed(m) for m in D.masks_of(p)] for p in parents], device="cuda")
    assert torch.equal(F.draft_masks(t), want)
    assert F.draft_masks(t[:0]).shape == (0, drafts)
    many = t[:1].repeat(1000, 1)
    assert torch.equal(F.draft_masks(many), want[:1].expand(1000, drafts))


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("dim", [128, 64, 80, 96, 8, 33, 200, 256])
@pytest.mark.parametrize("page", [1, 7, 16, 64])
def test_lengths(dtype, dim, page):
    """Lengths from none to several tiles of every warp, trees that cross tiles and pages, NaN in what is not seen."""
    lengths = [0, 1, 15, 16, 17, 63, 64, 65, 200, 1, -3, 531]
    drafts = 7
    masks = padded(trees(dim + page, [7, 1, 7, 3, 7, 2, 7, 5, 6, 7, 7, 7]), drafts)
    g = gen(dim + page)
    args, rows = paged(g, lengths, masks, page, 2, dim, dtype)
    q = randn(g, len(lengths), drafts, 6, dim, dtype=dtype, scale=1.5)
    compare(q, args, rows, lengths, masks)


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("heads,kv,drafts", [(1, 1, 1), (1, 1, 64), (4, 1, 4), (4, 1, 5), (8, 1, 4), (8, 1, 5), (9, 1, 3), (7, 7, 17),
                                             (16, 1, 64), (24, 2, 33), (12, 4, 50), (40, 2, 13), (32, 8, 64)])
def test_rows(dtype, heads, kv, drafts):
    """From one row per key-value head to more than a thousand."""
    lengths = [70, 300, 1]
    masks = padded(trees(heads + drafts, [drafts, max(1, drafts // 2), drafts]), drafts)
    g = gen(heads + drafts)
    args, rows = paged(g, lengths, masks, 16, kv, 128, dtype)
    compare(randn(g, 3, drafts, heads, 128, dtype=dtype), args, rows, lengths, masks)


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("batch,kv,length,drafts", [(1, 1, 3000, 6), (1, 8, 2500, 40), (3, 8, 1111, 9), (40, 4, 130, 20), (200, 2, 90, 3)])
def test_splits(dtype, batch, kv, length, drafts):
    """From a cluster of many CTAs per block of rows to one CTA; capped and biased too."""
    g = gen(batch)
    lengths = [max(0, length - 37 * b) for b in range(batch)]
    masks = padded(trees(batch, [1 + (drafts * (b + 1) * 5) % drafts for b in range(batch)]), drafts)
    args, rows = paged(g, lengths, masks, 16, kv, 64, dtype)
    q = randn(g, batch, drafts, 2 * kv, 64, dtype=dtype, scale=2.0)
    compare(q, args, rows, lengths, masks)
    slopes = torch.tensor([2.0 ** -(h + 2) for h in range(2 * kv)], device="cuda")
    compare(q, args, rows, lengths, masks, softcap=10.0, slopes=slopes)
    compare(q, args, rows, lengths, masks, slopes=slopes, scale=-0.07)


@pytest.mark.parametrize("dtype", DTYPES[:2], ids=IDS[:2])
@pytest.mark.parametrize("heads,kv,dim,drafts,page", [(32, 32, 64, 26, 16), (8, 8, 128, 17, 24), (16, 8, 128, 32, 64), (16, 4, 80, 24, 256),
                                                      (32, 8, 128, 64, 16), (8, 1, 96, 64, 8), (12, 1, 64, 64, 128), (40, 8, 128, 31, 7)])
def test_much_work(dtype, heads, kv, dim, drafts, page):
    """Sequences of many and of few keys and no tree at all, in a page table with room for much more: work that is cut across
    sequences, heads and blocks of rows; blocks that begin in one CTA's share and end in another's, and whole ones."""
    lengths = [3000, 0, 63, 1, 700, -2, 129, 64, 2000, 5, 190, 1]
    sizes = [drafts, drafts, 1, drafts // 2, drafts, 3, 2, drafts, 5, drafts, drafts, 1]
    masks = padded(trees(heads + drafts, sizes), drafts)
    masks[6] = [0] * drafts
    g = gen(dim + drafts)
    args, rows = paged(g, lengths, masks, page, kv, dim, dtype)
    table = torch.full((len(lengths), -(-60_000 // page)), 1 << 30, dtype=torch.int32, device="cuda")
    table[:, :args[2].shape[1]] = args[2]
    args = (*args[:2], table, *args[3:])
    q = randn(g, len(lengths), drafts, heads, dim, dtype=dtype, scale=1.5)
    out, lse = compare(q, args, rows, lengths, masks)
    for _ in range(2):
        again = F.draft_attention(q, *args, with_lse=True)
        assert torch.equal(again[0], out) and torch.equal(again[1], lse)
    slopes = torch.tensor([2.0 ** -(8 * (h + 1) / heads) for h in range(heads)], device="cuda")
    compare(q, args, rows, lengths, masks, softcap=20.0, slopes=slopes)
    assert torch.equal(F.draft_attention(q, *args, out=q), out)
    # values that are not finite at a node, for those that see it and those that do not; a page that is none
    j = lengths[4] + 1
    args[1][table[4, j // page], j % page, 0, 3] = math.inf
    out2 = F.draft_attention(q, *args)
    assert not torch.isfinite(out2[4, 1, 0, 3])
    clean = [i for i in range(drafts) if not masks[4][i] >> 1 & 1]
    assert torch.isfinite(out2[4, clean]).all()
    table[0, 100 // page] = -3
    table[8, 1999 // page] = args[0].shape[0]
    out3, lse3 = F.draft_attention(q, *args, with_lse=True)
    for b in (0, 8):
        sees = torch.tensor([m != 0 for m in masks[b]], device="cuda")
        assert torch.isnan(out3[b, sees]).all() and torch.isnan(lse3[b, sees]).all() and not out3[b, ~sees].any()
    others = [b for b in range(len(lengths)) if b not in (0, 4, 8)]
    assert torch.equal(out3[others], out2[others])


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("drafts", [3, 40, 64])
def test_masks_of_the_callers_own(dtype, drafts):
    """Bits beyond the nodes, nodes that do not see themselves or see later ones, rows without a bit in the middle, the sign
    bit, sequences in which nothing is seen."""
    rng = random.Random(drafts)
    masks = [[rng.getrandbits(64) for _ in range(drafts)] for _ in range(5)]
    masks[1] = [m & ~(1 << i) if i % 3 else 0 for i, m in enumerate(masks[1])]
    masks[2] = [0 if drafts == 64 else 1 << 63 for _ in range(drafts)]
    masks[3] = [1 << (drafts - 1) for _ in range(drafts)]
    masks[4] = [1 if i == 1 else 0 for i in range(drafts)]
    lengths = [100, 37, 50, 0, 20]
    g = gen(drafts)
    args, rows = paged(g, lengths, masks, 8, 2, 64, dtype)
    q = randn(g, 5, drafts, 4, 64, dtype=dtype)
    compare(q, args, rows, lengths, masks)
    slopes = torch.tensor([0.3, 0.1, 0.05, 0.01], device="cuda")
    compare(q, args, rows, lengths, masks, slopes=slopes)


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("dim,heads,kv", [(128, 4, 2), (64, 12, 1), (40, 2, 2), (33, 4, 1)])
def test_strides(dtype, dim, heads, kv):
    """A cache with heads before rows, one off every vector boundary, q and out as parts of wider tensors, nodes first."""
    g = gen(dim)
    lengths, drafts = [100, 37], 9
    masks = padded(trees(dim, [9, 6]), drafts)
    (kc, vc, *rest), rows = paged(g, lengths, masks, 8, kv, dim, dtype)
    wide = randn(g, 2, drafts + 2, heads + 3, dim + 8, dtype=dtype)
    q = wide[:, 1:drafts + 1, 1:heads + 1, :dim]
    out = torch.zeros(drafts, 2, heads + 2, dim, dtype=dtype, device="cuda")
    want, _ = compare(q, (kc, vc, *rest), rows, lengths, masks, out=out.transpose(0, 1)[:, :, :heads])
    want = want.clone()
    assert not out[:, :, heads:].any()
    first = [x.transpose(1, 2).contiguous().transpose(1, 2) for x in (kc, vc)]
    assert torch.equal(compare(q, (*first, *rest), rows, lengths, masks)[0], want)
    off = [torch.empty(x.numel() + 1, dtype=dtype, device="cuda")[1:].view(x.shape).copy_(x) for x in (kc, vc)]
    compare(q, (*off, *rest), rows, lengths, masks)
    inplace = q.clone()
    F.draft_attention(inplace, kc, vc, *rest, out=inplace)
    assert torch.equal(inplace, want)


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("drafts,heads", [(4, 4), (6, 8), (64, 4)])
def test_what_a_row_does_not_see_does_not_reach_it(dtype, drafts, heads):
    """Keys and values of siblings that are NaN, infinite or the type's lowest: rows that see them are not finite (values) or
    NaN (keys), the others are what they are without."""
    g = gen(drafts)
    n = 37
    masks = padded([[-1] * drafts], drafts)               # each sees itself alone
    (kc, vc, table, lengths, words), rows = paged(g, [n], masks, 16, 2, 128, dtype, garbage=0.0)
    q = randn(g, 1, drafts, heads, 128, dtype=dtype)
    want, want_lse = F.draft_attention(q, kc, vc, table, lengths, words, with_lse=True)

    def at(j):
        return table[0, j // 16], j % 16
    for bad in (math.nan, math.inf, -math.inf):
        for j in (0, 1, drafts - 1):
            v = vc.clone()
            v[at(n + j)][0, 5] = bad
            out, lse = F.draft_attention(q, kc, v, table, lengths, words, with_lse=True)
            mine = torch.zeros_like(out, dtype=torch.bool)
            mine[0, j, :heads // 2, 5] = True
            assert not torch.isfinite(out[mine]).any() and torch.equal(out[~mine], want[~mine]) and torch.equal(lse, want_lse)
            k = kc.clone()
            k[at(n + j)][1] = bad
            out, lse = F.draft_attention(q, k, vc, table, lengths, words, with_lse=True)
            mine[...] = False
            mine[0, j, heads // 2:] = True
            assert torch.equal(out[~mine], want[~mine])
            if bad != bad:
                assert torch.isnan(out[mine]).all() and torch.isnan(lse[mine[..., 0]]).all()
    low = torch.finfo(dtype).min
    v = vc.clone()
    v[at(n + 1)] = low
    out = F.draft_attention(q, kc, v, table, lengths, words)
    others = [i for i in range(drafts) if i != 1]
    assert torch.equal(out[:, others], want[:, others])


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("drafts", [3, 20])
def test_bad_pages_and_lengths_are_nan(dtype, drafts):
    g = gen(8)
    lengths = [100, 37, 50, 20, 9]
    masks = padded(trees(drafts, [drafts, drafts, drafts, drafts, 1]), drafts)
    (kc, vc, table, ns, words), rows = paged(g, lengths, masks, 8, 2, 64, dtype)
    q = randn(g, 5, drafts, 4, 64, dtype=dtype)
    want, want_lse = F.draft_attention(q, kc, vc, table, ns, words, with_lse=True)
    table[1, 2] = -1                       # no page of the cache
    table[2, 0] = kc.shape[0]
    ns[3] = table.shape[1] * 8             # more keys than the page table can hold
    table[4, 1] = -7                       # the node's own page
    out, lse = F.draft_attention(q, kc, vc, table, ns, words, with_lse=True)
    assert torch.equal(out[0], want[0]) and torch.equal(lse[0], want_lse[0])
    assert torch.isnan(out[1:4]).all() and torch.isnan(lse[1:4]).all()
    assert torch.isnan(out[4, 0]).all() and not out[4, 1:].any() and (lse[4, 1:] == -math.inf).all()
    for n in ((1 << 31) - 1, (1 << 31) - 65):
        ns[:] = n
        out, lse = F.draft_attention(q, kc, vc, table, ns, words, with_lse=True)
        assert torch.isnan(out[:4]).all() and torch.isnan(lse[:4]).all()
    for n in (-1, -(1 << 31)):
        ns[:] = n
        out, lse = F.draft_attention(q, kc, vc, table, ns, words, with_lse=True)
        assert not out.any() and (lse == -math.inf).all()
    ns[:] = 5
    none = torch.zeros(0, 8, 2, 64, dtype=dtype, device="cuda")
    assert torch.isnan(F.draft_attention(q, none, none, table, ns, words)[:4]).all()
    assert F.draft_attention(q[:0], kc, vc, table[:0], ns[:0], words[:0]).shape == (0, drafts, 4, 64)


def test_one_node_is_the_next_token():
    """A tree of one node is decode_attention of one key more, up to the order of additions."""
    g = gen(3)
    lengths = [5, 0, 300]
    masks = [[1]] * 3
    args, rows = paged(g, lengths, masks, 16, 2, 128, torch.float32)
    q = randn(g, 3, 1, 8, 128, dtype=torch.float32)
    out, _ = compare(q, args, rows, lengths, masks)
    want = F.decode_attention(q[:, 0], *args[:3], args[3] + 1)
    assert float((out[:, 0] - want).abs().max()) <= 1e-5      # sums of at most 301 terms of unit size, twice


def test_offsets_beyond_32_bits():
    """Pages whose elements lie past 2^32 in the cache."""
    page, kv, dim, drafts = 64, 8, 128, 12
    total = (1 << 32) // (page * kv * dim) + 40
    kc = torch.empty(total, page, kv, dim, dtype=torch.bfloat16, device="cuda")
    vc = torch.empty_like(kc)
    g = gen(2)
    ids = [total - 1, 3, total - 17, total // 2]
    n = 4 * page - 9 - drafts
    k, v = (randn(g, 4 * page, kv, dim, dtype=torch.bfloat16) for _ in range(2))
    for i, p in enumerate(ids):
        kc[p], vc[p] = k[i * page:(i + 1) * page], v[i * page:(i + 1) * page]
    masks = padded(trees(1, [drafts]), drafts)
    words = torch.tensor([[D.signed(m) for m in masks[0]]], device="cuda")
    table = torch.tensor([ids], dtype=torch.int32, device="cuda")
    q = randn(g, 1, drafts, 32, dim, dtype=torch.bfloat16)
    args = (kc, vc, table, torch.tensor([n], dtype=torch.int32, device="cuda"), words)
    compare(q, args, [(k[:n + drafts], v[:n + drafts])], [n], masks)


@pytest.mark.parametrize("drafts,room", [(5, 0), (64, 0), (5, 100_000), (64, 100_000)])
def test_repeatable_stream_and_graph(drafts, room):
    g = gen(6)
    lengths = [3000, 17]
    masks = padded(trees(7, [drafts, 3]), drafts)
    args, rows = paged(g, lengths, masks, 16, 8, 128, torch.bfloat16)
    if room:                                            # a page table for long answers
        table = torch.zeros(2, room // 16, dtype=torch.int32, device="cuda")
        table[:, :args[2].shape[1]] = args[2]
        args = (*args[:2], table, *args[3:])
    q = randn(g, 2, drafts, 32, 128, dtype=torch.bfloat16)
    want = F.draft_attention(q, *args)
    for _ in range(3):
        assert torch.equal(F.draft_attention(q, *args), want)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    outs = [torch.zeros_like(q) for _ in range(2)]
    graphs = []
    with torch.cuda.stream(s):
        got = F.draft_attention(q, *args)
        for out in outs:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=s):
                F.draft_attention(q, *args, out=out)
            graphs.append(graph)
    s.synchronize()
    assert torch.equal(got, want)
    other = torch.cuda.Stream()
    for _ in range(3):
        for graph, stream in zip(graphs, (s, other)):   # side by side, and beside a call
            with torch.cuda.stream(stream):
                graph.replay()
        assert torch.equal(F.draft_attention(q, *args), want)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], want) and torch.equal(outs[1], want)


def test_refusals():
    q = torch.zeros(2, 3, 4, 64, device="cuda", dtype=torch.bfloat16)
    kc = torch.zeros(5, 8, 2, 64, device="cuda", dtype=torch.bfloat16)
    pages = torch.zeros(2, 2, device="cuda", dtype=torch.int32)
    ns = torch.zeros(2, device="cuda", dtype=torch.int32)
    words = torch.ones(2, 3, device="cuda", dtype=torch.int64)

    def call(**kw):
        a = dict(q=q, k=kc, v=kc, pages=pages, lengths=ns, masks=words) | kw
        extra = {n: a.pop(n) for n in ("out", "slopes", "scale", "softcap") if n in a}
        return F.draft_attention(*a.values(), **extra)
    call()
    for bad in ({"q": q[0]}, {"masks": words[:, :2]}, {"masks": words[:1]}, {"lengths": ns[:1]}, {"pages": pages[:1]}, {"v": kc[:, :4]},
                {"k": kc[:, :, :1]}, {"q": q[:, :0]}, {"q": q.transpose(2, 3)}, {"out": q[:, :2]}, {"slopes": torch.zeros(3, device="cuda")},
                {"q": torch.zeros(2, 65, 4, 64, device="cuda", dtype=torch.bfloat16),
                 "masks": torch.ones(2, 65, device="cuda", dtype=torch.int64)}):
        with pytest.raises(ValueError):
            call(**bad)
    for bad in ({"masks": words.int()}, {"masks": None}, {"lengths": ns.long()}, {"q": q.float()}, {"q": q.cpu()}, {"pages": pages.long()}):
        with pytest.raises(TypeError):
            call(**bad)
    for bad in ({"scale": math.nan}, {"softcap": -1.0}, {"out": q[:, :1].expand(2, 3, 4, 64)}, {"out": kc[:2, :3].repeat(1, 1, 2, 1)[:, :, :1].expand(2, 3, 4, 64)}):
        with pytest.raises(F._zo.ZoError):
            call(**bad)
    with pytest.raises(F._zo.ZoError):
        call(out=kc.view(-1)[:q.numel()].view(q.shape))
    with pytest.raises(RuntimeError):
        call(q=q.clone().requires_grad_())
    with torch.no_grad():
        call(q=q.clone().requires_grad_())
    for bad in (torch.zeros(2, 3, device="cuda", dtype=torch.int64), torch.zeros(2, 3, dtype=torch.int32), None):
        with pytest.raises(TypeError):
            F.draft_masks(bad)
    for bad in (torch.zeros(3, device="cuda", dtype=torch.int32), torch.zeros(2, 65, device="cuda", dtype=torch.int32),
                torch.zeros(2, 0, device="cuda", dtype=torch.int32), torch.zeros(3, 2, device="cuda", dtype=torch.int32).T):
        with pytest.raises(ValueError):
            F.draft_masks(bad)
