"""Attention of packed documents (zo_attention) against 64 bits, within bounds that forward_ref.py derives."""
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


def starts(lengths):
    return torch.tensor([sum(lengths[:i]) for i in range(len(lengths) + 1)], dtype=torch.int32, device="cuda")


def compare(q, k, v, spans, scale=None, softcap=0.0, slopes=None, **kw):
    out, lse = F.attention(q, k, v, spans, scale=scale, softcap=softcap, slopes=slopes, with_lse=True, **kw)
    s = spans.long()
    n, d = k.shape[0], q.shape[2]
    want, want_lse, worst, weighted = R.attention(q, k, v, s[0].clamp(min=0), s[1].clamp(max=n), s[2],
                                                  d ** -0.5 if scale is None else scale, softcap, slopes)
    R.check(out, want, R.attention_bound(want, weighted, worst, q.dtype, d, n), "out")
    R.check(lse, want_lse, R.lse_bound(want_lse, worst, d, n), "lse")
    return out, lse


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("dim", [128, 64, 80, 96, 16, 8, 33, 200, 256])
@pytest.mark.parametrize("heads,kv", [(4, 2), (3, 3), (6, 1)])
def test_documents(dtype, dim, heads, kv):
    """Ragged documents, some of one token and some empty, and rows past the last."""
    lengths = [1, 130, 0, 64, 7, 1, 0, 257, 90]
    t = sum(lengths) + 5
    g = gen(dim * 10 + heads)
    q, k, v = (randn(g, t, h, dim, dtype=dtype, scale=1.5 if h == heads else 1.0) for h in (heads, kv, kv))
    compare(q, k, v, F.document_spans(starts(lengths), tokens=t))


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("t", [1, 2, 63, 64, 65, 127, 128, 129, 255, 256, 257, 383, 640, 1000])
def test_one_document(dtype, t):
    g = gen(t)
    q, k, v = (randn(g, t, h, 128, dtype=dtype) for h in (8, 2, 2))
    compare(q, k, v, F.document_spans(starts([t]), tokens=t))


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("dim", [128, 64, 72, 160])
@pytest.mark.parametrize("softcap,bias,prefix", [(0.0, True, False), (20.0, False, False), (5.0, True, True), (0.0, False, True)])
def test_capped_biased_prefixed(dtype, dim, softcap, bias, prefix):
    """Keys that were there before the queries, fewer keys than queries, a prefix, a cap and a bias by distance."""
    qn, kn = [3, 140, 1, 60, 9], [50, 300, 200, 20, 9]
    g = gen(dim + int(softcap))
    q, k, v = (randn(g, n, h, dim, dtype=dtype, scale=2.0 if h == 6 else 1.0)
               for n, h in ((sum(qn), 6), (sum(kn), 3), (sum(kn), 3)))
    pre = torch.tensor([10, 250, 1, 40, 0], dtype=torch.int32, device="cuda") if prefix else None
    slopes = torch.tensor([2.0 ** -(h + 1) for h in range(6)], device="cuda") if bias else None
    compare(q, k, v, F.document_spans(starts(qn), starts(kn), pre, tokens=sum(qn)), softcap=softcap, slopes=slopes)


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("heads,kv", [(2, 2), (4, 1)])
def test_any_spans(dtype, heads, kv):
    """Spans in no order, empty ones, ones that pass the ends of the keys, windows."""
    t, n = 300, 517
    g = gen(11)
    q, k, v = (randn(g, m, h, 64, dtype=dtype) for m, h in ((t, heads), (n, kv), (n, kv)))
    first = torch.randint(-20, n, (t,), generator=g, device="cuda", dtype=torch.int32)
    end = first + torch.randint(-30, 400, (t,), generator=g, device="cuda", dtype=torch.int32)
    compare(q, k, v, torch.stack([first, end, first]))
    first = torch.zeros(t, dtype=torch.int32, device="cuda")  # two rows of a tile far apart
    first[7::128] = n - 1
    compare(q, k, v, torch.stack([first, first + 1, first]))
    at = torch.arange(t, dtype=torch.int32, device="cuda")    # a sliding window
    compare(q, k, v, torch.stack([(at - 70).clamp(min=0), at + 1, at]))


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
def test_nothing_to_see(dtype):
    q = randn(gen(1), 70, 4, 128, dtype=dtype)
    none = torch.zeros(3, 70, dtype=torch.int32, device="cuda")
    for keys in (0, 40):
        k = randn(gen(2), keys, 2, 128, dtype=dtype)
        out, lse = F.attention(q, k, k, none, with_lse=True)
        assert not out.any() and (lse == -math.inf).all()
    e = torch.empty(0, 4, 128, dtype=dtype, device="cuda")
    assert F.attention(e, q[:, :2], q[:, :2], none[:, :0].contiguous()).shape == e.shape


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("dim", [128, 64, 40, 33, 250])
def test_strides_and_alignment(dtype, dim):
    """Views of a fused projection, heads before tokens, a base off every vector boundary, a wider output."""
    t, hq, hk = 200, 4, 2
    g = gen(dim)
    spans = F.document_spans(starts([70, 130]), tokens=t)
    qkv = randn(g, t, (hq + 2 * hk) * dim, dtype=dtype)
    q, k, v = (x.view(t, -1, dim) for x in qkv.split([hq * dim, hk * dim, hk * dim], 1))
    want, _ = compare(q, k, v, spans)
    first = [x.transpose(0, 1).contiguous().transpose(0, 1) for x in (q, k, v)]
    assert torch.equal(compare(*first, spans)[0], want)
    wide = torch.zeros(t, hq + 1, dim + 24, dtype=dtype, device="cuda")
    compare(q, k, v, spans, out=wide[:, :hq, :dim])
    assert not wide[:, hq].any() and not wide[..., dim:].any()
    off = [torch.empty(x.numel() + 1, dtype=dtype, device="cuda")[1:].view(x.shape).copy_(x) for x in (q, k, v)]
    compare(*off, spans)
    shared = k[:, :1].expand(t, hk, dim)     # one head for all: stride 0
    compare(q, shared, v, spans)


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("dim", [128, 48])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
def test_unseen_keys_do_not_matter(dtype, dim, value):
    """NaN and infinities at keys that some or all rows of a tile do not see."""
    lengths, pad = [100, 60, 150], 30
    t = sum(lengths)
    g = gen(5)
    q, k, v = (randn(g, n, h, dim, dtype=dtype) for n, h in ((t, 4), (t + pad, 2), (t + pad, 2)))
    spans = F.document_spans(starts(lengths), tokens=t)
    want, want_lse = F.attention(q, k[:t], v[:t], spans, with_lse=True)
    k[t:], v[t:] = value, value              # beyond every document: never written memory
    out, lse = F.attention(q, k, v, spans, with_lse=True)
    assert torch.equal(out, want) and torch.equal(lse, want_lse)
    v[120:125], k[121] = value, value        # inside the second document: it shows in its own rows from there on alone
    out, lse = F.attention(q, k, v, spans, with_lse=True)
    clean = torch.ones(t, dtype=torch.bool, device="cuda")
    clean[120:160] = False
    s = spans.long()
    zeroed_k, zeroed_v = k.clone(), v.clone()
    zeroed_k[120:125], zeroed_v[120:125] = 0, 0
    zeroed_k[t:], zeroed_v[t:] = 0, 0
    ref, ref_lse, worst, weighted = R.attention(q, zeroed_k, zeroed_v, s[0], s[1], s[2], dim ** -0.5, 0.0, None)
    R.check(out[clean], ref[clean], R.attention_bound(ref, weighted, worst, dtype, dim, t)[clean])
    R.check(lse[:, clean], ref_lse[:, clean], R.lse_bound(ref_lse, worst, dim, t)[:, clean])
    assert not torch.isfinite(out[120:160]).any()


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
def test_large_scores_and_growing_maxima(dtype):
    """The running maximum moves at every tile, by much: a sum that is not rescaled would overflow or vanish."""
    t = 700
    g = gen(9)
    q = randn(g, t, 2, 64, dtype=dtype).abs() + 0.5
    k = randn(g, t, 2, 64, dtype=dtype)
    ramp = torch.linspace(-6, 6, t, device="cuda")[:, None, None]
    spans = F.document_spans(starts([t]), torch.tensor([0, t], dtype=torch.int32, device="cuda"),
                             torch.tensor([t], dtype=torch.int32, device="cuda"), tokens=t)
    for r in (ramp, -ramp):
        kk = (k.float() * 0.1 + r).to(dtype)
        compare(q, kk, randn(g, t, 2, 64, dtype=dtype), spans)


def test_repeatable_streams_and_graph():
    t = 900
    g = gen(4)
    q, k, v = (randn(g, t, h, 128, dtype=torch.bfloat16) for h in (8, 2, 2))
    spans = F.document_spans(starts([300, 600]), tokens=t)
    want = F.attention(q, k, v, spans)
    for _ in range(3):
        assert torch.equal(F.attention(q, k, v, spans), want)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    out = torch.zeros_like(q)
    with torch.cuda.stream(s):
        got = F.attention(q, k, v, spans)
        F.attention(q, k, v, spans, out=out)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            F.attention(q, k, v, spans, out=out)
    s.synchronize()
    assert torch.equal(got, want)
    out.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("tokens,keys", [(1, 1000), (40, 5000), (130, 900)])
def test_few_rows_many_keys(dtype, tokens, keys):
    """Clusters that share a row's keys, tiles that no row sees among them, and rows that see nothing beside."""
    g = gen(tokens)
    q, k, v = (randn(g, n, 2, 96, dtype=dtype) for n in (tokens, keys, keys))
    for spans in (F.document_spans(starts([tokens]), starts([keys]), tokens=tokens),
                  torch.zeros(3, tokens, dtype=torch.int32, device="cuda")):
        compare(q, k, v, spans)
        if tokens > 40:
            spans[1, 64:] = 0
            compare(q, k, v, spans)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=IDS[:2])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("docs,longest", [(6, 120), (1, 700), (8, 300), (3, 1000)])
def test_many_launches_agree(dtype, dim, docs, longest):
    """Many CTAs per SM, launch after launch on other data in between: the same bits every time, and none that a wait gave
    up on (those are NaN)."""
    g = gen(docs + dim)
    lengths = [longest - (37 * i) % (longest // 2) for i in range(docs)]
    t = sum(lengths)
    spans = F.document_spans(starts(lengths), tokens=t)
    sets = [[randn(g, t, 32, dim, dtype=dtype) for _ in range(3)] for _ in range(2)]
    want = [compare(*x, spans)[0] for x in sets]
    outs = [torch.empty_like(sets[0][0]) for _ in range(40)]
    for i, out in enumerate(outs):
        F.attention(*sets[i % 2], spans, out=out)
    assert all(torch.equal(out, want[i % 2]) for i, out in enumerate(outs))
