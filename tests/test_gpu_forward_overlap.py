"""Which outputs may lie in the memory of the inputs: those that share no element with them, and each operator's own
in-place form."""
import pytest
import torch

from paper_2609_38095_gb300 import build as zo_build
from paper_2609_38095_gb300 import forward as F
from paper_2609_38095_gb300 import zo

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    zo_build.build()


def randn(seed, *shape, dtype=torch.bfloat16):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(*shape, generator=g, device="cuda").to(dtype)


def ints(*v, dtype=torch.int32):
    return torch.tensor(v, dtype=dtype, device="cuda")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_attention_beside_its_inputs(dtype):
    t, heads, dim = 200, 4, 64
    spans = F.document_spans(ints(0, 90, t), tokens=t)
    rows = randn(1, t, 4 * heads * dim, dtype=dtype)
    q, k, v, out = (x.view(t, heads, dim) for x in rows.split(heads * dim, 1))
    want = F.attention(q.clone(), k.clone(), v.clone(), spans)
    F.attention(q, k, v, spans, out=out)                       # a fourth part of the same rows
    assert torch.equal(out, want)
    mixed = randn(2, t, 2 * heads, dim, dtype=dtype)           # heads of queries and outputs in turn
    q, out = mixed[:, ::2], mixed[:, 1::2]
    want = F.attention(q.clone(), k, v, spans)
    F.attention(q, k, v, spans, out=out)
    assert torch.equal(out, want)
    first = randn(3, 2 * heads, t, dim, dtype=dtype)           # heads first, outputs behind
    q, out = first[:heads].transpose(0, 1), first[heads:].transpose(0, 1)
    want = F.attention(q.clone(), k, v, spans)
    F.attention(q, k, v, spans, out=out)
    assert torch.equal(out, want)
    for bad in (q, k, v, q[:, :1].expand(t, heads, dim)):
        with pytest.raises(zo.ZoError):
            F.attention(q, k, v, spans, out=bad)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_decode_in_place(dtype):
    q, kc, vc = randn(1, 3, 4, 64, dtype=dtype), randn(2, 9, 8, 2, 64, dtype=dtype), randn(3, 9, 8, 2, 64, dtype=dtype)
    pages, lengths = ints(*range(9)).view(3, 3), ints(20, 1, 24)
    want = F.decode_attention(q, kc, vc, pages, lengths)
    with pytest.raises(zo.ZoError):
        F.decode_attention(q, kc, vc, pages, lengths, out=kc[0, :3, :1].expand(3, 4, 64))
    with pytest.raises(zo.ZoError):
        F.decode_attention(q[:, :2], kc, vc, pages, lengths, out=vc[2, :3])
    with pytest.raises(zo.ZoError):
        F.decode_attention(q[:2], kc, vc, pages[:2], lengths[:2], out=q[1:])
    assert torch.equal(F.decode_attention(q, kc, vc, pages, lengths, out=q), want)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rotate(dtype):
    t, dim = 24, 64
    table, positions = F.rotary_table(64, dim), torch.arange(t, device="cuda")
    common = {"table": table, "positions": positions}
    rows = randn(1, t, 6, dim, dtype=dtype)
    q, k = rows[:, :4], rows[:, 4:]
    want_q, want_k = F.rotate_heads(q.clone(), k.clone(), **common)
    for kw in ({"q_out": k[:, :1].expand(t, 4, dim)}, {"q_out": rows[:, 1:5]}, {"k_out": q[:, :2]}, {"q_out": rows[:, 2:]}):
        with pytest.raises(zo.ZoError):
            F.rotate_heads(q, k, **kw, **common)
    cache = randn(2, 3, 8, 2, dim, dtype=dtype)
    slots = torch.arange(t, device="cuda")
    with pytest.raises(zo.ZoError):                            # keys and values to the same rows
        F.rotate_heads(q, k, k, k_out=cache, v_out=cache, slots=slots, **common)
    with pytest.raises(zo.ZoError):                            # from the cache to other rows of it
        F.rotate_heads(q[:8], cache[1], k_out=cache, slots=slots[:8], table=table, positions=positions[:8])
    same = cache.view(t, 2, dim)                               # each to its own row
    want = F.rotate_heads(same.clone(), **common)
    F.rotate_heads(q, same, k_out=same, slots=slots, **common)
    assert torch.equal(same, want)
    F.rotate_heads(q, k, q_out=q, k_out=k, **common)           # in place within one projection
    assert torch.equal(q, want_q) and torch.equal(k, want_k)
