"""Forms of the forward point's calls that its other tests leave out: the caller's scale, weights of another type on
aligned heads, calls from two host threads."""
import threading

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
@pytest.mark.parametrize("scale", [0.3, 0.0, -0.2])
@pytest.mark.parametrize("softcap,biased", [(0.0, False), (5.0, False), (0.0, True), (5.0, True)])
def test_scale(dtype, scale, softcap, biased):
    dim, lengths = 64, [70, 1, 140]
    t = sum(lengths)
    q, k, v = (randn(i, t, 2 if i else 4, dim, dtype=dtype) for i in range(3))
    slopes = torch.tensor([0.5, 0.25, 0.125, 0.0625], device="cuda") if biased else None
    spans = F.document_spans(torch.tensor([0, 70, 71, t], dtype=torch.int32, device="cuda"), tokens=t)
    out, lse = F.attention(q, k, v, spans, scale=scale, softcap=softcap, slopes=slopes, with_lse=True)
    s = spans.long()
    want, want_lse, worst, weighted = R.attention(q, k, v, s[0], s[1], s[2], scale, softcap, slopes)
    R.check(out, want, R.attention_bound(want, weighted, worst, dtype, dim, t), "out")
    R.check(lse, want_lse, R.lse_bound(want_lse, worst, dim, t), "lse")
    # the last row of each document, over pages
    page, ends, starts = 16, [69, 70, t - 1], [0, 70, 71]
    need = [-(-n // page) for n in lengths]
    kc, vc = (torch.full((sum(need), page, 2, dim), float("nan"), dtype=dtype, device="cuda") for _ in range(2))
    pages = torch.full((3, max(need)), -1, dtype=torch.int32, device="cuda")
    for b, n in enumerate(lengths):
        at = sum(need[:b])
        pages[b, :need[b]] = torch.arange(at, at + need[b], dtype=torch.int32)
        for cache, x in ((kc, k), (vc, v)):
            cache[at:at + need[b]].view(-1, 2, dim)[:n] = x[starts[b]:starts[b] + n]
    out, lse = F.decode_attention(q[ends], kc, vc, pages, torch.tensor(lengths, dtype=torch.int32, device="cuda"), scale=scale,
                                  softcap=softcap, slopes=slopes, with_lse=True)
    R.check(out, want[ends], R.attention_bound(want, weighted, worst, dtype, dim, t)[ends], "decode out")
    R.check(lse.T, want_lse[:, ends], R.lse_bound(want_lse, worst, dim, t)[:, ends], "decode lse")


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("weight", DTYPES, ids=IDS)
@pytest.mark.parametrize("dim,rotary,layout", [(128, 128, "half"), (128, 64, "interleaved"), (64, 64, "half"), (80, 40, "half")])
def test_weights_of_another_type(dtype, weight, dim, rotary, layout):
    t, hq, hk = 300, 8, 2
    q, k = (randn(i, t, h, dim, dtype=dtype) for i, h in enumerate((hq, hk)))
    wq, wk = ((1 + randn(7 + i, dim, dtype=torch.float32, scale=0.2)).to(weight) for i in range(2))
    table = F.rotary_table(512, rotary)
    positions = torch.arange(t, device="cuda") + 3
    got = F.rotate_heads(q, k, table=table, positions=positions, q_weight=wq, k_weight=wk, layout=layout)
    for x, w, y in ((q, wq, got[0]), (k, wk, got[1])):
        want, size = R.rotate(x, w, table, positions, 1e-6, layout)
        R.check(y, want, R.rotate_bound(want, size, dtype, dim))


def test_two_host_threads():
    """Calls on two streams from two threads at once give what they give alone."""
    t, dim = 700, 128
    spans = F.document_spans(torch.tensor([0, 300, t], dtype=torch.int32, device="cuda"), tokens=t)
    table, positions = F.rotary_table(1024, dim), torch.arange(t, device="cuda")
    pages = torch.arange(44, dtype=torch.int32, device="cuda")[None]

    def point(seed):
        q, k, v = (randn(seed + i, t, 8, dim, dtype=torch.bfloat16) for i in range(3))
        logits = randn(seed, 64, 9000, dtype=torch.bfloat16)
        lengths = torch.tensor([t - seed], dtype=torch.int32, device="cuda")

        def run():
            a, b = F.rotate_heads(q, k, table=table, positions=positions)
            out = F.attention(a, b, v, spans)
            cache = torch.zeros(2, 44, 16, 8, dim, dtype=torch.bfloat16, device="cuda")
            cache.view(2, -1, 8, dim)[0, :t], cache.view(2, -1, 8, dim)[1, :t] = b, v
            return out, F.decode_attention(a[-1:], cache[0], cache[1], pages, lengths), F.token_loss(logits, positions[:64])
        return run
    runs = [point(3), point(50)]
    want = [run() for run in runs]
    torch.cuda.synchronize()
    failed = []

    def work(n):
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(50):
                got = runs[n]()
                torch.cuda.current_stream().synchronize()
                if not all(torch.equal(x, y) for x, y in zip(got, want[n])):
                    failed.append(n)
    threads = [threading.Thread(target=work, args=(n,)) for n in range(2)]
    for x in threads:
        x.start()
    for x in threads:
        x.join()
    assert not failed
