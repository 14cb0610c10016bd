"""Head norms and rotation (zo_rotate_heads), the rotary table and document spans against 64 bits."""
import math

import numpy as np
import pytest
import torch

import forward_ref as R
from paper_2609_38095_gb300 import build as zo_build
from paper_2609_38095_gb300 import forward as F

pytestmark = pytest.mark.gpu

DTYPES = [torch.bfloat16, torch.float16, torch.float32]


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    zo_build.build()


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(g, *shape, dtype):
    return torch.randn(*shape, generator=g, device="cuda").to(dtype)


def test_table():
    got = F.rotary_table(5000, 64, base=1e6).double().cpu().numpy()
    w = 1e6 ** (-np.arange(0, 64, 2) / 64.0)
    ang = np.arange(5000)[:, None] * w
    assert np.abs(got - np.concatenate([np.cos(ang), np.sin(ang)], 1)).max() <= 2.0 ** -24 * 1.01 + 5000 * 2.0 ** -50


@pytest.mark.parametrize("original", [0, 4096])
def test_table_scaled(original):
    got = F.rotary_table(70000, 128, base=1e4, scale=8.0, original=original, low=1.0, high=32.0, magnitude=1.2)
    w = 1e4 ** (-np.arange(0, 128, 2) / 128.0)
    g = np.clip((original * w / (2 * np.pi) - 1.0) / 31.0, 0, 1) if original else 0.0
    ang = np.arange(70000)[:, None] * (w * ((1 - g) / 8.0 + g))
    want = 1.2 * np.concatenate([np.cos(ang), np.sin(ang)], 1)
    assert np.abs(got.double().cpu().numpy() - want).max() <= 1.2 * (2.0 ** -24 * 1.01 + 70000 * 2.0 ** -49)


SHAPES = [(128, 128), (128, 64), (64, 64), (64, 32), (80, 80), (80, 32), (96, 48), (256, 256), (256, 64), (16, 16), (32, 16),
          (33, 2), (7, 6), (2, 2), (200, 200), (130, 128)]


@pytest.mark.parametrize("dtype", DTYPES, ids=["bf16", "f16", "f32"])
@pytest.mark.parametrize("dim,rotary", SHAPES)
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rotate(dtype, dim, rotary, layout):
    """q and k as views of a fused projection, with and without norms; values copied; sizes that end inside a CTA."""
    for n, (t, hq, hk, norm, offset) in enumerate([(1, 1, 1, True, 0), (9, 7, 1, False, 0), (37, 32, 8, True, 0),
                                                   (70, 5, 5, True, 1)]):
        g = gen(100 * dim + n)
        flat = randn(g, t * (hq + 2 * hk) * dim + offset, dtype=dtype)
        qkv = flat[offset:].view(t, -1)
        q, k, v = (x.view(t, -1, dim) for x in qkv.split([hq * dim, hk * dim, hk * dim], 1))
        table = F.rotary_table(64, rotary, base=1e4)
        pos = torch.randint(0, 64, (t,), generator=g, device="cuda", dtype=torch.int64 if n % 2 else torch.int32)
        wq, wk = ((1 + 0.2 * randn(g, dim, dtype=torch.float32)).to(dtype if n else torch.float32) for _ in range(2))
        keep = flat.clone()
        got = F.rotate_heads(q, k, v, table=table, positions=pos, q_weight=wq if norm else None,
                             k_weight=wk if norm else None, eps=1e-5, layout=layout)
        assert torch.equal(flat, keep)
        for x, w, y in ((q, wq, got[0]), (k, wk, got[1])):
            want, size = R.rotate(x, w if norm else None, table, pos, 1e-5, layout)
            R.check(y, want, R.rotate_bound(want, size, dtype, dim), (t, hq, norm))
        assert torch.equal(got[2], v)
        # in place: the same bits
        F.rotate_heads(q, k, table=table, positions=pos, q_weight=wq if norm else None, k_weight=wk if norm else None,
                       eps=1e-5, layout=layout, q_out=q, k_out=k)
        assert torch.equal(q, got[0]) and torch.equal(k, got[1])


@pytest.mark.parametrize("dtype", DTYPES, ids=["bf16", "f16", "f32"])
@pytest.mark.parametrize("dim", [128, 80, 33])
@pytest.mark.parametrize("layout", ["pages", "heads first", "rows"])
def test_append(dtype, dim, layout):
    """Keys and values at their slots of a cache; every other row keeps its bits, and tokens without a slot write none."""
    t, hk, pages, size = 23, 3, 9, 5
    g = gen(7 + dim)
    rotary = dim // 2 * 2
    q, k, v = (randn(g, t, h, dim, dtype=dtype) for h in (6, hk, hk))
    shape = {"pages": (pages, size, hk, dim), "heads first": (pages, hk, size, dim), "rows": (pages * size, hk, dim)}[layout]
    kc, vc = (randn(g, *shape, dtype=dtype) for _ in range(2))
    if layout == "heads first":
        kc, vc = kc.transpose(1, 2), vc.transpose(1, 2)
    table = F.rotary_table(40, rotary)
    pos = torch.randint(0, 40, (t,), generator=g, device="cuda")
    slots = torch.randperm(pages * size, generator=g, device="cuda")[:t]
    slots[3], slots[11] = -1, pages * size     # no row of the cache
    want_k, _ = R.rotate(k, None, table, pos, 0, "half")
    plain = F.rotate_heads(q, k, table=table, positions=pos)
    before = [x.clone() for x in (kc, vc)]
    out, kc2, vc2 = F.rotate_heads(q, k, v, table=table, positions=pos, k_out=kc, v_out=vc, slots=slots)
    assert kc2 is kc and vc2 is vc and torch.equal(out, plain[0])
    for cache, old, new in ((kc, before[0], plain[1]), (vc, before[1], v)):
        rows = old.reshape(pages * size, hk, dim).clone()
        for i, s in enumerate(slots.tolist()):
            if 0 <= s < pages * size:
                rows[s] = new[i]
        assert torch.equal(cache.reshape(pages * size, hk, dim), rows)


def test_positions_outside_the_table_are_nan():
    g = gen(3)
    q = randn(g, 6, 2, 128, dtype=torch.bfloat16)
    table = F.rotary_table(10, 64)
    pos = torch.tensor([0, 10, 9, -1, 1 << 40, 5], device="cuda")
    for x in (q, randn(g, 6, 2, 127, dtype=torch.bfloat16)):
        got = F.rotate_heads(x, table=table, positions=pos)
        bad = torch.tensor([False, True, False, True, True, False], device="cuda")
        assert torch.isnan(got[bad][..., :64]).all() and torch.isfinite(got[~bad]).all()
        assert torch.equal(got[bad][..., 64:], x[bad][..., 64:])


def test_no_tokens_and_other_stream():
    table = F.rotary_table(10, 64)
    empty = torch.empty(0, 4, 64, device="cuda", dtype=torch.float16)
    assert F.rotate_heads(empty, table=table, positions=torch.empty(0, dtype=torch.int64, device="cuda")).shape == (0, 4, 64)
    q = randn(gen(1), 300, 4, 64, dtype=torch.float16)
    pos = torch.arange(300, device="cuda") % 10
    want = F.rotate_heads(q, table=table, positions=pos)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = F.rotate_heads(q, table=table, positions=pos)
    s.synchronize()
    assert torch.equal(got, want)


@pytest.mark.parametrize("case", range(8))
def test_spans(case):
    rng = np.random.default_rng(case)
    docs = [0, 1, 2, 5, 40, 7, 3, 11][case]
    qn = rng.integers(0, 9, docs)
    kn = rng.integers(0, 12, docs) if case % 2 else qn
    qs, ks = (np.concatenate([[0], np.cumsum(x)]).astype(np.int32) for x in (qn, kn))
    prefix = rng.integers(0, 15, docs).astype(np.int32) if case in (2, 3, 4) else None
    t = int(qs[-1]) + case
    dev = lambda a: torch.from_numpy(a).cuda()  # noqa: E731
    got = F.document_spans(dev(qs), None if kn is qn else dev(ks), None if prefix is None else dev(prefix), tokens=t).cpu().numpy()
    for i in range(docs):
        for r in range(qn[i]):
            row = qs[i] + r
            own = ks[i + 1] - (qn[i] - r)
            keys = [j for j in range(ks[i], ks[i + 1]) if j <= own or (prefix is not None and j - ks[i] < prefix[i])]
            seen = [j for j in range(int(ks[-1])) if got[0, row] <= j < got[1, row]]
            assert seen == keys, (i, r)
            assert got[2, row] == own
    assert (got[:, int(qs[-1]):] == 0).all()
