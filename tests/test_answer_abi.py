"""The operators of learning from answers without a GPU: what their calls refuse (addresses here are never dereferenced)."""
import ctypes

import pytest
import torch

from paper_2609_38095_gb300 import build as zo_build
from paper_2609_38095_gb300 import forward, zo

FAKE = 0x7F0000000000
FAR = [FAKE + (i << 34) for i in range(10)]
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def L():
    zo_build.build()
    return forward._lib()


_kept = []


def pages(*v):
    _kept.append((ctypes.c_int64 * 4)(*v))
    return ctypes.addressof(_kept[-1])


def test_draft_masks(L):
    def call(parents=FAKE, batch=3, drafts=8, masks=FAR[1]):
        return L.zo_draft_masks(parents, batch, drafts, masks, None)
    for bad in ({"batch": -1}, {"batch": 1 << 40}, {"drafts": 0}, {"drafts": 65}, {"drafts": -1}, {"parents": None}, {"masks": None},
                {"masks": FAKE}, {"masks": FAKE + 88}, {"masks": FAKE - 184}):
        assert call(**bad) == zo.ZO_ERR_ARG, bad
    assert call(parents=FAKE + 2) == zo.ZO_ERR_ALIGN and call(masks=FAR[1] + 4) == zo.ZO_ERR_ALIGN
    assert call(batch=0, parents=None, masks=None) == zo.ZO_OK


def test_attention_draft(L):
    def call(q=pages(FAR[0], 1024, 128, 64), k=pages(FAR[1], 1024, 64, 64), v=pages(FAR[2], 1024, 64, 64),
             out=pages(FAR[3], 1024, 128, 64), batch=2, drafts=8, heads=2, kv=1, dim=64, dtype=1, table=FAKE, stride=4, most=4, n=9,
             page=16, lengths=FAKE, masks=FAKE, scale=1.0, cap=0.0, slopes=None, lse=None, work=FAR[5], wb=1 << 30):
        return L.zo_attention_draft(q, k, v, out, batch, drafts, heads, kv, dim, dtype, table, stride, most, n, page, lengths, masks,
                                    scale, cap, slopes, lse, work, wb, None)
    for bad in ({"q": None}, {"k": None}, {"v": None}, {"out": None}, {"q": pages(0, 1, 1, 1)}, {"k": pages(0, 1, 1, 1)},
                {"v": pages(FAKE, 1, -1, 1)}, {"q": pages(FAKE, -1, 1, 1)}, {"out": pages(0, 1, 1, 1)}, {"batch": -1}, {"batch": 1 << 26},
                {"drafts": 0}, {"drafts": 65}, {"heads": 3, "kv": 2}, {"heads": 1025}, {"dim": 300}, {"table": None}, {"stride": -1},
                {"most": -1}, {"n": -1}, {"most": 1 << 31}, {"page": 0}, {"lengths": None}, {"masks": None}, {"scale": INF}, {"cap": -2.0},
                {"cap": NAN},
                {"out": pages(FAR[0], 1024, 64, 128)},             # over q with other strides
                {"out": pages(FAR[0] + 128, 1024, 128, 64)},
                {"out": pages(FAR[1] + 64, 1024, 128, 64)}, {"out": pages(FAR[2], 1024, 128, 64)},
                {"out": pages(FAR[3], 512, 128, 64)},              # sequences over one another
                {"out": pages(FAR[3], 1024, 0, 64)}, {"out": pages(FAR[3], 1024, 128, 32)}):
        assert call(**bad) == zo.ZO_ERR_ARG, bad
    assert call(dtype=5) == zo.ZO_ERR_DTYPE
    for bad in ({"k": pages(FAR[1] + 1, 1, 1, 1)}, {"q": pages(FAR[1] + 1, 1, 1, 1)}, {"table": FAKE + 1}, {"lengths": FAKE + 2},
                {"lse": FAKE + 2}, {"slopes": FAKE + 1}):
        assert call(**bad) == zo.ZO_ERR_ALIGN, bad
    assert call(batch=0, lengths=None, masks=None) == zo.ZO_OK
    size = L.zo_attention_draft_workspace_size
    for few in ((2, 8, 2, 1, 64, 1), (2, 8, 4, 2, 64, 2), (2, 64, 4, 1, 64, 0), (2, 64, 4, 1, 200, 1), (2, 0, 2, 1, 64, 1), (2, 8, 3, 2, 64, 1), (-1, 64, 4, 1, 64, 1)):
        assert size(*few) == 0, few
    assert size(2, 64, 4, 1, 64, 1) % 16 == 0 and size(500, 64, 4, 1, 64, 1) > size(2, 64, 4, 1, 64, 1) > 0


def test_policy_loss(L):
    ws = L.zo_policy_loss_workspace_size(10)
    assert ws >= 200 and ws % 8 == 0 and L.zo_policy_loss_workspace_size(0) > 0

    def call(logits=FAR[0], row=100, tokens=10, vocab=100, dtype=1, targets=FAR[1], tb=8, old=FAR[2], a=FAR[3], ref=None, w=None,
             low=0.2, high=0.2, kl=0.0, flags=0, loss=FAR[4], grad=None, grad_row=100, scale=1.0, logp=None, work=FAR[5], wb=ws):
        return L.zo_policy_loss(logits, row, tokens, vocab, dtype, targets, tb, old, a, ref, w, low, high, kl, flags, loss, grad,
                                grad_row, scale, logp, work, wb, None)
    for bad in ({"tokens": -1}, {"tokens": 1 << 29}, {"vocab": 0}, {"vocab": 1 << 31}, {"row": -1}, {"tb": 2}, {"flags": 8}, {"flags": 16},
                {"loss": None}, {"logits": None}, {"targets": None}, {"old": None}, {"a": None}, {"kl": 0.1}, {"kl": NAN, "ref": FAR[6]},
                {"kl": -1.0, "ref": FAR[6]}, {"low": -0.1}, {"low": 1.1}, {"low": NAN}, {"high": -0.1}, {"high": INF}, {"high": NAN},
                {"grad": FAR[7], "grad_row": -1}, {"grad": FAR[7], "grad_row": 99}, {"grad": FAR[7], "scale": NAN},
                {"grad": FAR[0] + 2}, {"grad": FAR[0], "grad_row": 101}, {"grad": FAR[1] + 8}, {"grad": FAR[2] - 20}, {"grad": FAR[4] - 8},
                {"loss": FAR[0] + 80}, {"loss": FAR[3] + 32}, {"logp": FAR[0]}, {"logp": FAR[2]}, {"logp": FAR[4] - 36},
                {"logp": FAR[7] + 8, "grad": FAR[7]}):
        assert call(**bad) == zo.ZO_ERR_ARG, bad
    assert call(dtype=3) == zo.ZO_ERR_DTYPE
    for bad in ({"logits": FAKE + 1}, {"targets": FAR[1] + 4}, {"loss": FAR[4] + 4}, {"old": FAR[2] + 2}, {"a": FAR[3] + 1}, {"w": FAR[6] + 2},
                {"ref": FAR[6] + 2}, {"grad": FAR[7] + 1}, {"logp": FAR[8] + 2}, {"work": FAR[5] + 4}):
        assert call(**bad) == zo.ZO_ERR_ALIGN, bad
    assert call(work=None) == zo.ZO_ERR_WORKSPACE and call(wb=ws - 1) == zo.ZO_ERR_WORKSPACE


def test_preference_loss(L):
    ws = L.zo_preference_loss_workspace_size(10, 3)
    assert ws >= 248 and ws % 8 == 0 and L.zo_preference_loss_workspace_size(0, 0) > 0

    def call(logits=FAR[0], row=100, tokens=10, vocab=100, dtype=1, targets=FAR[1], tb=4, starts=FAR[2], pairs=3, ref=None, beta=0.1,
             margin=0.0, smoothing=0.0, flags=0, loss=FAR[4], grad=None, grad_row=100, scale=1.0, logp=None, work=FAR[5], wb=ws):
        return L.zo_preference_loss(logits, row, tokens, vocab, dtype, targets, tb, starts, pairs, ref, beta, margin, smoothing, flags,
                                    loss, grad, grad_row, scale, logp, work, wb, None)
    for bad in ({"tokens": -1}, {"vocab": 0}, {"row": -1}, {"tb": 1}, {"flags": 16}, {"loss": None}, {"logits": None}, {"targets": None},
                {"starts": None}, {"pairs": -1}, {"pairs": 1 << 40}, {"beta": -0.1}, {"beta": INF}, {"beta": NAN}, {"margin": INF},
                {"smoothing": -0.1}, {"smoothing": 1.1}, {"smoothing": NAN}, {"grad": FAR[7], "scale": INF}, {"grad": FAR[7], "grad_row": 0},
                {"grad": FAR[2]}, {"logp": FAR[2] + 8}, {"logp": FAR[6], "ref": FAR[6]}, {"loss": FAR[2] + 24}):
        assert call(**bad) == zo.ZO_ERR_ARG, bad
    assert call(dtype=-1) == zo.ZO_ERR_DTYPE
    for bad in ({"starts": FAR[2] + 2}, {"ref": FAR[3] + 2}, {"loss": FAR[4] + 4}, {"logp": FAR[6] + 1}, {"work": FAR[5] + 4}):
        assert call(**bad) == zo.ZO_ERR_ALIGN, bad
    assert call(work=None) == zo.ZO_ERR_WORKSPACE and call(wb=ws - 1) == zo.ZO_ERR_WORKSPACE


def test_binding_refuses_cpu_tensors():
    x = torch.zeros(4, 2, 3, 8)
    i = torch.zeros(4, 3, dtype=torch.int64)
    f = torch.zeros(4)
    with pytest.raises(TypeError):
        forward.draft_attention(x, x, x, i, i, i)
    with pytest.raises(TypeError):
        forward.draft_masks(i.int())
    with pytest.raises(TypeError):
        forward.policy_loss(x[0, 0], i[:, 0], f, f)
    with pytest.raises(TypeError):
        forward.preference_loss(x[0, 0], i[:, 0], i[0])
    for call in (forward.policy_loss, forward.preference_loss):
        with pytest.raises(ValueError):
            call(x[0, 0], i[:, 0], *[f] * (2 if call is forward.policy_loss else 1), dtype=torch.float16)
