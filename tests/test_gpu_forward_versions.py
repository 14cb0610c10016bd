"""Outputs that a call writes in place have a new version, as after an in-place operation of torch."""
import pytest
import torch

from paper_2609_38095_gb300 import build as zo_build
from paper_2609_38095_gb300 import forward as F

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    zo_build.build()


def heads(*shape):
    return torch.ones(*shape, device="cuda")


def ints(*v, dtype=torch.int32):
    return torch.tensor(v, dtype=dtype, device="cuda")


def test_outputs_in_place_are_seen_by_autograd():
    """A tensor that a call writes has a new version: a backward pass that saved it before raises, not uses it."""
    q, k = heads(4, 2, 64), heads(4, 1, 64)
    spans = F.document_spans(ints(0, 4), tokens=4)
    table, positions = F.rotary_table(8, 64), ints(0, 1, 2, 3, dtype=torch.int64)
    kc, vc = heads(9, 8, 1, 64), heads(9, 8, 1, 64)
    table_of_losses = torch.zeros(3, 3, dtype=torch.float64, device="cuda")
    out = heads(4, 2, 64)
    for written, call in (
            ((q, k), lambda: F.rotate_heads(q, k, table=table, positions=positions, q_out=q, k_out=k)),
            ((kc, vc), lambda: F.rotate_heads(q, k, k, table=table, positions=positions, k_out=kc, v_out=vc, slots=positions)),
            ((out,), lambda: F.attention(q, k, k, spans, out=out)),
            ((out,), lambda: F.decode_attention(q[:2], kc, vc, ints(0, 1)[:, None], ints(3, 4), out=out[:2])),
            ((table_of_losses,), lambda: F.token_loss(heads(4, 64), positions, out=table_of_losses[1, 1:2]))):
        before = [t._version for t in written]
        call()
        assert all(t._version > v for t, v in zip(written, before))
    w = heads(4, 2, 64).requires_grad_(True)
    loss = (w * out).sum()                      # saves out
    F.attention(q, k, k, spans, out=out)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()


def test_inference_mode():
    spans = F.document_spans(ints(0, 4), tokens=4)
    with torch.inference_mode():
        q = heads(4, 2, 64)
        out = torch.zeros_like(q)
        F.attention(q, q, q, spans, out=out)
    q = heads(4, 2, 64)
    F.attention(q, q, q, spans, out=out)         # a tensor of inference mode has no version
    assert torch.equal(out, F.attention(q, q, q, spans))
