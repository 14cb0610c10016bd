"""Tangents of forward-mode differentiation are refused as gradients are."""
import pytest
import torch
from torch.autograd import forward_ad

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


def calls():
    """One call per operator as a function of the tensor that it would be differentiated by."""
    spans = F.document_spans(ints(0, 4), tokens=4)
    table, positions = F.rotary_table(8, 64), ints(0, 1, 2, 3, dtype=torch.int64)
    return [
        (heads(4, 2, 64), lambda q: F.rotate_heads(q, table=table, positions=positions)),
        (heads(64), lambda w: F.rotate_heads(heads(4, 2, 64), table=table, positions=positions, q_weight=w)),
        (heads(4, 2, 64), lambda v: F.attention(heads(4, 2, 64), heads(4, 2, 64), v, spans)),
        (heads(2, 2, 64), lambda q: F.decode_attention(q, heads(9, 8, 1, 64), heads(9, 8, 1, 64), ints(0, 1)[:, None], ints(3, 4))),
        (heads(4, 64), lambda x: F.token_loss(x, positions)),
    ]


@pytest.mark.parametrize("n", range(5))
def test_tangents_are_refused(n):
    x, call = calls()[n]
    call(x)
    with forward_ad.dual_level():
        dual = forward_ad.make_dual(x, torch.ones_like(x))
        with pytest.raises(RuntimeError, match="gradient"):
            call(dual)
        with torch.no_grad(), pytest.raises(RuntimeError, match="gradient"):   # which leaves tangents alone
            call(dual)
        call(forward_ad.unpack_dual(dual).primal)
    with pytest.raises(RuntimeError):
        torch.func.jvp(call, (x,), (torch.ones_like(x),))
    call(x)
