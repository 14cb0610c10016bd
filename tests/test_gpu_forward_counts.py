"""Counts that do not fit 32 bits are refused, not cut to their lower half."""
import pytest
import torch

from paper_2609_38095_gb300 import build as zo_build
from paper_2609_38095_gb300 import forward as F

pytestmark = pytest.mark.gpu

MANY = (1 << 32) + 2


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    zo_build.build()


def zeros(*shape, dtype=torch.bfloat16):
    return torch.zeros(*shape, dtype=dtype, device="cuda")


def test_heads():
    """No tokens, so that nothing is computed: 2^32 + 2 heads are not 2."""
    q, k = zeros(0, 1, 8).expand(0, MANY, 8), zeros(0, 2, 8)
    spans = zeros(3, 0, dtype=torch.int32)
    with pytest.raises(ValueError):
        F.attention(q, k, k, spans)
    with pytest.raises(ValueError):
        F.attention(q, q, q, spans)
    with pytest.raises(ValueError):
        F.decode_attention(q, zeros(1, 1, 2, 8), zeros(1, 1, 2, 8), zeros(0, 1, dtype=torch.int32), zeros(0, dtype=torch.int32))
    with pytest.raises(ValueError):
        F.rotate_heads(q, table=F.rotary_table(4, 8), positions=zeros(0, dtype=torch.int64))


def test_page_size():
    """Pages of 2^32 + 2 rows (all of them the same one) are not pages of 2."""
    q = zeros(1, 1, 8)
    cache = zeros(1, 1, 1, 8).expand(1, MANY, 1, 8)
    with pytest.raises(ValueError):
        F.decode_attention(q, cache, cache, zeros(1, 1, dtype=torch.int32), torch.ones(1, dtype=torch.int32, device="cuda"))
