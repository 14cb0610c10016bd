"""What the Python functions of a forward point refuse without a GPU."""
import pytest
import torch

from paper_2609_38095_gb300 import build as zo_build
from paper_2609_38095_gb300 import forward


@pytest.mark.parametrize("starts", [[0, 3], None, torch.tensor([0, 3], dtype=torch.int32)])
def test_document_spans_wants_a_cuda_tensor(starts):
    zo_build.build()
    with pytest.raises(TypeError, match="q_starts must be a CUDA tensor"):
        forward.document_spans(starts, tokens=3)
