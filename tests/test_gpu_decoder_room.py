"""The example's answers: a sequence that has no page for its next token does not write to another's."""
import pytest
import torch

import decoder_step as D
from paper_2609_38095_gb300 import build as zo_build

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    zo_build.build()


def test_the_last_row_is_the_last():
    """Two sequences of 3 and 20 tokens with room for 5 more in pages of 4: the first has 8 rows, the second 28."""
    model = D.Decoder(seed=4)
    answer = D.Answer(model, [[1, 2, 3], list(range(20))], room=5, page_size=4)
    assert torch.equal(answer.pages[0] >= 0, torch.tensor([True] * 2 + [False] * 5, device="cuda"))
    for n in range(5):
        answer.next(torch.tensor([n, n], device="cuda"))
    bits = lambda: [c.view(torch.int16).clone() for pair in answer.caches for c in pair]  # noqa: E731 (unwritten rows may be NaN)
    before = bits()
    lengths = answer.lengths.clone()
    with pytest.raises(ValueError, match="room"):
        answer.next(torch.tensor([5, 5], device="cuda"))
    assert torch.equal(answer.lengths, lengths)
    assert all(torch.equal(x, y) for x, y in zip(bits(), before))


def test_rows_without_a_page_have_no_slot():
    model = D.Decoder(seed=4)
    answer = D.Answer(model, [[1, 2, 3], list(range(20))], room=5, page_size=4)
    slots = answer._slots(torch.tensor([0, 0, 1], device="cuda"), torch.tensor([7, 8, 8], device="cuda"))
    assert slots[0] >= 0 and slots[1] < 0 and slots[2] >= 0
