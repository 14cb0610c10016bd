"""The example's answers by drafted tokens where sequences differ in how much of their trees is accepted: each takes the room of
its own tokens, and none goes on behind the last that is asked for."""
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


PROMPTS = [[3, 5, 7, 9], [1, 2, 3, 4, 5, 6, 7, 8], [40, 41, 42, 43]]      # whole pages of 4


@pytest.fixture(scope="module")
def model():
    """A trained model in fp32: its best two logits are further apart than two ways' roundings."""
    m = D.Decoder(dtype=torch.float32, seed=2)
    for s in range(6):
        D.step(m, D.Batch([60, 33, 90, 17], m.vocab, s), 1000 + s, 16, 1e-3, 2e-3)
    return m


def proposer(want, vocab, right, nodes=12):
    """Trees of `nodes` tokens: a path of right[b] true ones (where there are as many), and wrong ones beside it."""
    def propose(got):
        trees = []
        for b, g in enumerate(got):
            path = [int(x) for x in want[b, len(g):len(g) + right[b]]]
            true = int(want[b, len(g)]) if len(g) < want.shape[1] else 0
            wrong = [(true + 1 + i) % vocab for i in range(nodes - len(path))]
            trees.append((path + wrong, list(range(-1, len(path) - 1)) + [-1] * len(wrong)))
        return trees
    return propose


@pytest.mark.parametrize("right", [[4, 0, 1], [0, 0, 0], [12, 0, 2], [12, 12, 12]], ids=str)
@pytest.mark.parametrize("n", [1, 8, 20])
@pytest.mark.parametrize("beyond", [0, 4, 16])
def test_room_for_the_tokens(model, right, n, beyond):
    """One sequence accepts whole paths beside one that accepts nothing, with room for the tokens and little beyond."""
    room = -(-n // 4) * 4
    want = D.Answer(model, PROMPTS, room, page_size=4).greedy(room)
    answer = D.Answer(model, PROMPTS, room + beyond, page_size=4)
    got = answer.greedy_drafted(n, proposer(want, model.vocab, right))
    assert torch.equal(got, want[:, :n])
    # what is in the cache: all but the last token, which no pass has seen yet
    assert answer.lengths.tolist() == [len(p) + n - 1 for p in PROMPTS]
    answer.next(got[:, -1])
    if n < room:
        assert torch.equal(answer.logits.argmax(-1), want[:, n])


def test_no_room(model):
    """Pages that end before the tokens do: refused as a token by itself is, and nothing is written outside them."""
    want = D.Answer(model, PROMPTS, 16, page_size=4).greedy(16)
    answer = D.Answer(model, PROMPTS, 8, page_size=4)
    with pytest.raises(ValueError, match="room"):
        answer.greedy_drafted(12, proposer(want, model.vocab, [3, 0, 1]))


def test_draft_of_trees_that_fit_their_own_pages(model):
    """Sizes of the trees on the host: a sequence's pages hold its own tree, not the largest one."""
    answer = D.Answer(model, [[1, 2, 3], list(range(20))], room=5, page_size=4)        # 5 rows left, and 8
    tokens = torch.arange(16, device="cuda").view(2, 8)
    chain = torch.arange(-1, 7, device="cuda", dtype=torch.int32).repeat(2, 1)
    with pytest.raises(ValueError, match="room"):
        answer.draft(tokens, chain)
    with pytest.raises(ValueError, match="room"):
        answer.draft(tokens, chain, sizes=[6, 8])
    cut = chain.clone()
    cut[0, 5:] = -2
    for bad in ([5], [5, 9], [-1, 8], [5, 8, 1]):
        with pytest.raises(ValueError, match="size"):
            answer.draft(tokens, cut, sizes=bad)
    whole = answer.draft(tokens, cut, sizes=[5, 8]).clone()
    again = answer.draft(tokens, chain, sizes=[5, 8])             # what is behind a tree's size is no node
    assert torch.equal(whole[0, :5], again[0, :5]) and torch.equal(whole[1], again[1])
    answer.accept([[0, 1, 2, 3, 4], list(range(8))])
    with pytest.raises(ValueError, match="room"):
        answer.next(torch.tensor([5, 5], device="cuda"))
