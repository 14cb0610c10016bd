"""The decoder example's answers by drafted tokens, and its steps on answers: the operators together, as they are used."""
import pytest
import torch

import decoder_step as D
import paper_2609_38095_gb300 as zo
from paper_2609_38095_gb300 import build as zo_build
from test_gpu_decoder_step import plain_logits

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    zo_build.build()


def plain_after(model, sequences):
    """fp64 logits after each whole sequence."""
    lengths = [len(s) for s in sequences]
    starts = torch.tensor([sum(lengths[:i]) for i in range(len(lengths) + 1)], device="cuda")
    positions = torch.cat([torch.arange(n, device="cuda") for n in lengths])
    return plain_logits(model, torch.tensor(sum(sequences, []), device="cuda"), positions, starts)[starts[1:] - 1]


@pytest.mark.parametrize("dtype,tol", [(torch.float32, 2e-4), (torch.bfloat16, 0.25)], ids=["f32", "bf16"])
def test_drafted_trees(dtype, tol):
    """Each node's logits are those of a packed forward of the sequence and the node's path; a path that is accepted is as if
    its tokens had been appended one by one. Tolerances: those of the example's forward point, derived beside it."""
    model = D.Decoder(dtype=dtype, seed=4)
    sequences = [list(range(1, 20)), [7], list(range(100, 140))]
    answer = D.Answer(model, sequences, room=40, page_size=8)
    shapes = [[-1, 0, 0, 1, 3, 2, -1], [-1, 0, 1, 2, 3, 4, 5], [-1, -1, 1, -2, -2, -2, -2]]
    for turn, paths in enumerate(([[0, 2, 5], [0, 1, 2, 3], [1, 2]], [[6], [], [0]], [[0, 1, 3, 4], [0, 1, 2, 3, 4, 5, 6], []])):
        tokens = [[(31 * turn + 17 * b + 5 * j) % model.vocab for j in range(7)] for b in range(3)]
        got = answer.draft(torch.tensor(tokens, device="cuda"), torch.tensor(shapes, dtype=torch.int32, device="cuda"))
        wholes, places = [], []
        for b, up in enumerate(shapes):
            for j in range(7):
                path, at = [], j
                while at >= 0:
                    path.insert(0, tokens[b][at])
                    at = up[at]
                if at == -1:
                    wholes.append(sequences[b] + path)
                    places.append((b, j))
        want = plain_after(model, wholes)
        have = torch.stack([got[b, j] for b, j in places])
        assert float((have.double() - want).abs().max()) <= tol * max(1.0, float(want.abs().max()) / 4), turn
        answer.accept(paths)
        sequences = [s + [tokens[b][j] for j in path] for b, (s, path) in enumerate(zip(sequences, paths))]
        assert answer.lengths.tolist() == [len(s) for s in sequences]
        want = plain_after(model, sequences)
        assert float((answer.logits.double() - want).abs().max()) <= tol * max(1.0, float(want.abs().max()) / 4), turn
    more = torch.tensor([3, 4, 5], device="cuda")
    got = answer.next(more)
    want = plain_after(model, [s + [t] for s, t in zip(sequences, more.tolist())])
    assert float((got.double() - want).abs().max()) <= tol * max(1.0, float(want.abs().max()) / 4)
    with pytest.raises(ValueError):
        answer.draft(torch.zeros(3, 60, dtype=torch.long, device="cuda"), torch.full((3, 60), -1, dtype=torch.int32, device="cuda"))


def test_drafted_answers_are_the_greedy_ones():
    """A trained model's answers, some proposals right and some wrong (fp32: its best two logits are further apart than the two
    ways' roundings)."""
    model = D.Decoder(dtype=torch.float32, seed=2)
    for s in range(6):
        D.step(model, D.Batch([60, 33, 90, 17], model.vocab, s), 1000 + s, 16, 1e-3, 2e-3)
    prompts = [[3, 5, 7, 9], [1, 2, 3, 4, 5, 6], [40]]
    want = D.Answer(model, prompts, 12).greedy(12)
    passes = []

    def propose(got):
        passes.append(1)
        trees = D.strides(got, model.vocab)
        if len(passes) % 2:      # the true next two among them
            trees = [([int(x) for x in want[b, len(g):len(g) + 2]] + t, [-1, 0][:len(want[b, len(g):len(g) + 2])] +
                      [u + len(want[b, len(g):len(g) + 2]) if u >= 0 else -1 for u in up]) for b, (g, (t, up)) in enumerate(zip(got, trees))]
        return trees
    got = D.Answer(model, prompts, 60).greedy_drafted(12, propose)
    assert torch.equal(got, want)
    assert len(passes) < 12
    with pytest.raises(ValueError, match="vocabulary"):
        D.Answer(model, prompts, 60).greedy_drafted(4, lambda got: [([model.vocab], [-1])] * 3)


@pytest.mark.parametrize("kind", ["policy", "preference"])
def test_steps_on_answers_are_algorithm_1(kind):
    """The fused schedule's weights and losses on answers, bit for bit those of +eps, -2 eps, +eps per probe and the update;
    at the model that gave the answers a pair's loss is log 2 and a policy's minus its mean advantage."""
    K, eps, lr, seed = 4, 1e-3, 1e-3, 77
    a, b = D.Decoder(dtype=torch.float32, seed=1), D.Decoder(dtype=torch.float32, seed=1)
    batch = D.answered(a, 5, kind)
    table, status = D.step(a, batch, seed, K, eps, lr)
    want = torch.empty(K, 3, dtype=torch.float64, device="cuda")
    batch.loss_into(b, want[0, 2:3])
    want[1:, 2] = want[0, 2]
    for k in range(K):
        zo.perturb(b.params, seed, k, eps)
        batch.loss_into(b, want[k, 0:1])
        zo.perturb(b.params, seed, k, -2 * eps)
        batch.loss_into(b, want[k, 1:2])
        zo.perturb(b.params, seed, k, eps)
    c, _ = zo.precondition(want, eps)
    zo.update(b.params, seed, c, lr)
    assert int(status) == zo.ZO_OK and torch.equal(table, want)
    assert all(torch.equal(x, y) for x, y in zip(a.params.tensors, b.params.tensors))
    assert float((table[:, 0] - table[:, 1]).abs().max()) > 0
    counted = batch.targets >= 0
    here = 0.6931471805599453 if kind == "preference" else -float(batch.advantages[counted].double().mean())
    # the ratios are 1 within the roundings of log-probabilities of at most 2^4: 2^-20 of unit-sized advantages
    assert abs(float(table[0, 2]) - here) <= 1e-5
