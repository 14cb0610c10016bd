"""Losses over answers called from several host threads at once, through the C ABI: nothing of one call's size is shared by another."""
import threading

import pytest
import torch

from paper_2609_38095_gb300 import build as zo_build
from paper_2609_38095_gb300 import forward as F
from paper_2609_38095_gb300 import zo
from test_gpu_answer_losses import check_policy, policy_inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    zo_build.build()


class Call:
    """zo_policy_loss with its gradient of one row, on a stream and in memory of its own."""

    def __init__(self, vocab, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.logits = torch.randn(1, vocab, generator=g, device="cuda")
        self.target = torch.tensor([vocab // 2], dtype=torch.int32, device="cuda")
        self.old = torch.full((1,), -11.0, device="cuda")
        self.advantage = torch.ones(1, device="cuda")
        self.loss = torch.zeros(1, dtype=torch.float64, device="cuda")
        self.grad = torch.zeros(1, vocab, device="cuda")
        self.size = F._lib().zo_policy_loss_workspace_size(1)
        self.work = torch.zeros(self.size, dtype=torch.uint8, device="cuda")
        self.stream = torch.cuda.Stream()
        self.status = []

    def __call__(self):
        vocab = self.logits.shape[1]
        return F._lib().zo_policy_loss(
            self.logits.data_ptr(), vocab, 1, vocab, 0, self.target.data_ptr(), 4, self.old.data_ptr(), self.advantage.data_ptr(),
            None, None, 0.2, 0.2, 0.0, 0, self.loss.data_ptr(), self.grad.data_ptr(), vocab, 1.0, None, self.work.data_ptr(),
            self.size, self.stream.cuda_stream)

    def many(self, start, times):
        start.wait()
        for i in range(times):
            self.status.append(self())
            if i % 16 == 0:              # the queue stays short: a call that waits for it meets no other
                self.stream.synchronize()


def test_host_threads():
    """Rows whose parts take 75 KB of an SM's shared memory each, beside ones whose parts take 18 and 20 KB: none is refused."""
    calls = [Call(151_936, 1), Call(9_000, 2), Call(5_000, 3)]
    want = []
    for c in calls:
        assert c() == zo.ZO_OK
        torch.cuda.synchronize()
        want.append((c.loss.clone(), c.grad.clone()))
        c.loss.zero_(), c.grad.zero_()
    torch.cuda.synchronize()
    start = threading.Barrier(len(calls))
    threads = [threading.Thread(target=c.many, args=(start, 20_000)) for c in calls]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    for c, (loss, grad) in zip(calls, want):
        assert len(c.status) == 20_000 and set(c.status) == {zo.ZO_OK}
        assert torch.equal(c.loss, loss) and torch.equal(c.grad, grad)


@pytest.mark.parametrize("vocab", [409_568, 409_569])
def test_the_largest_rows(vocab):
    """Rows of which a part is all the shared memory that a call may take, and a logit more."""
    check_policy(*policy_inputs(3, 2, vocab, torch.float32), kl=0.1, mean=True)
