"""How the normalisation and the head's loss are called: under function transforms, and in whole steps from several threads at once."""
import threading

import pytest

torch = pytest.importorskip("torch")

from paper_2510_20271_amd.loss import linear_cross_entropy
from paper_2510_20271_amd.norm import group_norm_act

pytestmark = pytest.mark.gpu


def _rand(*shape, seed=0):
    return torch.randn(*shape, device="cuda", generator=torch.Generator("cuda").manual_seed(seed))


def test_function_transforms_are_refused():
    """As for the soft layer: an error, not a result without its transform."""
    x, W = _rand(4, 8), _rand(5, 8, seed=1)
    labels = torch.arange(4, device="cuda")
    for call in (lambda t: group_norm_act(t, 2).sum(), lambda t: linear_cross_entropy(t, W, labels)):
        with pytest.raises(RuntimeError):
            torch.func.grad(call)(x)
        with pytest.raises(RuntimeError):
            torch.func.vmap(call)(x[None])


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
def test_steps_of_several_threads(dtype):
    """Forward and backward on streams of their own: each thread's gradients are those of a step alone."""
    x, W = _rand(20, 300, 16, seed=2).to(dtype), _rand(2000, 16, seed=3).to(dtype)
    labels = torch.arange(20 * 300, device="cuda").view(20, 300) % 2000
    labels[3] = -100

    def step(k):
        a = (x + k).to(dtype).requires_grad_(True)
        c = W.clone().requires_grad_(True)
        loss = linear_cross_entropy(group_norm_act(a * a, 4), c, labels, reduction="none")
        return (loss.detach(), *torch.autograd.grad(loss.sum(), (a, c)))
    want = [step(k) for k in range(3)]
    torch.cuda.synchronize()
    failed = []

    def work(k):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(8):
                    got = step(k)
                    torch.cuda.current_stream().synchronize()
                    assert all(torch.equal(a, c) for a, c in zip(got, want[k]))
        except BaseException as e:  # (handed to the test's own thread)
            failed.append(e)
    threads = [threading.Thread(target=work, args=(k,)) for k in range(3)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed, failed
