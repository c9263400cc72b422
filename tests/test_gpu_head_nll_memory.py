"""What the scalar of losses.head_nll holds on to."""
import pytest
import torch

from tests.test_gpu_head_grads import DEV, weights
from tests.test_gpu_head_logprobs import make

pytestmark = pytest.mark.gpu


def test_gradients_are_released_by_the_backward_pass():
    from paper_2602_01274_b200 import losses
    h, w, tok, _ = make(300, 20011, 512)
    weight = weights(300)[0]
    h, w = h.requires_grad_(True), w.requires_grad_(True)
    both = (h.numel() + w.numel()) * 2
    losses.head_nll(h, w, tok, weight).backward()                           # (what the library and torch set up once)
    want = h.grad.clone(), w.grad.clone()
    h.grad = w.grad = None
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    total = losses.head_nll(h, w, tok, weight)
    total.backward()
    assert torch.cuda.memory_allocated() - before < 1.05 * both and total.grad_fn is not None
    assert torch.equal(h.grad, want[0]) and torch.equal(w.grad, want[1])
    with pytest.raises(RuntimeError, match="second time"):
        total.backward()
    # kept where it is asked for
    h.grad = w.grad = None
    total = losses.head_nll(h, w, tok, weight)
    total.backward(retain_graph=True)
    total.backward()
    assert torch.equal(h.grad, 2 * want[0]) and torch.equal(w.grad, 2 * want[1])
