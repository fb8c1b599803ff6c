"""The cross entropy's gradient in the logits' place, under autograd."""
import pytest
import torch

from paper_2504_18454_b200 import autograd as A

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
def test_the_gradient_is_a_tensor_of_its_own_in_the_logits_memory(dt):
    z = torch.randn(2, 30, 101, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda").to(dt).requires_grad_()
    t = torch.randint(-1, 101, (2, 30), device="cuda", dtype=torch.int32)
    want, = torch.autograd.grad(A.cross_entropy(z, t).sum(), z)
    logits = z * 1.0
    loss = A.cross_entropy(logits, t, in_place=True).sum()
    g, = torch.autograd.grad(loss, logits, retain_graph=True)
    assert g.grad_fn is None and not g.requires_grad
    assert g.data_ptr() == logits.data_ptr() and torch.equal(g, want)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):       # the logits are gone
        torch.autograd.grad(loss, logits)
