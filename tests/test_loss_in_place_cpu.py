"""The cross entropy's gradient in the logits' place, under autograd, with plain 64-bit torch in the kernels' place."""
import pytest
import torch

from paper_2504_18454_b200 import autograd as A
from paper_2504_18454_b200 import block as B

TARGETS = torch.tensor([[1, -1, 5, 0, 2], [3, 3, -1, 4, 0]], dtype=torch.int32)


def _forward(logits, targets):
    lse = torch.logsumexp(logits, -1)
    at = logits.gather(-1, targets.long().clamp_min(0)[..., None])[..., 0]
    return torch.where(targets >= 0, lse - at, 0.0), lse


def _backward(dloss, logits, targets, lse, *, out):
    hot = torch.zeros_like(logits).scatter_(-1, targets.long().clamp_min(0)[..., None], 1.0)
    g = (torch.exp(logits - lse[..., None]) - hot) * torch.where(targets >= 0, dloss, 0.0)[..., None]
    return g if out is None else out.copy_(g)


@pytest.fixture(autouse=True)
def plain(monkeypatch):
    monkeypatch.setattr(B, "cross_entropy_forward", _forward)
    monkeypatch.setattr(B, "cross_entropy_backward", _backward)


def _leaf():
    return torch.randn(2, 5, 6, generator=torch.Generator().manual_seed(8), dtype=torch.float64).requires_grad_()


def test_the_gradient_is_a_tensor_of_its_own_in_the_logits_memory():
    z = _leaf()
    want = torch.autograd.grad(A.cross_entropy(z * 2, TARGETS).sum(), z)[0] / 2
    logits = z * 2
    loss = A.cross_entropy(logits, TARGETS, in_place=True).sum()
    g, = torch.autograd.grad(loss, logits, retain_graph=True)
    assert g.grad_fn is None and not g.requires_grad and g is not logits
    assert g.data_ptr() == logits.data_ptr() and torch.allclose(g, want)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):       # the logits are gone
        torch.autograd.grad(loss, logits)


@pytest.mark.parametrize("own", [True, False])
@pytest.mark.parametrize("view", [lambda p: p.view(2, 5, 6), lambda p: p.view(1, 10, 6)[:, 2:].view(2, 4, 6), lambda p: p.view(2, 5, 6)[:, :, 1:], lambda p: p.view(5, 2, 6).transpose(0, 1)])
def test_a_view_of_a_leaf_is_refused(view, own):
    """The gradient would be written over the parameter, be it a tensor of its own or (as an arena's) a view of a buffer."""
    p = torch.empty(60, dtype=torch.float64) if own else torch.empty(2, 90, dtype=torch.float64)[1, 30:]
    p = p.copy_(_leaf().detach().view(60)).detach().requires_grad_()
    before = p.detach().clone()
    z = view(p)
    with pytest.raises(RuntimeError, match="leaf"):
        A.cross_entropy(z, TARGETS[:, :z.shape[1]].clamp_max(4), in_place=True)
    A.cross_entropy(z, TARGETS[:, :z.shape[1]].clamp_max(4)).sum().backward()
    assert torch.equal(p, before) and p.grad is not None and p.grad.data_ptr() != p.data_ptr()


def test_a_view_of_a_result_is_not():
    z = _leaf()
    want, = torch.autograd.grad(A.cross_entropy(z * 2, TARGETS).sum(), z)
    logits = (z * 2).view(10, 6).view(2, 5, 6)
    got, = torch.autograd.grad(A.cross_entropy(logits, TARGETS, in_place=True).sum(), z)
    assert torch.allclose(got, want)
    bent = z.exp().clamp_max(50.0)                         # one input all the way down to the leaf, but memory of its own
    A.cross_entropy(bent, TARGETS, in_place=True).sum().backward()
    assert z.grad is not None
