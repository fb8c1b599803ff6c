"""What the autograd functions of the linear operator, the layer norm and the cross entropy do around the kernels, with plain 64-bit
torch in the kernels' place."""
import pytest
import torch

from paper_2504_18454_b200 import autograd as A
from paper_2504_18454_b200 import block as B


def _linear_forward(x, w, bias, residual, *, activation, save):
    z = x @ w.mT + (0 if bias is None else bias[:, None])
    y = (z.clamp_min(0) if activation == B.ACT_RELU else z) + (0 if residual is None else residual)
    return y, None if save == B.SAVE_NONE else z


def _linear_backward(dy, x, w, saved, *, activation, need_dx, need_dbias):
    assert (saved is None) == (activation == B.ACT_NONE)
    dz = dy if saved is None else dy * (saved > 0)
    return dz @ w if need_dx else None, dz.mT @ x, dz.sum(1) if need_dbias else None


def _norm_forward(x, w, b, residual, *, eps, stats):
    h = x if residual is None else x + residual
    mean = h.mean(-1)
    rstd = 1 / torch.sqrt(h.var(-1, correction=0) + eps)
    return (h - mean[..., None]) * rstd[..., None] * w[:, None] + b[:, None], h, mean if stats else None, rstd if stats else None


def _norm_backward(dy, x, w, mean, rstd, dtotal):
    xh = (x - mean[..., None]) * rstd[..., None]
    g = dy * w[:, None]
    dx = rstd[..., None] * (g - g.mean(-1, keepdim=True) - xh * (g * xh).mean(-1, keepdim=True))
    return dx if dtotal is None else dx + dtotal, (dy * xh).sum(1), dy.sum(1)


def _loss_forward(logits, targets):
    lse = torch.logsumexp(logits, -1)
    at = logits.gather(-1, targets.long().clamp_min(0)[..., None])[..., 0]
    return torch.where(targets >= 0, lse - at, 0.0), lse


def _loss_backward(dloss, logits, targets, lse, *, out):
    hot = torch.zeros_like(logits).scatter_(-1, targets.long().clamp_min(0)[..., None], 1.0)
    g = (torch.exp(logits - lse[..., None]) - hot) * torch.where(targets >= 0, dloss, 0.0)[..., None]
    return g if out is None else out.copy_(g)


@pytest.fixture
def plain(monkeypatch):
    for name, f in (("linear_forward", _linear_forward), ("linear_backward", _linear_backward), ("layer_norm_forward", _norm_forward),
                    ("layer_norm_backward", _norm_backward), ("cross_entropy_forward", _loss_forward), ("cross_entropy_backward", _loss_backward)):
        monkeypatch.setattr(B, name, f)


def _leaf(*shape, seed):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64).requires_grad_()


def _args():
    return _leaf(2, 5, 4, seed=1), _leaf(2, 6, 4, seed=2), _leaf(2, 6, seed=3), _leaf(2, 5, 6, seed=4)


TARGETS = torch.tensor([[1, -1, 5, 0, 2], [3, 3, -1, 4, 0]], dtype=torch.int32)


def test_gradients_agree_with_differences(plain):
    x, w, b, r = _args()
    for act in (B.ACT_NONE, B.ACT_RELU):
        assert torch.autograd.gradcheck(lambda *a: A.linear(*a, activation=act), (x, w, b, r))
    assert torch.autograd.gradcheck(lambda x, w: A.linear(x, w), (x, w))
    g, c = _leaf(2, 6, seed=5), _leaf(2, 6, seed=6)
    z = _leaf(2, 5, 6, seed=7)
    assert torch.autograd.gradcheck(lambda *a: A.layer_norm(*a), (z, g, c))
    assert torch.autograd.gradcheck(lambda *a: A.layer_norm(*a), (z, g, c, r))
    assert torch.autograd.gradcheck(lambda *a: A.layer_norm(*a)[0], (z, g, c, r))
    assert torch.autograd.gradcheck(lambda *a: A.layer_norm(*a)[1], (z, g, c, r))
    assert torch.autograd.gradcheck(lambda z: A.cross_entropy(z, TARGETS), (z,))


@pytest.mark.parametrize("need", range(1, 16))
def test_only_what_needs_a_gradient_gets_one(plain, need):
    args = [t.detach().requires_grad_(bool(need >> i & 1)) for i, t in enumerate(_args())]
    A.linear(*args, activation=B.ACT_RELU).sum().backward()
    ref = [t.detach().requires_grad_() for t in args]
    (_linear_forward(*ref, activation=B.ACT_RELU, save=B.SAVE_NONE)[0]).sum().backward()
    for i, (a, b) in enumerate(zip(args, ref)):
        assert (a.grad is not None) == bool(need >> i & 1)
        if a.grad is not None:
            assert torch.allclose(a.grad, b.grad, rtol=1e-12)


def test_a_second_derivative_raises(plain):
    x, w, b, r = _args()
    for f in (lambda: A.linear(x, w, b, r).sum(), lambda: A.layer_norm(r, b, b)[0].sum(), lambda: A.cross_entropy(r, TARGETS).sum()):
        with pytest.raises(RuntimeError, match="once"):
            torch.autograd.grad(f() + r.square().sum(), r, create_graph=True)


def test_nothing_is_kept_where_gradients_are_off(plain, monkeypatch):
    calls = []
    monkeypatch.setattr(B, "linear_forward", lambda *a, save, **k: calls.append(save) or _linear_forward(*a, save=save, **k))
    monkeypatch.setattr(B, "layer_norm_forward", lambda *a, stats, **k: calls.append(stats) or _norm_forward(*a, stats=stats, **k))
    monkeypatch.setattr(B, "act8_pack", lambda x: pytest.fail("a checkpoint that nothing will read"))
    x, w, b, r = _args()
    with torch.no_grad():
        A.linear(x, w, b, r, activation=B.ACT_RELU, checkpoint8=True), A.layer_norm(r, b, b)
    A.linear(*(t.detach() for t in (x, w, b)), r, activation=B.ACT_RELU)          # the residual's gradient needs nothing
    assert calls == [B.SAVE_NONE, False, B.SAVE_NONE]


def test_in_place_the_gradient_takes_the_logits_memory(plain):
    z = _leaf(2, 5, 6, seed=8)
    want = torch.autograd.grad(A.cross_entropy(z * 2, TARGETS).sum(), z)[0]
    logits = z * 2
    loss = A.cross_entropy(logits, TARGETS, in_place=True).sum()
    assert torch.allclose(torch.autograd.grad(loss, z, retain_graph=True)[0], want)
    assert not torch.equal(logits, z * 2)
    with pytest.raises(RuntimeError, match="leaf"):
        A.cross_entropy(z, TARGETS, in_place=True)


def test_the_model_of_the_trainer_has_the_tensors_of_the_gptneo_lists():
    """The same names and shapes as `workloads` lists for the 8M shape (matrices transposed), but for the positions and the head."""
    import workloads as W
    from paper_2504_18454_b200.train import neo_shapes
    want = {s.name: tuple(s.shape) for s in W.gptneo_8m_shape()}
    got = dict(neo_shapes(8192, 256, 1024, 8, 128))
    for name, shape in want.items():
        mine = name[1:] if name.startswith("h") else name
        mine = "embed" if mine == "wte" else mine
        assert got[mine] == (shape if mine == "embed" or len(shape) == 1 else shape[::-1]), name
