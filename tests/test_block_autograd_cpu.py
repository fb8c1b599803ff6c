"""What the block operators' autograd functions do around the kernels, with plain 64-bit torch in the kernels' place."""
import pytest
import torch

from paper_2504_18454_b200 import autograd as A
from paper_2504_18454_b200 import block as B


def _ffn_backward(dy, x, w_gate, w_up, w_down, saved, *, activation, need_dx):
    g, u = saved
    a, slope = g.clamp_min(0), (g > 0).to(g.dtype)       # the tests use ReLU
    dh = dy @ w_down
    dg, du = dh * u * slope, dh * a
    return (dg @ w_gate + du @ w_up if need_dx else None), dg.mT @ x, du.mT @ x, dy.mT @ (a * u)


def _ffn_forward(x, w_gate, w_up, w_down, *, activation, save):
    g, u = x @ w_gate.mT, x @ w_up.mT
    return (g.clamp_min(0) * u) @ w_down.mT, None if save == B.SAVE_NONE else (g, u)


def _qk(q, k, w_q, w_k, cos, sin, positions, *, eps, interleaved):
    return q * w_q[:, None, None], k * w_k[:, None, None]


def _qk_backward(dq, dk, q, k, w_q, w_k, cos, sin, positions, *, eps, interleaved):
    return dq * w_q[:, None, None], dk * w_k[:, None, None], (dq * q).sum((1, 2)), (dk * k).sum((1, 2))


@pytest.fixture
def plain(monkeypatch):
    monkeypatch.setattr(B, "ffn_forward", _ffn_forward)
    monkeypatch.setattr(B, "ffn_backward", _ffn_backward)
    monkeypatch.setattr(B, "qk_norm_rope", _qk)
    monkeypatch.setattr(B, "qk_norm_rope_backward", _qk_backward)


def _leaf(*shape, seed):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64).requires_grad_()


def _ffn_args():
    return _leaf(1, 5, 4, seed=1), _leaf(1, 6, 4, seed=2), _leaf(1, 6, 4, seed=3), _leaf(1, 4, 6, seed=4)


def _qk_args():
    return _leaf(1, 3, 2, 4, seed=1), _leaf(1, 3, 1, 4, seed=2), _leaf(1, 4, seed=3), _leaf(1, 4, seed=4)


@pytest.mark.parametrize("reduce", [lambda y: y.sum(), lambda y: y.square().sum()], ids=["linear", "square"])
def test_a_second_derivative_raises(plain, reduce):
    """Their gradients carry no graph: a second derivative would lack their part without a word, also where the incoming
    gradient needs none itself (a sum) and where only one input's is asked for."""
    x, *w = _ffn_args()
    with pytest.raises(RuntimeError, match="once"):
        torch.autograd.grad(reduce(A.gated_ffn(x, *w, activation=B.ACT_RELU)) + x.square().sum(), x, create_graph=True)
    q, k, wq, wk = _qk_args()
    with pytest.raises(RuntimeError, match="once"):
        torch.autograd.grad(sum(map(reduce, A.qk_norm_rope(q, k, wq, wk, None, None, None))) + q.square().sum(), q, create_graph=True)


def test_first_derivatives_do_not(plain):
    x, *w = _ffn_args()
    got = torch.autograd.grad(A.gated_ffn(x, *w, activation=B.ACT_RELU).square().sum(), (x, *w))
    want = torch.autograd.grad(_ffn_forward(x, *w, activation=B.ACT_RELU, save=B.SAVE_NONE)[0].square().sum(), (x, *w))
    for a, b in zip(got, want):
        assert torch.allclose(a, b, rtol=1e-12)
    args = _qk_args()
    got = torch.autograd.grad(sum(t.square().sum() for t in A.qk_norm_rope(*args, None, None, None)), args)
    want = torch.autograd.grad(sum(t.square().sum() for t in _qk(*args, None, None, None, eps=0, interleaved=0)), args)
    for a, b in zip(got, want):
        assert torch.allclose(a, b, rtol=1e-12)


@pytest.mark.parametrize("checkpoint8", [False, True])
def test_nothing_is_kept_where_gradients_are_off(plain, monkeypatch, checkpoint8):
    """Evaluation of a model whose parameters want gradients, under no_grad."""
    saves = []

    def forward(*a, save, **k):
        saves.append(save)
        return _ffn_forward(*a, save=save, **k)

    def pack(x, **k):
        raise AssertionError("a checkpoint that nothing will read")

    monkeypatch.setattr(B, "ffn_forward", forward)
    monkeypatch.setattr(B, "act8_pack", pack)
    with torch.no_grad():
        A.gated_ffn(*_ffn_args(), activation=B.ACT_RELU, checkpoint8=checkpoint8)
    A.gated_ffn(*(t.detach() for t in _ffn_args()), activation=B.ACT_RELU, checkpoint8=checkpoint8)
    assert saves == [B.SAVE_NONE, B.SAVE_NONE]
    A.gated_ffn(*_ffn_args(), activation=B.ACT_RELU)
    assert saves[2:] == [B.SAVE_FULL]
