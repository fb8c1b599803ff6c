"""The block operators under autograd, and the whole path: K workers train a small language model with them."""
import math

import pytest
import torch

import paper_2504_18454_b200 as P
from paper_2504_18454_b200 import autograd as A
from _block_ref import ffn_backward64, qk_backward64, within

pytestmark = pytest.mark.gpu


def _leaf(*shape, std=1.0, dt=torch.float32, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(*shape, generator=gen, device="cuda") * std).to(dt).requires_grad_()


@pytest.mark.parametrize("checkpoint8", [False, True])
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
def test_gated_ffn_gradients(checkpoint8, dt):
    K, M, D, F = 2, 37, 40, 72
    x, wg, wu, wd = (_leaf(*s, std=v, dt=dt, seed=i) for i, (s, v) in enumerate(
        [((K, M, D), 1.0), ((K, F, D), D ** -0.5), ((K, F, D), D ** -0.5), ((K, D, F), F ** -0.5)]))
    dy = _leaf(K, M, D, std=0.01, dt=dt, seed=9).detach()
    y = A.gated_ffn(x, wg, wu, wd, activation=P.ACT_GELU, checkpoint8=checkpoint8)
    y.backward(dy)
    # the gradient is taken at what was kept
    _, (g, u) = P.ffn_forward(x.detach(), wg.detach(), wu.detach(), wd.detach(), activation=P.ACT_GELU,
                              save=P.SAVE_8BIT if checkpoint8 else P.SAVE_FULL)
    xs = x.detach()
    if checkpoint8:
        g, u, xs = (P.act8_unpack(t, dtype=torch.float32) for t in (g, u, P.act8_pack(xs)))
    want = ffn_backward64(dy, xs, wg.detach(), wu.detach(), wd.detach(), g, u, P.ACT_GELU, dt == torch.bfloat16)
    for t, name in zip((x, wg, wu, wd), ("dx", "dw_gate", "dw_up", "dw_down")):
        within(t.grad, *want[name], name)


def test_gated_ffn_without_gradients_keeps_nothing():
    x, wg, wu, wd = (_leaf(*s).detach() for s in [(1, 5, 16), (1, 24, 16), (1, 24, 16), (1, 16, 24)])
    assert A.gated_ffn(x, wg, wu, wd).grad_fn is None


def test_qk_norm_rope_gradients():
    K, M, HQ, HK, DH = 2, 19, 4, 2, 32
    q, k = _leaf(K, M, HQ, DH, seed=1), _leaf(K, M, HK, DH, seed=2)
    wq, wk = _leaf(K, DH, seed=3), _leaf(K, DH, seed=4)
    ang = torch.rand(M, DH // 2, device="cuda", dtype=torch.float64) * 6
    cos, sin = ang.cos().float(), ang.sin().float()
    pos = torch.arange(M, device="cuda", dtype=torch.int32)[None].expand(K, M)
    oq, ok = A.qk_norm_rope(q, k, wq, wk, cos, sin, pos, eps=1e-5)
    gq, gk = _leaf(K, M, HQ, DH, seed=5).detach(), _leaf(K, M, HK, DH, seed=6).detach()
    ((oq * gq).sum() + (ok * gk).sum()).backward()
    for x, w, g in ((q, wq, gq), (k, wk, gk)):
        dx, dw = qk_backward64(g, x.detach(), w.detach(), pos, cos, sin, 1e-5, False, False)
        within(x.grad, *dx, "dx")
        within(w.grad, *dw, "dw")


@pytest.mark.parametrize("precision,checkpoint8", [(P.PREC_BF16_MASTER, True), (P.PREC_FP32, False)])
def test_workers_learn_the_rule(precision, checkpoint8):
    """Uniform guessing costs ln 64; the rule can be read off any two tokens, so what cannot be learnt is one guess out of
    four at the first token of a sequence of 64: ln 4 / 64 = 0.02.  A sixth of the first loss is far from both."""
    from paper_2504_18454_b200.train import run
    loss = run(K=3, steps=80, layers=2, width=128, hidden=192, precision=precision, checkpoint8=checkpoint8)
    P.block_status()
    assert abs(loss[0] - math.log(64)) < 1.0
    assert sum(loss[-5:]) / 5 < loss[0] / 6
