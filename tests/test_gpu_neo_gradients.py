"""The gradients of the trainer's GPT-Neo model as it trains by default: bfloat16, activations in 8 bits, the loss in place."""
import pytest
import torch

import paper_2504_18454_b200 as P
from test_gpu_more_train import _plain_loss

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("precision,checkpoint8", [(P.PREC_BF16_MASTER, True), (P.PREC_BF16_MASTER, False), (P.PREC_FP32, True)])
def test_the_default_models_gradients_are_those_of_its_formula(precision, checkpoint8):
    """Every tensor's gradient within a quarter of its norm of the 64-bit model's at the same weights.  The twelve results of a layer are each
    off by at most 2^-8 of themselves (one rounding to bfloat16); through two layers and back, 48 of them in a chain, that is 0.19 of
    a gradient's norm.  A checkpoint is off by half a step, 2^-7 of its group's largest value at most, 0.01 of the norm of 32 values of a normal
    distribution, and each gradient has up to five of them in its way: 0.05.  A gradient that is left out, has the wrong sign or is
    twice or half as large is off by half its norm or more."""
    from paper_2504_18454_b200.train import Workers, batch
    w = Workers(2, 64, 128, 192, 2, 32, precision=precision, checkpoint8=checkpoint8, neo=True, seed=3)
    ctx = w.arena.make_context(stream=torch.cuda.current_stream().cuda_stream, H=16, p=0.1, seed=1)      # (it rounds the masters to the weights)
    tokens = batch(2, 8, 32, 64, torch.Generator(device="cuda").manual_seed(4))
    losses = w.gradients(tokens)
    P.block_status()
    p = {n: w.arena.worker_tensor("param", j, *s).double().requires_grad_() for j, (n, s) in enumerate(w.shapes)}
    want = _plain_loss(w, p, tokens)
    want.sum().backward()
    assert torch.allclose(losses.double(), want, rtol=2.0 ** -5)
    for j, (n, s) in enumerate(w.shapes):
        g, r = w.arena.worker_tensor("grad", j, *s).double(), p[n].grad
        for k in range(2):
            off, size = float((g[k] - r[k]).norm()), float(r[k].norm())
            assert size > 0 and off <= 0.25 * size, (n, k, off, size)
    del ctx
