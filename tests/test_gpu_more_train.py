"""The linear operator, the layer norm and the cross entropy under autograd, and the trainer's GPT-Neo block."""
import subprocess
import sys

import pytest
import torch

import paper_2504_18454_b200 as P
from paper_2504_18454_b200 import autograd as A
from _block_ref import within
from _more_ref import linear_backward64, loss_backward64, norm_backward64

pytestmark = pytest.mark.gpu


def _leaf(*shape, std=1.0, dt=torch.float32, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(*shape, generator=gen, device="cuda") * std).to(dt).requires_grad_()


@pytest.mark.parametrize("checkpoint8", [False, True])
@pytest.mark.parametrize("kind", [P.ACT_NONE, P.ACT_GELU])
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
def test_linear_gradients(checkpoint8, kind, dt):
    K, M, D, N = 2, 37, 40, 72
    x, w, b, r = _leaf(K, M, D, dt=dt, seed=1), _leaf(K, N, D, std=D ** -0.5, dt=dt, seed=2), _leaf(K, N, dt=dt, seed=3), _leaf(K, M, N, dt=dt, seed=4)
    dy = _leaf(K, M, N, std=0.01, dt=dt, seed=9).detach()
    A.linear(x, w, b, r, activation=kind, checkpoint8=checkpoint8).backward(dy)
    xs, z = x.detach(), None
    if kind != P.ACT_NONE:                                 # the gradient is taken at what was kept
        _, z = P.linear_forward(xs, w.detach(), b.detach(), activation=kind, save=P.SAVE_8BIT if checkpoint8 else P.SAVE_FULL)
    if checkpoint8:
        xs, z = (None if t is None else P.act8_unpack(t, dtype=torch.float32) for t in (P.act8_pack(xs), z))
    want = linear_backward64(dy, xs, w.detach(), z, kind, dt == torch.bfloat16)
    for t, name in ((x, "dx"), (w, "dw"), (b, "db")):
        within(t.grad, *want[name], name)
    assert torch.equal(r.grad, dy)


@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
def test_layer_norm_gradients(dt):
    K, M, D = 2, 41, 72
    x, r, w, b = _leaf(K, M, D, dt=dt, seed=1), _leaf(K, M, D, dt=dt, seed=2), _leaf(K, D, dt=dt, seed=3), _leaf(K, D, dt=dt, seed=4)
    dy, dt_ = (_leaf(K, M, D, std=0.1, dt=dt, seed=s).detach() for s in (5, 6))
    y, total = A.layer_norm(x, w, b, r)
    torch.autograd.backward((y, total), (dy, dt_))
    _, t, mean, rstd = P.layer_norm_forward(x.detach(), w.detach(), b.detach(), r.detach())
    want = norm_backward64(dy, t, w.detach(), mean, rstd, dt_, dt == torch.bfloat16)
    for g, name in ((x.grad, "dx"), (r.grad, "dx"), (w.grad, "dw"), (b.grad, "db")):
        within(g, *want[name], name)


@pytest.mark.parametrize("in_place", [False, True])
def test_cross_entropy_gradients_of_an_expanded_mean(in_place):
    z = _leaf(2, 30, 100, seed=1)
    t = torch.randint(-1, 100, (2, 30), device="cuda", dtype=torch.int32)
    logits = z * 1.0
    A.cross_entropy(logits, t, in_place=in_place).mean(-1).sum().backward()
    _, lse = P.cross_entropy_forward(z.detach(), t)
    within(z.grad, *loss_backward64(torch.full((2, 30), 1 / 30, device="cuda"), z.detach(), t, lse, False), "dlogits")


def test_gradients_of_broadcast_inputs():
    """One weight, bias and input of all workers: their gradients are sums over the workers (by autograd, behind the operator)."""
    K, M, D, N = 3, 20, 24, 40
    x, w, b, r = _leaf(1, M, D, seed=1), _leaf(1, N, D, seed=2), _leaf(1, N, seed=3), _leaf(1, 1, N, seed=4)
    dy = _leaf(K, M, N, seed=5).detach()
    A.linear(x.expand(K, M, D), w.expand(K, N, D), b.expand(K, N), r.expand(K, M, N)).backward(dy)
    want = linear_backward64(dy, x.detach().expand(K, M, D), w.detach().expand(K, N, D), None, P.ACT_NONE, False)
    # K more roundings of each sum's terms, in binary32
    for t, name in ((x, "dx"), (w, "dw"), (b, "db")):
        v, e = want[name]
        within(t.grad, v.sum(0, keepdim=True), e.sum(0, keepdim=True) + K * 2.0 ** -23 * v.abs().sum(0, keepdim=True), name)
    assert torch.allclose(r.grad, dy.sum((0, 1), keepdim=True), rtol=1e-5, atol=1e-4)


def _plain_loss(w, p, tokens):
    """The trainer's GPT-Neo model in elementary torch, 64 bits."""
    K, B, S = tokens.shape[0], tokens.shape[1], tokens.shape[2] - 1
    H, norm = w.width // 64, lambda x, n: (x - x.mean(-1, keepdim=True)) / torch.sqrt(x.var(-1, correction=0, keepdim=True) + 1e-5) * p[n + ".w"][:, None] + p[n + ".b"][:, None]
    lin = lambda x, n: x @ p[n + ".w"].mT + p[n + ".b"][:, None]
    ids = tokens[:, :, :-1].reshape(K, B * S)
    x = torch.stack([p["embed"][k][ids[k]] for k in range(K)]) + p["wpe"][:, :S].repeat(1, B, 1)
    for i in range(w.layers):
        q, k, v = (t.unflatten(1, (B, S)).unflatten(3, (H, 64)).transpose(2, 3) for t in lin(norm(x, f"{i}.ln1"), f"{i}.qkv").split(w.width, 2))
        a = torch.softmax(q @ k.mT / 8 + w.mask[:S, :S].double(), -1) @ v
        x = x + lin(a.transpose(2, 3).reshape(K, B * S, w.width), f"{i}.proj")
        z = lin(norm(x, f"{i}.ln2"), f"{i}.fc")
        x = x + lin(z * torch.sigmoid(1.5957691216057308 * (z + 0.044715 * z ** 3)), f"{i}.fc2")
    logits = norm(x, "ln_f") @ p["head"].mT
    at = logits.gather(-1, tokens[:, :, 1:].reshape(K, B * S, 1))[..., 0]
    return (torch.logsumexp(logits, -1) - at).mean(-1)


def test_the_trainers_neo_model_has_the_gradients_of_its_formula():
    """fp32: a result of each of the 12 operators of a layer is within 64 roundings (2^-18) of its norm; through two layers and
    back, 48 of them in a chain, that is 2^-12 of a gradient's norm."""
    from paper_2504_18454_b200.train import Workers, batch
    w = Workers(2, 64, 128, 192, 2, 32, precision=P.PREC_FP32, checkpoint8=False, neo=True)
    tokens = batch(2, 3, 32, 64, torch.Generator(device="cuda").manual_seed(3))
    losses = w.gradients(tokens)
    p = {n: w.arena.worker_tensor("param", j, *s).double().requires_grad_() for j, (n, s) in enumerate(w.shapes)}
    want = _plain_loss(w, p, tokens)
    want.sum().backward()
    assert torch.allclose(losses.double(), want, rtol=2.0 ** -14)
    for j, (n, s) in enumerate(w.shapes):
        g, r = w.arena.worker_tensor("grad", j, *s).double(), p[n].grad
        assert float((g - r).norm()) <= 2.0 ** -12 * float(r.norm()) + 1e-9, n


@pytest.mark.parametrize("precision,checkpoint8", [(P.PREC_BF16_MASTER, True), (P.PREC_BF16_MASTER, False), (P.PREC_FP32, True)])
def test_workers_train_the_neo_model(precision, checkpoint8):
    from paper_2504_18454_b200.train import run
    loss = run(K=3, steps=12, layers=2, width=128, hidden=192, precision=precision, checkpoint8=checkpoint8, neo=True)
    P.block_status()
    assert len(loss) == 12 and all(0.0 < v < 10.0 for v in loss)


def test_the_command_runs_the_neo_model():
    r = subprocess.run([sys.executable, "-m", "paper_2504_18454_b200.train", "--block", "neo", "--workers", "2", "--steps", "3", "--width", "64", "--layers", "1"],
                       capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "step    2" in r.stdout, r.stderr[-2000:]


def test_a_captured_step_of_the_autograd_functions():
    """Forward and backward in one captured graph, warmed up on a side stream as torch asks for, replayed with new inputs."""
    K, M, D, N = 2, 130, 64, 96
    x, w, b, lw, lb = _leaf(K, M, D, seed=1), _leaf(K, N, D, std=0.1, seed=2), _leaf(K, N, seed=3), _leaf(K, D, seed=4), _leaf(K, D, seed=5)
    t = torch.randint(0, N, (K, M), device="cuda", dtype=torch.int32)
    leaves = (x, w, b, lw, lb)

    def step():
        loss = A.cross_entropy(A.linear(A.layer_norm(x, lw, lb), w, b, activation=P.ACT_SILU), t).mean()
        return (loss.detach(), *torch.autograd.grad(loss, leaves))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    with torch.no_grad():
        for leaf in leaves:
            leaf.mul_(0.9)
    graph.replay()
    want = step()
    assert all(torch.equal(a, c) for a, c in zip(got, want))
