"""The linear operator, the layer norm and the cross entropy at the edges: streams, graphs, workspaces, threads, offsets beyond 32
bits, very large values, refusals."""
import threading

import pytest
import torch

import paper_2504_18454_b200 as P
from _block_ref import within
from _more_ref import linear64, linear_backward64, loss64, loss_backward64, norm64, norm_backward64

pytestmark = pytest.mark.gpu
DT = {"fp32": torch.float32, "bf16": torch.bfloat16}


def _randn(*shape, seed, dt=torch.bfloat16, std=1.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(*shape, generator=gen, device="cuda") * std).to(dt)


def _chain(dt=torch.bfloat16, M=300, seed=1):
    """Inputs, and a function of them that runs every operator forward and backward, as a block would."""
    K, D, N, V = 2, 264, 200, 1031
    r = lambda *s, std=1.0, i=0: _randn(*s, seed=seed * 100 + i, dt=dt, std=std)
    t = dict(x=r(K, M, D), res=r(K, M, D, i=1), lw=r(K, D, i=2), lb=r(K, D, i=3), w1=r(K, N, D, std=D ** -0.5, i=4), b1=r(K, N, i=5),
             w2=r(K, D, N, std=N ** -0.5, i=6), b2=r(K, D, i=7), head=r(K, V, D, std=D ** -0.5, i=8))
    targets = torch.arange(K * M, device="cuda", dtype=torch.int32).view(K, M) % V
    dloss = torch.full((K, M), 1.0 / M, device="cuda")

    def run(**ws):
        n, total, mean, rstd = P.layer_norm_forward(t["x"], t["lw"], t["lb"], t["res"])
        h, z = P.linear_forward(n, t["w1"], t["b1"], activation=P.ACT_GELU, save=P.SAVE_8BIT, **ws)
        y, _ = P.linear_forward(h, t["w2"], t["b2"], total, **ws)
        logits, _ = P.linear_forward(y, t["head"], **ws)
        loss, lse = P.cross_entropy_forward(logits, targets)
        dz = P.cross_entropy_backward(dloss, logits, targets, lse, out=logits)
        dy, dhead, _ = P.linear_backward(dz, y, t["head"], need_dbias=False, **ws)
        dh, dw2, db2 = P.linear_backward(dy, h, t["w2"], **ws)
        dn, dw1, db1 = P.linear_backward(dh, n, t["w1"], z, activation=P.ACT_GELU, **ws)
        dx, dlw, dlb = P.layer_norm_backward(dn, total, t["lw"], mean, rstd, dy, **ws)
        return loss, dhead, dw2, db2, dw1, db1, dx, dlw, dlb

    return t, run


def _same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("M", [3, 300])
def test_a_run_of_them_against_the_statements(dtype, M):
    """The whole chain once, every step compared at the values that it was given."""
    bf, (t, _) = dtype == "bf16", _chain(DT[dtype], M)
    K, D = t["lw"].shape
    V = t["head"].shape[1]
    targets = torch.arange(K * M, device="cuda", dtype=torch.int32).view(K, M) % V
    n, total, mean, rstd = P.layer_norm_forward(t["x"], t["lw"], t["lb"], t["res"])
    within(n, *norm64(t["x"], t["res"], t["lw"], t["lb"], 1e-5, bf)["y"], "norm")
    h, z = P.linear_forward(n, t["w1"], t["b1"], activation=P.ACT_GELU, save=P.SAVE_FULL)
    within(h, *linear64(n, t["w1"], t["b1"], None, P.ACT_GELU, bf)["y"], "h")
    y, _ = P.linear_forward(h, t["w2"], t["b2"], total)
    within(y, *linear64(h, t["w2"], t["b2"], total, P.ACT_NONE, bf)["y"], "y")
    logits, _ = P.linear_forward(y, t["head"])
    loss, lse = P.cross_entropy_forward(logits, targets)
    within(loss, *loss64(logits, targets)[0], "loss")
    d = torch.full((K, M), 1.0 / M, device="cuda")
    want = loss_backward64(d, logits, targets, lse, bf)
    dz = P.cross_entropy_backward(d, logits, targets, lse, out=logits)
    within(dz, *want, "dlogits")
    dy, dhead, none = P.linear_backward(dz, y, t["head"], need_dbias=False)
    ref = linear_backward64(dz, y, t["head"], None, P.ACT_NONE, bf)
    within(dy, *ref["dx"], "dy")
    within(dhead, *ref["dw"], "dhead")
    dn, dw, db = P.linear_backward(_randn(*h.shape, seed=77, dt=DT[dtype]), n, t["w1"], z, activation=P.ACT_GELU)
    ref = linear_backward64(_randn(*h.shape, seed=77, dt=DT[dtype]), n, t["w1"], z, P.ACT_GELU, bf)
    for a, name in ((dn, "dx"), (dw, "dw"), (db, "db")):
        within(a, *ref[name], name)
    ref = norm_backward64(dn, total, t["lw"], mean, rstd, dy, bf)
    for a, name in zip(P.layer_norm_backward(dn, total, t["lw"], mean, rstd, dy), ("dx", "dw", "db")):
        within(a, *ref[name], name)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("M", [5, 300])
def test_captured_calls_replay_with_new_inputs(dtype, M):
    t, run = _chain(DT[dtype], M, seed=2)
    other, run_other = _chain(DT[dtype], M, seed=3)
    want, want_other = run(), run_other()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run()
    graph.replay()
    assert _same(got, want)
    for n in t:
        t[n].copy_(other[n])
    for _ in range(2):
        graph.replay()
        assert _same(got, want_other)


def test_two_captured_graphs_side_by_side():
    """Each has workspaces of its own: replayed on two streams at the same time they do not disturb one another."""
    _, a = _chain(M=700, seed=4)
    _, b = _chain(M=650, seed=5)
    want = a(), b()
    graphs, got = [torch.cuda.CUDAGraph() for _ in range(2)], []
    for g, f in zip(graphs, (a, b)):
        with torch.cuda.graph(g):
            got.append(f())
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    assert all(_same(x, y) for x, y in zip(got, want))


def test_another_stream_and_a_given_workspace():
    t, run = _chain(seed=6)
    want = run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = run()
    side.synchronize()
    assert _same(got, want)
    ws = torch.empty(64 << 20, device="cuda", dtype=torch.uint8)
    assert _same(run(workspace=ws), want)
    raw = side.cuda_stream
    side.wait_stream(torch.cuda.current_stream())
    y0, _ = P.linear_forward(t["x"], t["w1"], t["b1"])
    y1, _ = P.linear_forward(t["x"], t["w1"], t["b1"], stream=raw)
    n1 = P.layer_norm_forward(t["x"], t["lw"], t["lb"], stream=raw)[0]
    side.synchronize()
    assert torch.equal(y0, y1) and torch.equal(n1, P.layer_norm_forward(t["x"], t["lw"], t["lb"])[0])
    for call in (lambda w: P.linear_backward(y0, t["x"], t["w1"], workspace=w), lambda w: P.layer_norm_backward(t["x"], t["x"], t["lw"], *P.layer_norm_forward(t["x"], t["lw"], t["lb"])[2:], workspace=w)):
        for bad in (ws[:0], ws[:100], ws[1:], ws.cpu(), ws.view(torch.int8)):
            with pytest.raises(P.PalsgdError):
                call(bad)


def test_host_threads_at_the_same_time():
    """Calls of distinct threads and streams are independent; a thread may be new to the GPU."""
    work = [_chain(M=200 + 50 * i, seed=10 + i) for i in range(3)]
    want, got = [f() for _, f in work], [None] * 3
    torch.cuda.synchronize()

    def call(i):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(5):
                    got[i] = work[i][1]()
                torch.cuda.current_stream().synchronize()
        except Exception as e:                           # noqa: BLE001 -- reported below, in the test's thread
            got[i] = e

    threads = [threading.Thread(target=call, args=(i,)) for i in range(3)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert all(_same(a, b) for a, b in zip(got, want)), got


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_offsets_beyond_32_bits(dtype):
    """Rows far apart in one long buffer, read and written: the norm, the loss and calls of few tokens."""
    K, M, D, far = 2, 5, 136, 2 ** 29 + 8
    flat = torch.empty((M - 1) * far + 4 * D * K, device="cuda", dtype=DT[dtype])
    view = lambda o, n=D: flat.as_strided((K, M, n), (2 * D, far, 1), o)
    x, y = view(0), view(D)
    src, w, b = _randn(K, M, D, seed=1, dt=DT[dtype]), _randn(K, D, seed=2, dt=DT[dtype]), _randn(K, D, seed=3, dt=DT[dtype])
    bf = dtype == "bf16"
    x.copy_(src)
    _, _, mean, rstd = P.layer_norm_forward(x, w, b, out=(y, None, None, None))
    within(y, *norm64(src, None, w, b, 1e-5, bf)["y"], "norm")
    dx, dw, _ = P.layer_norm_backward(src, x, w, mean, rstd, out=(y, None, None))
    within(y, *norm_backward64(src, src, w, mean, rstd, None, bf)["dx"], "dx")
    t, d = torch.arange(K * M, device="cuda", dtype=torch.int32).view(K, M), torch.ones(K, M, device="cuda")
    loss, lse = P.cross_entropy_forward(x, t)
    within(loss, *loss64(src, t)[0], "loss")
    within(P.cross_entropy_backward(d, x, t, lse, out=y), *loss_backward64(d, src, t, lse, bf), "dlogits")
    weight = _randn(K, D, D, seed=4, dt=DT[dtype], std=D ** -0.5)
    P.linear_forward(x, weight, out=y)
    within(y, *linear64(src, weight, None, None, P.ACT_NONE, bf)["y"], "linear")
    P.linear_backward(x, x, weight, out=(y, None, None))
    ref = linear_backward64(src, src, weight, None, P.ACT_NONE, bf)
    within(y, *ref["dx"], "dx")


def test_matrix_offsets_beyond_32_bits():
    """A million tokens: y and its saved form pass 2^31 elements; the last rows, and weight gradients that only they have."""
    M, D, N, tail = 1_000_037, 16, 2200, 300
    x, w, b, dy = _randn(1, M, D, seed=5), _randn(1, N, D, seed=6, std=0.25), _randn(1, N, seed=7), _randn(1, M, N, seed=8, std=0.01)
    dy[:, :-tail] = 0
    y, z = P.linear_forward(x, w, b, activation=P.ACT_SILU, save=P.SAVE_FULL)
    xt, dyt, zt = x[:, -tail:], dy[:, -tail:], z[:, -tail:]
    within(y[:, -tail:], *linear64(xt, w, b, None, P.ACT_SILU, True)["y"], "y")
    del y
    dx, dw, db = P.linear_backward(dy, x, w, z, activation=P.ACT_SILU)
    ref = linear_backward64(dyt, xt, w, zt, P.ACT_SILU, True)
    within(dx[:, -tail:], *ref["dx"], "dx")
    assert not bool(dx[:, :-tail].any())
    within(dw, *ref["dw"], "dw")
    within(db, *ref["db"], "db")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("kind", range(4))
@pytest.mark.parametrize("M", [1, 300])
def test_activations_of_very_large_values(dtype, kind, M):
    """act(z) is z or 0 there and its slope 1 or 0, up to the largest number.  (At -60 SiLU is 60 e^-60 = 5.3e-25 and its slope
    59 e^-60 = 5.2e-25 away from 0, both below 2^-80; the others, and all further out, are nearer.)"""
    v = torch.tensor([-3e38, -1e30, -1e19, -1e5, -60.0, 60.0, 1e5, 1e19, 1e30, 3e38], device="cuda").to(DT[dtype])
    n = len(v)
    x = torch.ones(1, M, 1, device="cuda", dtype=DT[dtype])
    y, z = P.linear_forward(x, v[None, :, None], activation=kind, save=P.SAVE_FULL)
    want = torch.where(v > 0, v, torch.zeros_like(v)).expand(1, M, n)
    within(y, want.double(), 2.0 ** -80, "y")
    dx, dw, db = P.linear_backward(torch.ones_like(y), x, torch.ones(1, n, 1, device="cuda", dtype=DT[dtype]), z, activation=kind)
    for t in (db[0], dw[0, :, 0]):                         # whole numbers up to 300: exact in binary32, and rounded once
        within(t, ((v > 0) * M).to(DT[dtype]).double(), M * 2.0 ** -80, "slopes")


def test_writing_to_given_memory_raises_its_version():
    t, _ = _chain()
    y = torch.empty(2, 300, 200, device="cuda", dtype=torch.bfloat16)
    before = y._version
    P.linear_forward(t["x"], t["w1"], out=y)
    assert y._version > before
    n = torch.empty_like(t["x"])
    before = n._version
    P.layer_norm_forward(t["x"], t["lw"], t["lb"], out=(n, None, None, None))
    assert n._version > before


def test_python_refusals():
    t, _ = _chain(M=20)
    x, w, b, lw, lb, res = (t[n] for n in ("x", "w1", "b1", "lw", "lb", "res"))
    y, z = P.linear_forward(x, w, b, activation=P.ACT_SILU, save=P.SAVE_FULL)
    _, _, mean, rstd = P.layer_norm_forward(x, lw, lb)
    targets, d = torch.zeros(2, 20, device="cuda", dtype=torch.int32), torch.zeros(2, 20, device="cuda")
    _, lse = P.cross_entropy_forward(x, targets)
    bad = [lambda: P.linear_forward(x.cpu(), w), lambda: P.linear_forward(x.half(), w.half()), lambda: P.linear_forward(x, w.float()),
           lambda: P.linear_forward(x, w[:, :, :-1]), lambda: P.linear_forward(x[0], w), lambda: P.linear_forward(x, w, b[:, :-1]),
           lambda: P.linear_forward(x, w, b, res), lambda: P.linear_forward(x, w, activation=5), lambda: P.linear_forward(x, w, save=P.SAVE_FULL),
           lambda: P.linear_forward(x, w, activation=0, save=3), lambda: P.linear_forward(x, w, activation=1 << 32), lambda: P.linear_forward(x, w, out=y[:, :-1]),
           lambda: P.linear_forward(x.mT.contiguous().mT, w), lambda: P.linear_forward(x, w, out=x[:, :, :200]),
           lambda: P.linear_forward(x, w, b, y, out=y), lambda: P.linear_backward(y, x, w, activation=P.ACT_SILU),
           lambda: P.linear_backward(y, x, w, z), lambda: P.linear_backward(y, x, w, z[:, :-1], activation=0),
           lambda: P.linear_backward(y, x, w, out=(x, None, None)), lambda: P.linear_backward(y, x, w, out=(None, None)),
           lambda: P.linear_backward(y, x, w, out=(None, w, None)), lambda: P.linear_backward(y.expand(2, 20, 200)[:, :, :1].expand(2, 20, 200), x, w),
           lambda: P.layer_norm_forward(x, lw, lb, res[:, :-1]), lambda: P.layer_norm_forward(x, lw.float(), lb), lambda: P.layer_norm_forward(x, lw, lb, eps=-1.0),
           lambda: P.layer_norm_forward(x, lw, lb, out=(x, None, None, None)), lambda: P.layer_norm_forward(x, lw, lb, res, out=(None, res, None, None)),
           lambda: P.layer_norm_forward(torch.zeros(1, 2, 16385, device="cuda"), torch.zeros(1, 16385, device="cuda"), torch.zeros(1, 16385, device="cuda")),
           lambda: P.layer_norm_backward(x, x, lw, mean.double(), rstd), lambda: P.layer_norm_backward(x, x, lw, mean, rstd[:, :-1]),
           lambda: P.layer_norm_backward(x, res, lw, mean, rstd, out=(x, None, None)), lambda: P.layer_norm_backward(x, x, lw, mean, rstd, out=(None,)),
           lambda: P.cross_entropy_forward(x, targets.long()), lambda: P.cross_entropy_forward(x, targets[:, :-1]), lambda: P.cross_entropy_forward(x.double(), targets),
           lambda: P.cross_entropy_backward(d.double(), x, targets, lse), lambda: P.cross_entropy_backward(d, x, targets, lse, out=x[:, :, 1:]),
           lambda: P.cross_entropy_backward(d.bfloat16(), x, targets, lse)]
    for i, call in enumerate(bad):
        with pytest.raises(P.PalsgdError):
            call()
            pytest.fail(f"call {i} was not refused")
    torch.cuda.synchronize()


def test_the_first_calls_of_a_process_may_be_captured():
    """Nothing has been set up on the device before: every operator's first call is inside a capture."""
    import os
    import subprocess
    import sys
    code = """
import torch, paper_2504_18454_b200 as P
x, w, lw = (torch.ones(*s, device="cuda", dtype=torch.bfloat16) for s in ((2, 2100, 64), (2, 600, 64), (2, 64)))
t, d = torch.zeros(2, 2100, device="cuda", dtype=torch.int32), torch.ones(2, 2100, device="cuda")
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    n, total, mean, rstd = P.layer_norm_forward(x, lw, lw, x)
    y, z = P.linear_forward(x, w, activation=P.ACT_SILU, save=P.SAVE_8BIT)
    few, _ = P.linear_forward(x[:, :3], w)
    grads = P.linear_backward(y, x, w, z, activation=P.ACT_SILU)
    few_grads = P.linear_backward(y[:, :3], x[:, :3], w)
    norm_grads = P.layer_norm_backward(x, total, lw, mean, rstd)
    loss, lse = P.cross_entropy_forward(y, t)
    dz = P.cross_entropy_backward(d, y, t, lse)
g.replay()
torch.cuda.synchronize()
assert bool((n == 1).all()) and bool((total == 2).all()) and bool((few == 64).all()) and bool((y == 64).all())
assert bool((few_grads[1] == 192).all()) and bool((norm_grads[2] == 2096).all())
assert abs(float(loss[0, 0]) - 6.3969) < 1e-3
P.block_status()
print("done")
"""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "done" in r.stdout, r.stderr[-2000:]
