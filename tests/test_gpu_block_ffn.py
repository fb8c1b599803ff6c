"""The gated feed-forward block against its 64-bit statement: types, activations, saved forms, odd sizes, strides."""
import pytest
import torch

import paper_2504_18454_b200 as P
from _block_ref import ffn_backward64, ffn_forward64, rounded, within

pytestmark = pytest.mark.gpu
DT = {"fp32": torch.float32, "bf16": torch.bfloat16}
# K, tokens, d_model, d_ff: one token, odd everything, one tile, just past a tile, several tiles, a long inner axis
SIZES = [(1, 1, 1, 1), (1, 1, 64, 128), (2, 3, 7, 5), (3, 129, 65, 257), (1, 128, 64, 256), (4, 17, 256, 683),
         (2, 300, 264, 520), (1, 40, 1032, 72), (1, 1000, 40, 48), (2, 257, 136, 1000)]


def _inputs(K, M, D, F, dt, seed=1):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s, std: (torch.randn(*s, generator=gen, device="cuda") * std).to(dt)
    return (r(K, M, D, std=1.0), r(K, F, D, std=D ** -0.5), r(K, F, D, std=D ** -0.5), r(K, D, F, std=F ** -0.5),
            r(K, M, D, std=0.01))


def _check_saved(saved, want, save, dt, K, M, F):
    for t, name in zip(saved, ("gate", "up")):
        v, e = want[name]
        if save == P.SAVE_FULL:
            within(t, v, rounded(v, e, dt == torch.bfloat16), name)
        else:
            step = torch.exp2(t.exponent.double() - 127).repeat_interleave(32, -1)[..., :F]
            within(P.act8_unpack(t, dtype=torch.float32), v, step / 2 + e, name)
            G = t.exponent.shape[-1]
            pad = torch.zeros(K, M, G * 32, device=v.device, dtype=torch.float64)
            pad[..., :F] = v.abs() + e
            top = pad.view(K, M, G, 32).amax(-1)
            # the smallest power of two that holds the group: the next smaller one would need more than 127 steps
            assert bool((torch.exp2(t.exponent.double() - 127) / 2 * 127 <= top).logical_or(t.exponent == 1).all())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("save", [P.SAVE_FULL, P.SAVE_8BIT])
def test_forward(dtype, size, save):
    K, M, D, F = size
    x, wg, wu, wd, _ = _inputs(K, M, D, F, DT[dtype])
    kind = (K + M) % 4
    y, saved = P.ffn_forward(x, wg, wu, wd, activation=kind, save=save)
    want = ffn_forward64(x, wg, wu, wd, kind, dtype == "bf16")
    within(y, *want["y"], "y")
    _check_saved(saved, want, save, DT[dtype], K, M, F)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("save", [P.SAVE_FULL, P.SAVE_8BIT])
def test_backward(dtype, size, save):
    K, M, D, F = size
    x, wg, wu, wd, dy = _inputs(K, M, D, F, DT[dtype], seed=2)
    kind = (K + M + 1) % 4
    gen = torch.Generator(device="cuda").manual_seed(3)
    g, u = ((torch.randn(K, M, F, generator=gen, device="cuda") * 1.5).to(DT[dtype]) for _ in range(2))
    xs, saved = x, (g, u)
    if save == P.SAVE_8BIT:
        saved = (P.act8_pack(g), P.act8_pack(u))
        xs = P.act8_pack(x)
        x, g, u = (P.act8_unpack(a, dtype=torch.float32) for a in (xs, *saved))
    got = P.ffn_backward(dy, xs, wg, wu, wd, saved, activation=kind)
    want = ffn_backward64(dy, x, wg, wu, wd, g, u, kind, dtype == "bf16")
    for t, name in zip(got, ("dx", "dw_gate", "dw_up", "dw_down")):
        within(t, *want[name], name)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("kind", range(4))
def test_every_activation_over_its_range(dtype, kind):
    # g runs over -12 .. 12 (and the exact 0): one inner element, weight 1, so g = x and u = 1
    x = torch.cat([torch.linspace(-12, 12, 512), torch.zeros(1)]).cuda().to(DT[dtype])[None, :, None]
    one = torch.ones(1, 1, 1, device="cuda", dtype=DT[dtype])
    y, saved = P.ffn_forward(x, one, one, one, activation=kind)
    want = ffn_forward64(x, one, one, one, kind, dtype == "bf16")
    within(y, *want["y"], "y")
    dy = torch.ones_like(x)
    got = P.ffn_backward(dy, x, one, one, one, saved, activation=kind)
    ref = ffn_backward64(dy, x, one, one, one, saved[0], saved[1], kind, dtype == "bf16")
    for t, name in zip(got, ("dx", "dw_gate", "dw_up", "dw_down")):
        within(t, *ref[name], name)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("odd", [False, True])
def test_strided_operands_and_untouched_surroundings(dtype, odd):
    """Weights and gradients as views of packed rows (at an odd offset: not 16-byte aligned), activations as views of
    wider rows, outputs inside sentinels."""
    dt, (K, M, D, F) = DT[dtype], (3, 70, 72, 136)
    x, wg, wu, wd, dy = _inputs(K, M, D, F, dt, seed=4)
    shift = 1 if odd else 8
    row = 3 * F * D + 64

    def arena():
        a = torch.full((K, row), 1536.0, device="cuda", dtype=dt)
        v = a[:, shift:shift + 3 * F * D]
        return a, v[:, :F * D].unflatten(1, (F, D)), v[:, F * D:2 * F * D].unflatten(1, (F, D)), v[:, 2 * F * D:].unflatten(1, (D, F))

    aw, vg, vu, vd = arena()
    vg.copy_(wg), vu.copy_(wu), vd.copy_(wd)
    wide = lambda n: torch.full((K, M, n + 16), 1536.0, device="cuda", dtype=dt)
    xb, yb, db, dyb, gb, ub = wide(D), wide(D), wide(D), wide(D), wide(F), wide(F)
    inner = lambda t, n: t[:, :, shift:shift + n]
    inner(xb, D).copy_(x), inner(dyb, D).copy_(dy)
    y, saved = P.ffn_forward(inner(xb, D), vg, vu, vd, out=inner(yb, D), saved=(inner(gb, F), inner(ub, F)))
    want = ffn_forward64(x, wg, wu, wd, 0, dtype == "bf16")
    within(inner(yb, D), *want["y"], "y")
    _check_saved(saved, want, P.SAVE_FULL, dt, K, M, F)
    ag, gg, gu, gd = arena()
    P.ffn_backward(inner(dyb, D), inner(xb, D), vg, vu, vd, saved, out=(inner(db, D), gg, gu, gd))
    ref = ffn_backward64(dy, x, wg, wu, wd, saved[0], saved[1], 0, dtype == "bf16")
    for t, name in zip((inner(db, D), gg, gu, gd), ("dx", "dw_gate", "dw_up", "dw_down")):
        within(t, *ref[name], name)
    for t, n in ((xb, D), (yb, D), (db, D), (dyb, D), (gb, F), (ub, F)):
        assert bool((t[:, :, :shift] == 1536).all()) and bool((t[:, :, shift + n:] == 1536).all())
    for a in (aw, ag):
        assert bool((a[:, :shift] == 1536).all()) and bool((a[:, shift + 3 * F * D:] == 1536).all())


def test_workers_share_one_matrix_and_tokens_interleave_with_workers():
    """worker stride 0 (all workers read one weight), and activations stored token-major (tokens, K, d)."""
    K, M, D, F = 3, 50, 64, 96
    x, wg, wu, wd, _ = _inputs(K, M, D, F, torch.bfloat16, seed=5)
    wg, wu, wd = (w[:1].expand(K, -1, -1) for w in (wg, wu, wd))
    xt = x.transpose(0, 1).contiguous().transpose(0, 1)
    out = torch.empty(M, K, D, device="cuda", dtype=torch.bfloat16).transpose(0, 1)
    y, _ = P.ffn_forward(xt, wg, wu, wd, save=P.SAVE_NONE, out=out)
    within(y, *ffn_forward64(x, wg, wu, wd, 0, True)["y"], "y")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_no_tokens_gives_zero_weight_gradients(dtype):
    K, D, F = 2, 40, 24
    x, wg, wu, wd, dy = _inputs(K, 0, D, F, DT[dtype])
    y, saved = P.ffn_forward(x, wg, wu, wd)
    assert y.shape == (K, 0, D)
    outs = tuple(torch.full(s, 7.0, device="cuda", dtype=DT[dtype]) for s in ((K, 0, D), (K, F, D), (K, F, D), (K, D, F)))
    P.ffn_backward(dy, x, wg, wu, wd, saved, out=outs)
    assert all(bool((t == 0).all()) for t in outs)


def test_nan_and_infinity_stay_in_their_rows():
    K, M, D, F = 1, 200, 64, 160
    x, wg, wu, wd, _ = _inputs(K, M, D, F, torch.bfloat16, seed=6)
    x[0, 17, 3], x[0, 150, 0] = float("nan"), float("inf")
    y, saved = P.ffn_forward(x, wg, wu, wd, save=P.SAVE_8BIT)
    rows = torch.isfinite(y[0].float()).all(-1)
    assert not bool(rows[17]) and not bool(rows[150]) and int(rows.sum()) == M - 2
    g = P.act8_unpack(saved[0])
    assert bool(g[0, 17].isnan().all()) and bool(torch.isfinite(g[0, rows].float()).all())


def test_no_input_gradient_and_repeatable():
    K, M, D, F = 2, 333, 96, 200
    x, wg, wu, wd, dy = _inputs(K, M, D, F, torch.bfloat16, seed=7)
    _, saved = P.ffn_forward(x, wg, wu, wd)
    a = P.ffn_backward(dy, x, wg, wu, wd, saved)
    b = P.ffn_backward(dy, x, wg, wu, wd, saved, need_dx=False)
    assert b[0] is None
    for s, t in zip(a[1:], b[1:]):
        assert torch.equal(s, t)
    for s, t in zip(a, P.ffn_backward(dy, x, wg, wu, wd, saved)):
        assert torch.equal(s, t)


def test_another_stream_and_a_given_workspace():
    K, M, D, F = 2, 100, 64, 96
    x, wg, wu, wd, dy = _inputs(K, M, D, F, torch.bfloat16, seed=8)
    y0, s0 = P.ffn_forward(x, wg, wu, wd)
    g0 = P.ffn_backward(dy, x, wg, wu, wd, s0)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    ws = torch.full((1 << 22,), 255, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    y1, s1 = P.ffn_forward(x, wg, wu, wd, workspace=ws, stream=side.cuda_stream)
    g1 = P.ffn_backward(dy, x, wg, wu, wd, s1, workspace=ws, stream=side.cuda_stream)
    side.synchronize()
    assert torch.equal(y0, y1) and all(torch.equal(a, b) for a, b in zip(g0, g1))
    with pytest.raises(P.PalsgdError):
        P.ffn_forward(x, wg, wu, wd, workspace=ws[:256])
    with pytest.raises(P.PalsgdError):
        P.ffn_forward(x, wg, wu, wd, workspace=ws[1:])


def test_calls_can_be_captured_in_a_graph():
    K, M, D, F = 2, 64, 64, 96
    x, wg, wu, wd, dy = _inputs(K, M, D, F, torch.bfloat16, seed=9)
    y0, s0 = P.ffn_forward(x, wg, wu, wd)
    g0 = P.ffn_backward(dy, x, wg, wu, wd, s0)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y1, s1 = P.ffn_forward(x, wg, wu, wd)
        g1 = P.ffn_backward(dy, x, wg, wu, wd, s1)
    graph.replay()
    assert torch.equal(y0, y1) and all(torch.equal(a, b) for a, b in zip(g0, g1))


def test_gradients_against_differences():
    """Directional differences of the fp32 forward pass.  f(t) = <dy, y(p + t v)> with |v| chosen so that y moves by
    about its own size at t = 1: at t = 2^-5 the third-order term is a few 1e-4 of f', rounding (2e-6 / 2^-5) less."""
    K, M, D, F = 2, 19, 24, 40
    x, wg, wu, wd, dy = _inputs(K, M, D, F, torch.float32, seed=10)
    _, saved = P.ffn_forward(x, wg, wu, wd, activation=P.ACT_GELU_TANH)
    grads = P.ffn_backward(dy, x, wg, wu, wd, saved, activation=P.ACT_GELU_TANH)
    f = lambda *a: (P.ffn_forward(*a, activation=P.ACT_GELU_TANH, save=P.SAVE_NONE)[0].double() * dy.double()).sum()
    args, h = [x, wg, wu, wd], 2.0 ** -5
    gen = torch.Generator(device="cuda").manual_seed(11)
    for i in range(4):
        v = torch.randn(args[i].shape, generator=gen, device="cuda") * args[i].std()
        up, down = ([a + s * h * v if j == i else a for j, a in enumerate(args)] for s in (1, -1))
        numeric = float((f(*up) - f(*down)) / (2 * h))
        scale = float(grads[i].double().norm() * v.double().norm())
        assert abs(numeric - float((grads[i].double() * v.double()).sum())) <= 2e-3 * scale


def test_python_refusals():
    K, M, D, F = 1, 4, 8, 16
    x, wg, wu, wd, dy = _inputs(K, M, D, F, torch.bfloat16)
    _, saved = P.ffn_forward(x, wg, wu, wd)
    bad = [lambda: P.ffn_forward(x.cpu(), wg, wu, wd), lambda: P.ffn_forward(x.half(), wg, wu, wd),
           lambda: P.ffn_forward(x, wg.float(), wu, wd), lambda: P.ffn_forward(x, wg, wu[:, :-1], wd),
           lambda: P.ffn_forward(x, wg, wu, wd.mT), lambda: P.ffn_forward(x[0], wg, wu, wd),
           lambda: P.ffn_forward(x, wg, wu, wd, activation=4), lambda: P.ffn_forward(x, wg, wu, wd, save=3),
           lambda: P.ffn_forward(x.mT.contiguous().mT, wg, wu, wd),
           lambda: P.ffn_backward(dy, P.act8_pack(x), wg, wu, wd, saved),
           lambda: P.ffn_backward(dy, x, wg, wu, wd, (saved[0], P.act8_pack(saved[1]))),
           lambda: P.ffn_backward(dy, x, wg, wu, wd, None),
           lambda: P.ffn_backward(dy, x, wg, wu, wd, saved, out=(None,))]
    for call in bad:
        with pytest.raises(P.PalsgdError):
            call()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("size", [(1, 1, 64, 4096), (1, 5, 33, 3001), (2, 3000, 72, 40), (1, 7000, 16, 264)], ids=str)
def test_long_inner_axes_with_few_tiles(dtype, size):
    """The products' inner axes are cut into shares here: few tiles, up to 110 steps of 64 each."""
    K, M, D, F = size
    x, wg, wu, wd, dy = _inputs(K, M, D, F, DT[dtype], seed=12)
    y, saved = P.ffn_forward(x, wg, wu, wd, activation=P.ACT_GELU)
    want = ffn_forward64(x, wg, wu, wd, P.ACT_GELU, dtype == "bf16")
    within(y, *want["y"], "y")
    got = P.ffn_backward(dy, x, wg, wu, wd, saved, activation=P.ACT_GELU)
    ref = ffn_backward64(dy, x, wg, wu, wd, saved[0], saved[1], P.ACT_GELU, dtype == "bf16")
    for t, name in zip(got, ("dx", "dw_gate", "dw_up", "dw_down")):
        within(t, *ref[name], name)
    for a, b in zip(got, P.ffn_backward(dy, x, wg, wu, wd, saved, activation=P.ACT_GELU)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("shift", range(1, 8))
def test_every_alignment_of_outputs_and_saved_checkpoints(shift):
    """Rows at every offset from a 16-byte boundary: forward writes to them, backward reads from them."""
    K, M, D, F = 2, 45, 50, 83
    x, wg, wu, wd, dy = _inputs(K, M, D, F, torch.bfloat16, seed=13)
    wide = lambda n, dt, v: torch.full((K, M, n + 19), v, device="cuda", dtype=dt)
    yb, gb, ub = wide(D, torch.bfloat16, 1536.0), wide(F, torch.int8, 99), wide(F, torch.int8, 99)
    ge, ue = (torch.empty(K, M, 3, device="cuda", dtype=torch.uint8) for _ in range(2))
    cut = lambda t, n: t[:, :, shift:shift + n]
    saved = (P.Act8(cut(gb, F), ge, x.dtype), P.Act8(cut(ub, F), ue, x.dtype))
    P.ffn_forward(x, wg, wu, wd, save=P.SAVE_8BIT, out=cut(yb, D), saved=saved)
    y0, saved0 = P.ffn_forward(x, wg, wu, wd, save=P.SAVE_8BIT)
    assert torch.equal(cut(yb, D), y0)
    for a, b in zip(saved, saved0):
        assert torch.equal(a.q, b.q) and torch.equal(a.exponent, b.exponent)
    for t, n, v in ((yb, D, 1536), (gb, F, 99), (ub, F, 99)):
        assert bool((t[:, :, :shift] == v).all()) and bool((t[:, :, shift + n:] == v).all())
    xb = wide(D, torch.int8, 99)
    px = P.act8_pack(x)
    cut(xb, D).copy_(px.q)
    for a, b in zip(P.ffn_backward(dy, P.Act8(cut(xb, D), px.exponent, x.dtype), wg, wu, wd, saved),
                    P.ffn_backward(dy, px, wg, wu, wd, saved0)):
        assert torch.equal(a, b)


def test_a_thread_that_has_not_used_the_gpu_yet():
    import threading
    K, M, D, F = 1, 40, 64, 96
    x, wg, wu, wd, dy = _inputs(K, M, D, F, torch.bfloat16, seed=14)
    y, saved = P.ffn_forward(x, wg, wu, wd)
    want, got = P.ffn_backward(dy, x, wg, wu, wd, saved), []
    torch.cuda.synchronize()

    def call():
        try:
            got.extend(P.ffn_backward(dy, x, wg, wu, wd, saved))
        except Exception as e:                           # noqa: BLE001 -- reported below, in the test's thread
            got.append(e)

    t = threading.Thread(target=call)
    t.start()
    t.join()
    torch.cuda.synchronize()
    assert len(got) == 4 and all(torch.equal(a, b) for a, b in zip(got, want)), got


def test_offsets_beyond_31_bits():
    """One worker, a million tokens: gate, up and the hidden rows pass 2^31 elements.  The last rows are compared with the
    64-bit statement, and so are the weight gradients of a batch whose gradient is zero but for them."""
    M, D, F, tail = 1_000_037, 16, 2200, 300
    x, wg, wu, wd, dy = _inputs(1, M, D, F, torch.bfloat16, seed=15)
    dy[:, :-tail] = 0
    y, saved = P.ffn_forward(x, wg, wu, wd)
    xt, dyt = x[:, -tail:], dy[:, -tail:]
    want = ffn_forward64(xt, wg, wu, wd, 0, True)
    within(y[:, -tail:], *want["y"], "y")
    _check_saved([s[:, -tail:] for s in saved], want, P.SAVE_FULL, torch.bfloat16, 1, tail, F)
    got = P.ffn_backward(dy, x, wg, wu, wd, saved)
    ref = ffn_backward64(dyt, xt, wg, wu, wd, *(s[:, -tail:] for s in saved), 0, True)
    within(got[0][:, -tail:], *ref["dx"], "dx")
    assert bool((got[0][:, :-tail] == 0).all())
    for t, name in zip(got[1:], ("dw_gate", "dw_up", "dw_down")):
        within(t, *ref[name], name)
