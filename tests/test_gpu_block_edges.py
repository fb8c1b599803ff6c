"""The block operators where values are not finite, sizes are empty, or work is long: against their 64-bit statements."""
import pytest
import torch

import paper_2504_18454_b200 as P
from _block_ref import act64, ffn_backward64, ffn_forward64, within

pytestmark = pytest.mark.gpu
DT = {"fp32": torch.float32, "bf16": torch.bfloat16}


def _ffn_inputs(K, M, D, F, dt, seed=1):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s, std: (torch.randn(*s, generator=gen, device="cuda") * std).to(dt)
    return (r(K, M, D, std=1.0), r(K, F, D, std=D ** -0.5), r(K, F, D, std=D ** -0.5), r(K, D, F, std=F ** -0.5),
            r(K, M, D, std=0.01))


# ---------------------------------------------------------------------------------------------- NaN in the gate

@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("kind", range(4))
def test_a_nan_of_the_gate_alone_reaches_the_result(dtype, kind):
    x, wg, wu, wd, _ = _ffn_inputs(1, 40, 64, 96, DT[dtype])
    wg[0, 5, 2] = float("nan")
    y, (g, u) = P.ffn_forward(x, wg, wu, wd, activation=kind)
    assert bool(g[..., 5].isnan().all()) and not bool(u.isnan().any()) and bool(y.isnan().all())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("save", [P.SAVE_FULL, P.SAVE_8BIT])
@pytest.mark.parametrize("kind", range(4))
def test_what_overflowed_in_the_gate_stays_visible_backward(dtype, save, kind):
    """One infinity: its whole group of a checkpoint reads back as NaN.  The gradients of its token and of its columns are
    NaN, all others are as without it."""
    K, M, D, F = 1, 40, 64, 96
    x, wg, wu, wd, dy = _ffn_inputs(K, M, D, F, DT[dtype], seed=2)
    gen = torch.Generator(device="cuda").manual_seed(3)
    g, u = ((torch.randn(K, M, F, generator=gen, device="cuda") * 1.5).to(DT[dtype]) for _ in range(2))
    cols = torch.zeros(F, dtype=torch.bool, device="cuda")
    if save == P.SAVE_8BIT:
        cols[32:64] = True
        g[0, 7, 40] = float("inf")
        saved = (P.act8_pack(g), P.act8_pack(u))
        g, u = (P.act8_unpack(a, dtype=torch.float32) for a in saved)
    else:
        cols[40] = True
        g[0, 7, 40] = float("nan")
        saved = (g, u)
    dx, dwg, dwu, dwd = P.ffn_backward(dy, x, wg, wu, wd, saved, activation=kind)
    assert bool(dx[0, 7].isnan().all())
    for t in (dwg[0, cols], dwu[0, cols], dwd[0][:, cols]):
        assert bool(t.isnan().all())
    want = ffn_backward64(dy, x, wg, wu, wd, g, u, kind, dtype == "bf16")
    rows = torch.arange(M, device="cuda") != 7
    keep = {"dx": (dx, lambda t: t[:, rows]), "dw_gate": (dwg, lambda t: t[:, ~cols]), "dw_up": (dwu, lambda t: t[:, ~cols]),
            "dw_down": (dwd, lambda t: t[:, :, ~cols])}
    for name, (t, cut) in keep.items():
        v, e = want[name]
        assert not bool(cut(t).isnan().any())
        within(cut(t), cut(v), cut(e), name)


# ---------------------------------------------------------------------------------------------- very large gates

@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("save", [P.SAVE_FULL, P.SAVE_8BIT])
@pytest.mark.parametrize("kind", range(4))
def test_the_slope_of_very_large_gates(dtype, save, kind):
    """act' is within 4e-8 of 1 or 0 there, up to the largest number (2^-20: 8 roundings of a number about 1).  With one value,
    u = dy = w_down = w_gate = 1 and w_up = 0, dx is act'(g)."""
    g = torch.tensor([s * v for v in (20.0, 1e3, 1e9, 1e10, 1e18, 2e19, 1e25, 3e38) for s in (1, -1)], device="cuda").to(DT[dtype])[None, :, None]
    one = torch.ones(1, 1, 1, device="cuda", dtype=DT[dtype])
    saved = (g, torch.ones_like(g))
    if save == P.SAVE_8BIT:
        saved = tuple(map(P.act8_pack, saved))
    dx, *_ = P.ffn_backward(torch.ones_like(g), torch.ones_like(g), one, torch.zeros_like(one), one, saved, activation=kind)
    within(dx, act64(kind, g)[1], 2.0 ** -20, "act'")


# ---------------------------------------------------------------------------------------------- q/k: nothing to sum

def _qk_inputs(K, M, HQ, HK, DH, R, dt, seed=1, rows=50):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s, m=0.0, std=1.0: (m + torch.randn(*s, generator=gen, device="cuda") * std).to(dt)
    q, k = r(K, M, HQ, DH), r(K, M, HK, DH, std=3.0)
    ang = torch.rand(rows, R // 2, generator=gen, device="cuda", dtype=torch.float64) * 6.3
    pos = torch.randint(0, rows, (K, M), generator=gen, device="cuda", dtype=torch.int32)
    return q, k, r(K, DH, m=1.0, std=0.2), r(K, DH, m=1.0, std=0.2), ang.cos().float(), ang.sin().float(), pos, r(K, M, HQ, DH, std=0.1), r(K, M, HK, DH, std=0.1)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("heads", [(3, 0), (0, 2), (0, 0)], ids=str)
@pytest.mark.parametrize("tokens", [0, 9])
@pytest.mark.parametrize("DH", [40, 33])
def test_the_weight_gradient_of_no_heads_is_zero(dtype, heads, tokens, DH):
    K = 2
    q, k, wq, wk, cos, sin, pos, dq, dk = _qk_inputs(K, tokens, *heads, DH, 8, DT[dtype])
    dw = tuple(torch.full((K, DH + 8), 7.0, device="cuda", dtype=DT[dtype]) for _ in range(2))
    inner = tuple(t[:, 3:3 + DH] for t in dw)
    P.qk_norm_rope_backward(dq, dk, q, k, wq, wk, cos, sin, pos, out=(None, None, *inner))
    for t, i, n in zip(dw, inner, heads):
        assert bool((i == 0).all()) if n == 0 or tokens == 0 else not bool((i == 7).any())
        assert bool((t[:, :3] == 7).all()) and bool((t[:, 3 + DH:] == 7).all())


def test_autograd_gives_zero_for_the_weights_of_no_heads():
    from paper_2504_18454_b200 import autograd as A
    q, k, wq, wk, cos, sin, pos, dq, dk = _qk_inputs(2, 9, 3, 0, 40, 8, torch.float32)
    junk = [torch.full((2, 40), float("nan"), device="cuda") for _ in range(64)]      # what a fresh tensor may lie over
    del junk
    wq.requires_grad_(), wk.requires_grad_()
    A.qk_norm_rope(q, k, wq, wk, cos, sin, pos)[0].backward(dq)
    assert bool((wk.grad == 0).all()) and bool((wq.grad != 0).any())


# ---------------------------------------------------------------------------------------------- q/k: an infinite gradient

@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("size", [(1, 33, 64, 64), (1, 41, 64, 20), (1, 65, 32, 32), (1, 33, 33, 20), (40003, 3, 64, 64)], ids=str)
@pytest.mark.parametrize("interleaved", [False, True])
def test_an_infinite_gradient_gives_an_infinite_weight_gradient(dtype, size, interleaved):
    """Not NaN: heads (or tokens) that a warp's last group lacks, and whose place held an infinity before, add nothing.  The
    gradient of one value is infinite in every head; it and its partner of the rotation have x > 0, so no infinities of
    both signs meet."""
    M, HQ, DH, R = size
    q, k, wq, wk, cos, sin, pos, dq, dk = _qk_inputs(1, M, HQ, 1, DH, R, DT[dtype], seed=4)
    cos.fill_(0.6), sin.fill_(0.8)
    a, b = (2, 3) if interleaved else (2, 2 + R // 2)
    dq[..., a], q[..., a], q[..., b] = float("inf"), 1.0, 1.0
    _, _, dw, _ = P.qk_norm_rope_backward(dq, dk, q, k, wq, wk, cos, sin, pos, interleaved=interleaved)
    assert float(dw[0, a]) == float("inf") and float(dw[0, b]) == float("-inf")
    rest = [i for i in range(DH) if i not in (a, b)]
    assert bool(dw[0, rest].isfinite().all())


# ---------------------------------------------------------------------------------------------- workspaces

def test_an_empty_workspace_is_refused():
    """Its address is NULL; a call that took that for the question how large it has to be would leave its outputs unwritten."""
    x, wg, wu, wd, dy = _ffn_inputs(1, 40, 64, 96, torch.bfloat16)
    none = torch.empty(0, dtype=torch.uint8, device="cuda")
    _, saved = P.ffn_forward(x, wg, wu, wd)
    q, k, wq, wk, cos, sin, pos, dq, dk = _qk_inputs(1, 9, 2, 1, 64, 64, torch.bfloat16)
    for call in (lambda: P.ffn_forward(x, wg, wu, wd, workspace=none), lambda: P.ffn_backward(dy, x, wg, wu, wd, saved, workspace=none),
                 lambda: P.qk_norm_rope_backward(dq, dk, q, k, wq, wk, cos, sin, pos, workspace=none)):
        with pytest.raises(P.PalsgdError, match="workspace"):
            call()


def test_no_tokens_with_the_workspace_that_the_library_asks_for():
    """The C calls as the header says: ask, allocate that much, call.  The weight gradients become zero."""
    import ctypes as C
    from paper_2504_18454_b200 import block as B
    K, D, F = 2, 40, 24
    dw = [torch.full((K, *s), 7.0, device="cuda", dtype=torch.bfloat16) for s in ((F, D), (F, D), (D, F))]
    w = [torch.zeros_like(t) for t in dw]
    mat = lambda t: C.byref(B.Mat(t.data_ptr(), t.stride(0), t.stride(1)))
    empty = C.byref(B.Mat(None, 0, 0))
    s, n = B.FfnShape(K, P.PREC_BF16_MASTER, 0, P.SAVE_FULL, 0, D, F), C.c_size_t(0)
    call = lambda ws: B.lib().palsgd_ffn_backward(C.byref(s), empty, empty, None, *map(mat, w), empty, empty, None, None, None, *map(mat, dw),
                                                  ws, C.byref(n), torch.cuda.current_stream().cuda_stream)
    assert call(None) == 0
    ws = torch.empty(n.value, dtype=torch.uint8, device="cuda")
    assert call(ws.data_ptr()) == 0
    assert all(bool((t == 0).all()) for t in dw)


# ---------------------------------------------------------------------------------------------- outputs that autograd has saved

def test_writing_to_given_memory_raises_its_version():
    x, wg, wu, wd, dy = _ffn_inputs(1, 40, 64, 96, torch.bfloat16)
    q, k, wq, wk, cos, sin, pos, dq, dk = _qk_inputs(1, 9, 2, 1, 64, 64, torch.bfloat16)
    _, saved = P.ffn_forward(x, wg, wu, wd)
    px, (_, saved8) = P.act8_pack(x), P.ffn_forward(x, wg, wu, wd, save=P.SAVE_8BIT)
    new = torch.empty_like
    calls = [(lambda o: P.ffn_forward(x, wg, wu, wd, out=o[0], saved=tuple(o[1:])), [x, *saved]),
             (lambda o: P.ffn_forward(x, wg, wu, wd, out=o[0], saved=(P.Act8(o[1], o[2], x.dtype), P.Act8(o[3], o[4], x.dtype)), save=P.SAVE_8BIT),
              [x, saved8[0].q, saved8[0].exponent, saved8[1].q, saved8[1].exponent]),
             (lambda o: P.ffn_backward(dy, x, wg, wu, wd, saved, out=tuple(o)), [x, wg, wu, wd]),
             (lambda o: P.act8_pack(x, out=P.Act8(o[0], o[1], x.dtype)), [px.q, px.exponent]), (lambda o: P.act8_unpack(px, out=o[0]), [x]),
             (lambda o: P.qk_norm_rope(q, k, wq, wk, cos, sin, pos, out=tuple(o)), [q, k]),
             (lambda o: P.qk_norm_rope_backward(dq, dk, q, k, wq, wk, cos, sin, pos, out=tuple(o)), [q, k, wq, wk])]
    for call, like in calls:
        outs = [new(t) for t in like]
        before = [t._version for t in outs]
        call(outs)
        assert all(t._version > v for t, v in zip(outs, before))
        with torch.inference_mode():
            call([new(t) for t in like])


def test_autograd_sees_that_a_saved_tensor_was_written_to():
    x, wg, wu, wd, _ = _ffn_inputs(1, 40, 64, 96, torch.bfloat16)
    h = x.requires_grad_() * 2
    z = h * h                                            # saves h
    P.ffn_forward(x.detach(), wg, wu, wd, save=P.SAVE_NONE, out=h.detach())
    with pytest.raises(RuntimeError, match="inplace"):
        z.sum().backward()


# ---------------------------------------------------------------------------------------------- overlap

def test_overlapping_outputs_are_refused():
    """dx written in the launch that reads dy would race; so would any other output over an input."""
    x, wg, wu, wd, dy = _ffn_inputs(1, 40, 64, 96, torch.bfloat16)
    _, saved = P.ffn_forward(x, wg, wu, wd)
    q, k, wq, wk, cos, sin, pos, dq, dk = _qk_inputs(1, 9, 2, 2, 64, 64, torch.bfloat16)
    p = P.act8_pack(x)
    for call in (lambda: P.ffn_backward(dy, x, wg, wu, wd, saved, out=(dy, None, None, None)),
                 lambda: P.ffn_backward(dy, x, wg, wu, wd, saved, out=(None, wg, None, None)),
                 lambda: P.ffn_forward(x, wg, wu, wd, out=x), lambda: P.ffn_forward(x, wg, wu, wd, saved=(saved[0], saved[0])),
                 lambda: P.act8_unpack(P.Act8(x.view(torch.int8)[..., :64], p.exponent, x.dtype), out=x),
                 lambda: P.act8_pack(x, out=P.Act8(x.view(torch.int8)[..., :64], p.exponent, x.dtype)),
                 lambda: P.qk_norm_rope(q, k, wq, wk, cos, sin, pos, out=(k, None)), lambda: P.qk_norm_rope(q, k, wq, wk, cos, sin, pos, out=(k, q)),
                 lambda: P.qk_norm_rope_backward(dq, dk, q, k, wq, wk, cos, sin, pos, out=(dk, None, None, None))):
        with pytest.raises(P.PalsgdError):
            call()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("size", [(2, 3001, 6, 2, 64, 64), (1, 700, 3, 3, 64, 20), (1, 300, 3, 1, 33, 20)], ids=str)
@pytest.mark.parametrize("interleaved", [False, True])
def test_heads_in_place(dtype, size, interleaved):
    """A head is read before it is written: q_out = q, and dq = dq_out or q, give the same bits."""
    q, k, wq, wk, cos, sin, pos, dq, dk = _qk_inputs(*size, DT[dtype], seed=8)
    kw = dict(interleaved=interleaved)
    want = P.qk_norm_rope(q, k, wq, wk, cos, sin, pos, **kw)
    back = P.qk_norm_rope_backward(dq, dk, q, k, wq, wk, cos, sin, pos, **kw)
    a, b = q.clone(), k.clone()
    P.qk_norm_rope(a, b, wq, wk, cos, sin, pos, out=(a, b), **kw)
    assert torch.equal(a, want[0]) and torch.equal(b, want[1])
    a, b = dq.clone(), k.clone()
    got = P.qk_norm_rope_backward(a, dk, q, b, wq, wk, cos, sin, pos, out=(a, b, None, None), **kw)
    assert all(torch.equal(s, t) for s, t in zip(got, back))


# ---------------------------------------------------------------------------------------------- a wait that gave up

def test_training_ends_with_an_error_where_a_kernel_gave_up(monkeypatch):
    """What palsgd_block_status reports of a bounded wait reaches whoever trains (the report itself is made on the host here)."""
    from paper_2504_18454_b200 import train
    seen = []

    def status(stream=None):
        seen.append(stream)
        if len(seen) == 2:
            raise P.PalsgdError(-3, "palsgd_block_status", "a matrix kernel's wait gave up")

    monkeypatch.setattr(train, "block_status", status)
    steps = []
    with pytest.raises(P.PalsgdError, match="gave up"):
        train.run(K=1, steps=40, layers=1, width=64, hidden=64, report=lambda t, v: steps.append(t))
    assert len(seen) == 2 and steps == [0]


# ---------------------------------------------------------------------------------------------- numbers of more than 32 bits

def test_an_activation_or_saved_form_beyond_32_bits_is_refused():
    """Not cut to its low half, which is a valid one."""
    x, wg, wu, wd, dy = _ffn_inputs(1, 40, 64, 96, torch.bfloat16)
    _, saved = P.ffn_forward(x, wg, wu, wd)
    for n in (2 ** 32, 2 ** 32 + 1, -2 ** 32):
        for call in (lambda: P.ffn_forward(x, wg, wu, wd, activation=n), lambda: P.ffn_forward(x, wg, wu, wd, save=n),
                     lambda: P.ffn_backward(dy, x, wg, wu, wd, saved, activation=n)):
            with pytest.raises(P.PalsgdError):
                call()
