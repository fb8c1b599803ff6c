"""The linear operator against its 64-bit statement: types, activations, saved forms, odd sizes, strides, few tokens, shares."""
import pytest
import torch

import paper_2504_18454_b200 as P
from _block_ref import rounded, within
from _more_ref import NONE, linear64, linear_backward64

pytestmark = pytest.mark.gpu
DT = {"fp32": torch.float32, "bf16": torch.bfloat16}
# K, tokens, d_in, d_out: one token, odd everything, few tokens, one tile, just past a tile, several tiles, a long inner axis
SIZES = [(1, 1, 1, 1), (1, 1, 64, 128), (2, 3, 7, 5), (1, 8, 2056, 40), (3, 5, 513, 33), (2, 9, 24, 33), (3, 129, 65, 257), (1, 128, 64, 256),
         (4, 17, 256, 683), (2, 300, 264, 520), (1, 40, 4104, 72), (1, 1000, 40, 48), (2, 257, 136, 1000), (1, 16, 40, 1500), (2, 17, 300, 1025), (3, 512, 100, 70), (1, 40, 9000, 1030),
         (2, 700, 600, 601), (1, 100, 9000, 265)]


def _inputs(K, M, D, N, dt, seed=1):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s, std: (torch.randn(*s, generator=gen, device="cuda") * std).to(dt)
    return (r(K, M, D, std=1.0), r(K, N, D, std=D ** -0.5), r(K, N, std=0.5), r(K, M, N, std=2.0), r(K, M, N, std=0.01),
            r(K, M, N, std=1.5))


def check_saved(saved, want, dt, N):
    v, e = want
    if not isinstance(saved, P.Act8):
        return within(saved, v, rounded(v, e, dt == torch.bfloat16), "z")
    step = torch.exp2(saved.exponent.double() - 127).repeat_interleave(32, -1)[..., :N]
    within(P.act8_unpack(saved, dtype=torch.float32), v, step / 2 + e, "z")
    pad = torch.nn.functional.pad(v.abs() + e, (0, -N % 32)).unflatten(-1, (-1, 32)).amax(-1)
    # the smallest power of two that holds the group: the next smaller one would need more than 127 steps
    assert bool((torch.exp2(saved.exponent.double() - 127) / 2 * 127 <= pad).logical_or(saved.exponent == 1).all())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("save", [P.SAVE_NONE, P.SAVE_FULL, P.SAVE_8BIT])
def test_forward(dtype, size, save):
    K, M, D, N = size
    x, w, b, r, _, _ = _inputs(*size, DT[dtype])
    kind = (K + M) % 4 if save != P.SAVE_NONE else ((K + M + N) % 5)
    bias, residual = (b if (M + N) % 3 else None), (r if (M + D) % 2 else None)
    y, saved = P.linear_forward(x, w, bias, residual, activation=kind, save=save)
    want = linear64(x, w, bias, residual, kind, dtype == "bf16")
    within(y, *want["y"], "y")
    if save == P.SAVE_NONE:
        assert saved is None
    else:
        check_saved(saved, want["z"], DT[dtype], N)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("M", [3, 40, 130, 700])
def test_every_part_of_the_epilogue(dtype, bias, residual, M):
    """A call of few tokens, two whose inner axis is cut into shares (in fp32 the longer one), one of whole tiles."""
    x, w, b, r, _, _ = _inputs(2, M, 4096 if M in (40, 130) else 520, 264, DT[dtype], seed=5)
    b, r = b if bias else None, r if residual else None
    for kind in (NONE, P.ACT_RELU):
        y, _ = P.linear_forward(x, w, b, r, activation=kind)
        within(y, *linear64(x, w, b, r, kind, dtype == "bf16")["y"], "y")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("save", [P.SAVE_NONE, P.SAVE_FULL, P.SAVE_8BIT])
def test_backward(dtype, size, save):
    K, M, D, N = size
    x, w, _, _, dy, z = _inputs(*size, DT[dtype], seed=2)
    kind = NONE if save == P.SAVE_NONE else (K + M + 1) % 4
    xs, saved = x, z
    if save == P.SAVE_NONE:
        saved = None
    elif save == P.SAVE_8BIT:
        saved, xs = P.act8_pack(z), P.act8_pack(x)
        z, x = (P.act8_unpack(a, dtype=torch.float32) for a in (saved, xs))
    got = P.linear_backward(dy, xs, w, saved, activation=kind)
    want = linear_backward64(dy, x, w, z, kind, dtype == "bf16")
    for t, name in zip(got, ("dx", "dw", "db")):
        within(t, *want[name], name)
    if save == P.SAVE_NONE:                                # the input in 8 bits, no activation
        x8 = P.act8_pack(x)
        got = P.linear_backward(dy, x8, w)
        want = linear_backward64(dy, P.act8_unpack(x8, dtype=torch.float32), w, z, kind, dtype == "bf16")
        for t, name in zip(got, ("dx", "dw", "db")):
            within(t, *want[name], name)
    if save == P.SAVE_8BIT:                                # the input in the storage type beside an 8-bit z
        within(P.linear_backward(dy, x.to(DT[dtype]), w, saved, activation=kind)[1], *want["dw"], "dw")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("kind", range(5))
@pytest.mark.parametrize("M", [1, 513])
def test_every_activation_over_its_range(dtype, kind, M):
    """z runs over -12 .. 12 and 0: one inner element, weights that are the values (M = 1) or 1."""
    v = torch.cat([torch.linspace(-12, 12, 512), torch.zeros(1)]).cuda().to(DT[dtype])
    one = torch.ones(1, 1, 1, device="cuda", dtype=DT[dtype])
    x, w = (one, v[None, :, None]) if M == 1 else (v[None, :, None], one)
    save = P.SAVE_NONE if kind == NONE else P.SAVE_FULL
    y, z = P.linear_forward(x, w, activation=kind, save=save)
    within(y, *linear64(x, w, None, None, kind, dtype == "bf16")["y"], "y")
    dy = torch.ones_like(y)
    want = linear_backward64(dy, x, w, z if z is not None else y, kind, dtype == "bf16")
    for t, name in zip(P.linear_backward(dy, x, w, z, activation=kind), ("dx", "dw", "db")):
        within(t, *want[name], name)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("odd", [False, True])
@pytest.mark.parametrize("M,D", [(6, 72), (70, 72), (2100, 264)])
@pytest.mark.parametrize("form", [P.SAVE_FULL, P.SAVE_8BIT])
def test_strided_operands_and_untouched_surroundings(dtype, odd, M, D, form):
    """Weights and gradients as views of packed rows (odd: not 16-byte aligned), activations inside wider rows, outputs inside
    sentinels."""
    dt, (K, N) = DT[dtype], (3, 136)
    x, w, b, r, dy, z = _inputs(K, M, D, N, dt, seed=4)
    shift, row = 1 if odd else 8, N * D + N + 64

    def arena():
        a = torch.full((K, row), 1536.0, device="cuda", dtype=dt)
        v = a[:, shift:shift + N * D + N]
        return a, v[:, :N * D].unflatten(1, (N, D)), v[:, N * D:]

    aw, vw, vb = arena()
    vw.copy_(w), vb.copy_(b)
    wide = lambda n: torch.full((K, M, n + 16), 1536.0, device="cuda", dtype=dt)
    inner = lambda t, n: t[:, :, shift:shift + n]
    xb, rb, yb, zb, dyb, dxb = wide(D), wide(N), wide(N), wide(N), wide(N), wide(D)
    inner(xb, D).copy_(x), inner(rb, N).copy_(r), inner(dyb, N).copy_(dy)
    saved, bytes_ = inner(zb, N), None
    if form == P.SAVE_8BIT:
        bytes_ = torch.full((2, K, M, N + 16), 99, device="cuda", dtype=torch.uint8)
        saved = P.Act8(bytes_[0, :, :, shift:shift + N].view(torch.int8), bytes_[1, :, :, shift:shift + (N + 31) // 32], dt)
    _, saved = P.linear_forward(inner(xb, D), vw, vb, inner(rb, N), activation=P.ACT_GELU, save=form, out=inner(yb, N), saved=saved)
    want = linear64(x, w, b, r, P.ACT_GELU, dtype == "bf16")
    within(inner(yb, N), *want["y"], "y")
    check_saved(saved, want["z"], dt, N)
    ag, gw, gb = arena()
    P.linear_backward(inner(dyb, N), inner(xb, D), vw, saved, activation=P.ACT_GELU, out=(inner(dxb, D), gw, gb))
    z = P.act8_unpack(saved, dtype=torch.float32) if bytes_ is not None else saved
    ref = linear_backward64(dy, x, w, z, P.ACT_GELU, dtype == "bf16")
    if bytes_ is not None:
        for t, n in ((bytes_[0], N), (bytes_[1], (N + 31) // 32)):
            assert bool((t[:, :, :shift] == 99).all()) and bool((t[:, :, shift + n:] == 99).all())
    for t, name in zip((inner(dxb, D), gw, gb), ("dx", "dw", "db")):
        within(t, *ref[name], name)
    for t, n in ((xb, D), (rb, N), (yb, N), (zb, N), (dyb, N), (dxb, D)):
        assert bool((t[:, :, :shift] == 1536).all()) and bool((t[:, :, shift + n:] == 1536).all())
    for a in (aw, ag):
        assert bool((a[:, :shift] == 1536).all()) and bool((a[:, shift + N * D + N:] == 1536).all())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("M", [5, 70, 10000])
def test_broadcast_inputs(dtype, M):
    """All workers read one weight, one bias and one input; every token reads one row of the residual."""
    K, D, N = 3, 72, 104
    x, w, b, r, dy, _ = _inputs(1, M, D, N, DT[dtype], seed=6)
    x, w, b, r, dy = x.expand(K, M, D), w.expand(K, N, D), b.expand(K, N), r[:, :1].expand(K, M, N), dy.expand(K, M, N)
    y, _ = P.linear_forward(x, w, b, r)
    within(y, *linear64(x, w, b, r, NONE, dtype == "bf16")["y"], "y")
    want = linear_backward64(dy, x, w, None, NONE, dtype == "bf16")
    for t, name in zip(P.linear_backward(dy, x, w), ("dx", "dw", "db")):
        within(t, *want[name], name)


@pytest.mark.parametrize("M", [33, 600])
def test_what_is_not_asked_for_is_left_out(M):
    x, w, _, _, dy, _ = _inputs(2, M, 40, 48, torch.bfloat16)
    full = P.linear_backward(dy, x, w)
    dx, dw, db = P.linear_backward(dy, x, w, need_dx=False, need_dbias=False)
    assert dx is None and db is None and torch.equal(dw, full[1])
    dx, dw, db = P.linear_backward(dy, x, w, need_dbias=False)
    assert db is None and torch.equal(dw, full[1]) and torch.equal(dx, full[0])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_no_tokens(dtype):
    x, w, b, r, dy, _ = _inputs(2, 0, 40, 48, DT[dtype])
    assert P.linear_forward(x, w, b, r)[0].shape == (2, 0, 48)
    out = torch.full_like(w, 7.0), torch.full_like(b, 7.0)
    dx, dw, db = P.linear_backward(dy, x, w, out=(None, *out))
    assert dx.shape == (2, 0, 40) and not bool(dw.any()) and not bool(db.any())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("M", [4, 50, 12000])
def test_infinities_and_nan_stay_where_they_are(dtype, M):
    """A NaN in one input row reaches that row alone, one in the bias its column, one in the residual its place."""
    x, w, b, r, _, _ = _inputs(1, M, 72, 264, DT[dtype], seed=8)
    x[0, 1, 3], b[0, 7], r[0, 2, 9] = float("nan"), float("inf"), float("-inf")
    y, z = P.linear_forward(x, w, b, r, activation=P.ACT_RELU, save=P.SAVE_8BIT)
    bad = torch.zeros(M, 264, dtype=torch.bool, device="cuda")
    bad[1] = True
    ok = ~bad
    ok[:, 7] = ok[2, 9] = False
    assert bool(y[0][bad].isnan().all()) and bool(y[0][ok].isfinite().all())
    assert float(y[0, 0, 7]) == float("inf") and float(y[0, 2, 9]) == float("-inf")
    v = P.act8_unpack(z, dtype=torch.float32)[0]
    assert bool(v[1].isnan().all()) and bool(v[:, :32].isnan().all()) and bool(v[ok.logical_and(torch.arange(264, device="cuda") >= 32)].isfinite().all())


def test_the_same_call_gives_the_same_bits():
    x, w, b, r, dy, z = _inputs(2, 900, 264, 300, torch.bfloat16, seed=9)
    first = (*P.linear_forward(x, w, b, r, activation=P.ACT_SILU, save=P.SAVE_FULL), *P.linear_backward(dy, x, w, z, activation=P.ACT_SILU))
    for _ in range(3):
        again = (*P.linear_forward(x, w, b, r, activation=P.ACT_SILU, save=P.SAVE_FULL), *P.linear_backward(dy, x, w, z, activation=P.ACT_SILU))
        assert all(torch.equal(a, c) for a, c in zip(first, again))


# several tiles of a pair of CTAs, and as many rows of a CTA before the activation
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("size", [(3, 1500, 264, 1100), (5, 1900, 520, 600)], ids=str)
@pytest.mark.parametrize("save", [P.SAVE_FULL, P.SAVE_8BIT])
def test_several_tiles_of_a_pair(dtype, size, save):
    K, M, D, N = size
    x, w, b, r, dy, _ = _inputs(*size, DT[dtype], seed=11)
    y, saved = P.linear_forward(x, w, b, r, activation=P.ACT_SILU, save=save)
    want = linear64(x, w, b, r, P.ACT_SILU, dtype == "bf16")
    within(y, *want["y"], "y")
    check_saved(saved, want["z"], DT[dtype], N)
    z = saved if save == P.SAVE_FULL else P.act8_unpack(saved, dtype=torch.float32)
    ref = linear_backward64(dy, x, w, z, P.ACT_SILU, dtype == "bf16")
    for t, name in zip(P.linear_backward(dy, x, w, saved, activation=P.ACT_SILU), ("dx", "dw", "db")):
        within(t, *ref[name], name)


@pytest.mark.parametrize("size", [(1, 200, 7600, 2501), (3, 130, 6500, 1001), (1, 70, 4100, 9601), (2, 64, 9000, 1032)], ids=str)
@pytest.mark.parametrize("need_dx", [False, True])
def test_bias_gradients_beside_many_tiles(size, need_dx):
    """Calls whose products take long enough for the sums of dy to run beside them: odd columns, ragged rows, more groups of columns
    than CTAs."""
    K, M, D, N = size
    pad = (N + 7) // 8 * 8 + 8
    dy = torch.full((K, M, pad), float("nan"), dtype=torch.bfloat16, device="cuda")[..., :N]
    gen = torch.Generator(device="cuda").manual_seed(41)
    r = lambda *s, std=1.0: (torch.randn(*s, generator=gen, device="cuda") * std).bfloat16()
    dy.copy_(r(K, M, N))
    x, w = r(K, M, D), r(K, N, D, std=N ** -0.5)
    dx, dw, db = P.linear_backward(dy, x, w, need_dx=need_dx)
    ref = linear_backward64(dy, x, w, None, P.ACT_NONE, True)
    assert (dx is not None) == need_dx
    for a, name in ((dx, "dx"), (dw, "dw"), (db, "db")):
        if a is not None:
            within(a, *ref[name], name)
    assert all(torch.equal(a, b) for a, b in zip((dw, db), P.linear_backward(dy, x, w, need_dx=need_dx)[1:]))
