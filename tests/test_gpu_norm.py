"""The layer norm against its 64-bit statement: types, widths of every team of warps, odd widths, strides, residuals, edges."""
import pytest
import torch

import paper_2504_18454_b200 as P
from _block_ref import within
from _more_ref import norm64, norm_backward64

pytestmark = pytest.mark.gpu
DT = {"fp32": torch.float32, "bf16": torch.bfloat16}
# K, tokens, width: one value; less than a piece; every count of pieces a lane and of warps a team, up to the widest; a last
# turn of a team that some teams do not have; many workers
SIZES = [(1, 1, 1), (2, 3, 5), (3, 77, 257), (1, 9, 256), (2, 40, 512), (1, 33, 768), (2, 2500, 72), (1, 700, 1000), (2, 5, 1023), (1, 70, 2048),
         (1, 21, 3001), (2, 9, 4096), (1, 5, 6002), (1, 3, 8192), (1, 4, 8200), (1, 3, 12000), (2, 2, 16384), (1, 2, 16383), (64, 3, 64)]


def _inputs(K, M, D, dt, seed=1):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s, std=1.0, m=0.0: (m + torch.randn(*s, generator=gen, device="cuda") * std).to(dt)
    return r(K, M, D, std=1.5, m=0.7), r(K, M, D, std=0.8), r(K, D, m=1.0, std=0.2), r(K, D, std=0.3), r(K, M, D, std=0.01), r(K, M, D, std=0.01)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("add", [False, True])
def test_forward_and_backward(dtype, size, add):
    bf, (x, r, w, b, dy, dt) = dtype == "bf16", _inputs(*size, DT[dtype])
    residual, past = (r, dt) if add else (None, None)
    y, total, mean, rstd = P.layer_norm_forward(x, w, b, residual, eps=1e-5)
    want = norm64(x, residual, w, b, 1e-5, bf)
    for t, name in ((y, "y"), (mean, "mean"), (rstd, "rstd")):
        within(t, *want[name], name)
    if add:
        within(total, *want["total"], "total")
    else:
        assert total is x
    got = P.layer_norm_backward(dy, total, w, mean, rstd, past)
    ref = norm_backward64(dy, total, w, mean, rstd, past, bf)
    for t, name in zip(got, ("dx", "dw", "db")):
        within(t, *ref[name], name)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("odd", [False, True])
@pytest.mark.parametrize("D", [96, 1031])
def test_strided_operands_and_untouched_surroundings(dtype, odd, D):
    dt, (K, M) = DT[dtype], (3, 50)
    x, r, w, b, dy, past = _inputs(K, M, D, dt, seed=4)
    shift = 1 if odd else 8
    wide = lambda: torch.full((K, M, D + 16 + D % 2), 1536.0, device="cuda", dtype=dt)
    inner = lambda t: t[:, :, shift:shift + D]
    vec = lambda: torch.full((K, D + 16), 1536.0, device="cuda", dtype=dt)
    cut = lambda t: t[:, shift:shift + D]
    xb, rb, yb, tb, dyb, pb, dxb = (wide() for _ in range(7))
    wb, bb, dwb, dbb = (vec() for _ in range(4))
    for to, t in ((xb, x), (rb, r), (dyb, dy), (pb, past)):
        inner(to).copy_(t)
    cut(wb).copy_(w), cut(bb).copy_(b)
    stats = torch.full((2, K, M + 2), 1536.0, device="cuda")
    mean, rstd = stats[0, :, 1:M + 1], stats[1, :, 1:M + 1]
    P.layer_norm_forward(inner(xb), cut(wb), cut(bb), inner(rb), eps=1e-6, out=(inner(yb), inner(tb), mean, rstd))
    want = norm64(x, r, w, b, 1e-6, dtype == "bf16")
    for t, name in ((inner(yb), "y"), (inner(tb), "total"), (mean, "mean"), (rstd, "rstd")):
        within(t, *want[name], name)
    P.layer_norm_backward(inner(dyb), inner(tb), cut(wb), mean, rstd, inner(pb), out=(inner(dxb), cut(dwb), cut(dbb)))
    ref = norm_backward64(dy, inner(tb), w, mean, rstd, past, dtype == "bf16")
    for t, name in ((inner(dxb), "dx"), (cut(dwb), "dw"), (cut(dbb), "db")):
        within(t, *ref[name], name)
    for t in (xb, rb, yb, tb, dyb, pb, dxb, wb, bb, dwb, dbb):
        assert bool((t[..., :shift] == 1536).all()) and bool((t[..., shift + D:] == 1536).all())
    assert bool((stats[..., 0] == 1536).all()) and bool((stats[..., -1] == 1536).all())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_broadcast_inputs(dtype):
    K, M, D = 3, 40, 136
    x, r, w, b, dy, _ = _inputs(1, M, D, DT[dtype], seed=5)
    x, r, w, b, dy = x.expand(K, M, D), r[:, :1].expand(K, M, D), w.expand(K, D), b.expand(K, D), dy[:, :1].expand(K, M, D)
    y, total, mean, rstd = P.layer_norm_forward(x, w, b, r)
    want = norm64(x, r, w, b, 1e-5, dtype == "bf16")
    within(y, *want["y"], "y")
    ref = norm_backward64(dy, total, w, mean, rstd, dy, dtype == "bf16")
    for t, name in zip(P.layer_norm_backward(dy, total, w, mean, rstd, dy), ("dx", "dw", "db")):
        within(t, *ref[name], name)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_a_mean_that_is_large_against_the_spread(dtype):
    """Rows around 1000 with a spread of 1: the squares' own mean would lose the variance."""
    x, _, w, b, _, _ = _inputs(1, 30, 768, torch.float32, seed=6)
    x = (1000 + x).to(DT[dtype])
    y, _, mean, rstd = P.layer_norm_forward(x, w.to(x.dtype), b.to(x.dtype))
    want = norm64(x, None, w.to(x.dtype), b.to(x.dtype), 1e-5, dtype == "bf16")
    for t, name in ((y, "y"), (mean, "mean"), (rstd, "rstd")):
        within(t, *want[name], name)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_rows_of_one_value_infinities_and_nan(dtype):
    """A row without spread: rstd = 1 / sqrt(eps), y = b; a NaN or an infinity spoils its own row only."""
    x, _, w, b, dy, _ = _inputs(1, 8, 264, DT[dtype], seed=7)
    x[0, 0], x[0, 1, 5], x[0, 2, 6] = 3.0, float("nan"), float("inf")
    y, _, mean, rstd = P.layer_norm_forward(x, w, b, eps=1e-4)
    assert torch.equal(y[0, 0], b[0]) and float(mean[0, 0]) == 3.0 and abs(float(rstd[0, 0]) - 100.0) < 1e-3
    assert bool(y[0, 1:3].isnan().all()) and bool(y[0, 3:].isfinite().all())
    dx, dw, db = P.layer_norm_backward(dy, x, w, mean, rstd)
    assert bool(dx[0, 1].isnan().all()) and bool(dx[0, 0].isfinite().all()) and bool(dx[0, 3:].isfinite().all())
    assert bool(dw.isnan().all()) and bool(db.isfinite().all())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_no_tokens(dtype):
    x, _, w, b, dy, _ = _inputs(2, 0, 40, DT[dtype])
    y, total, mean, rstd = P.layer_norm_forward(x, w, b)
    assert y.shape == (2, 0, 40) and mean.shape == (2, 0)
    out = torch.full_like(w, 7.0), torch.full_like(b, 7.0)
    _, dw, db = P.layer_norm_backward(dy, x, w, mean, rstd, out=(None, *out))
    assert not bool(dw.any()) and not bool(db.any())


def test_without_statistics():
    x, r, w, b, _, _ = _inputs(2, 7, 40, torch.float32)
    y, _, mean, rstd = P.layer_norm_forward(x, w, b, r, stats=False)
    assert mean is None and rstd is None and torch.equal(y, P.layer_norm_forward(x, w, b, r)[0])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("D", [64, 1000])
def test_every_row_counts_once_in_the_weight_gradients(dtype, D):
    """Whole numbers that nothing rounds: dy is 1 in one channel of a row, xh is 1."""
    M = 100 * D + 37 if D == 64 else 20011
    x, mean, rstd = torch.ones(1, M, D, device="cuda", dtype=DT[dtype]), torch.zeros(1, M, device="cuda"), torch.ones(1, M, device="cuda")
    channel = torch.arange(M, device="cuda") % D
    dy = torch.zeros(1, M, D, device="cuda", dtype=DT[dtype])
    dy[0, torch.arange(M, device="cuda"), channel] = 1.0
    _, dw, db = P.layer_norm_backward(dy, x, torch.ones(1, D, device="cuda", dtype=DT[dtype]), mean, rstd)
    count = torch.bincount(channel, minlength=D).float()
    assert int(count.max()) <= 256                         # (bfloat16 holds whole numbers to 256)
    assert torch.equal(dw[0].float(), count) and torch.equal(db[0].float(), count)


def test_the_same_call_gives_the_same_bits():
    x, r, w, b, dy, _ = _inputs(2, 3000, 520, torch.float32, seed=9)
    first = None
    for _ in range(3):
        y, total, mean, rstd = P.layer_norm_forward(x, w, b, r)
        now = (y, mean, rstd, *P.layer_norm_backward(dy, total, w, mean, rstd))
        assert first is None or all(torch.equal(a, c) for a, c in zip(first, now))
        first = now
