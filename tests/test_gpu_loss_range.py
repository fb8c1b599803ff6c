"""The gradient of the cross entropy over the whole range of its logits: rows of a dominant logit of any size, rows of nothing but
the type's lowest or largest value."""
import pytest
import torch

import paper_2504_18454_b200 as P
from _block_ref import BF, U, within

pytestmark = pytest.mark.gpu
DT = {"fp32": torch.float32, "bf16": torch.bfloat16}


def gradient64(d, z, t, lse, dt):
    """(e^(z - lse) - [t]) d at the given lse, and a bound on its evaluation: the difference is rounded once or twice and its product with
    log2(e) once (the constant itself to half as much), each a relative error of the exponential of U / 2 times |z - lse|; the
    exponential is off by 2^-21 of itself, 1 is taken off, d multiplied, and the result rounded."""
    z, lse, d = z.double(), lse.double()[..., None], d.double()[..., None]
    p = torch.exp(z - lse)
    hot = torch.zeros_like(z).scatter_(-1, t.long()[..., None], 1.0)
    e = d.abs() * (p * (2 * U * torch.where(p > 0, z - lse, 0.0).abs() + 2.0 ** -21) + 2 * U * (p + hot)) + 2.0 ** -126
    v = (p - hot) * d
    return v, e + (BF if dt == torch.bfloat16 else U) * (v.abs() + e)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("V", [3, 70, 5000])
def test_a_dominant_logit_of_any_size(dtype, V):
    """z_t = lse up to the type's largest value: the gradient is zero, and it is d where another row's target is elsewhere."""
    dt = DT[dtype]
    sizes = [s * m for m in (1e3, 1e4, 1.23e5, 1e6, 3.3e7, 1e8, 1e12, 1e30, 2.5e38, torch.finfo(dt).max) for s in (1, -1)]
    gen = torch.Generator(device="cuda").manual_seed(2)
    z = torch.empty(1, 2 * len(sizes), V, device="cuda", dtype=dt)
    for i, m in enumerate(sizes):                          # below a negative one, the others are lower still
        z[0, 2 * i:2 * i + 2] = -torch.finfo(dt).max if m < 0 else torch.randn(2, V, generator=gen, device="cuda").to(dt)
        z[0, 2 * i:2 * i + 2, 1] = min(max(m, -torch.finfo(dt).max * 0.99), torch.finfo(dt).max)
    t = torch.ones(1, z.shape[1], device="cuda", dtype=torch.int32)
    t[:, 1::2] = 2
    d = torch.randn(1, z.shape[1], generator=gen, device="cuda")
    loss, lse = P.cross_entropy_forward(z, t)
    top = z.amax(-1).float()                               # (the others add less than half a rounding of it)
    assert torch.equal(lse, top) and not bool(loss[:, ::2].any())
    for out in (None, z.clone()):
        if out is None:
            g = P.cross_entropy_backward(d, z, t, lse)
        else:
            g = P.cross_entropy_backward(d, out, t, lse, out=out)
        within(g, *gradient64(d, z, t, lse, dt), "dlogits")
        assert not bool(g[:, ::2, 1].any())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("V", [1, 70, 5000])
def test_rows_of_nothing_but_the_lowest_or_largest_value(dtype, V):
    """A mask that leaves nothing, of the type's lowest value: the target counts, so the loss is log V and the gradient finite."""
    lim = torch.finfo(DT[dtype])
    z = torch.empty(1, 4, V, device="cuda", dtype=DT[dtype])
    z[:, :2], z[:, 2:] = lim.min, lim.max
    t = torch.zeros(1, 4, device="cuda", dtype=torch.int32)
    d = torch.tensor([[0.5, 0.0, -2.0, 0.0]], device="cuda")
    loss, lse = P.cross_entropy_forward(z, t)
    assert torch.allclose(loss, torch.tensor(float(V), device="cuda").log(), rtol=1e-6, atol=1e-6)
    g = P.cross_entropy_backward(d, z, t, lse)
    assert bool((g.abs() <= d.abs()[..., None]).all())
    assert not bool(g[0, 1].any()) and not bool(g[0, 3].any())


def softmax_gradient64(d, z, t, dt):
    """(softmax(z) - [t]) d, and its bound: the sum of e^(z - largest) is off as lse is in loss64 -- the arguments by two roundings each, the
    exponential by 2^-21, a lane's share of the terms and a few dozen partial sums -- and the exponent by two roundings more, of z - largest
    and of what is left of lse behind it."""
    z, d = z.double(), d.double()[..., None]
    top = z.amax(-1, keepdim=True)
    rest = torch.logsumexp(z - top, -1, keepdim=True)
    p = torch.exp(z - top - rest)
    away = torch.where(p > 0, top - z, 0.0)
    e_sum = (p * 2 * U * away).sum(-1, keepdim=True) + 2.0 ** -21 + (z.shape[-1] / 32 + 64) * U
    hot = torch.zeros_like(z).scatter_(-1, t.long()[..., None], 1.0)
    e = d.abs() * (p * (2 * U * (away + rest) + e_sum + 2.0 ** -21) + 2 * U * (p + hot)) + 2.0 ** -126
    v = (p - hot) * d
    return v, e + (BF if dt == torch.bfloat16 else U) * (v.abs() + e)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("V", [1, 2, 70, 300, 5000, 50257])
@pytest.mark.parametrize("how", ["new", "in place", "unalike"])
def test_rows_far_from_zero_have_the_gradient_of_their_softmax(dtype, V, how):
    """lse holds nothing of the sum where all logits are the type's lowest value, and little of it where they share a large part."""
    dt = DT[dtype]
    lim = torch.finfo(dt)
    at = [lim.min, lim.max, 1e5, -1e5, 4096.0, -3.3e7, 1e30, 1030.0, -1023.0, 0.0]
    gen = torch.Generator(device="cuda").manual_seed(7)
    z = (torch.randn(1, 2 * len(at), V, generator=gen, device="cuda") * 3)
    for i, m in enumerate(at):
        z[0, 2 * i] = m                                    # all alike
        z[0, 2 * i + 1] += m                               # (beyond some size the addend is lost: alike too)
    z = z.to(dt)
    t = torch.randint(0, V, z.shape[:2], generator=gen, device="cuda", dtype=torch.int32)
    d = torch.randn(*z.shape[:2], generator=gen, device="cuda")
    loss, lse = P.cross_entropy_forward(z, t)
    assert bool(loss.isfinite().all())
    want = softmax_gradient64(d, z, t, dt)
    near = lse.abs() < 1024                                # (at the lse given, which is off by half a rounding more)
    extra = (want[0] + d[..., None] * torch.zeros_like(z).scatter_(-1, t.long()[..., None], 1.0)).abs() * U * lse[..., None].abs()
    want = want[0], want[1] + torch.where(near[..., None], extra * (1 + (BF if dt == torch.bfloat16 else U)), 0.0)
    if how == "new":
        g = P.cross_entropy_backward(d, z, t, lse)
    elif how == "in place":
        g = P.cross_entropy_backward(d, z, t, lse, out=z)
    else:
        g = torch.full((1, z.shape[1], V + 9), 7.0, device="cuda", dtype=dt)[:, :, 3:3 + V]
        P.cross_entropy_backward(d, z, t, lse, out=g)
    within(g, *want, "dlogits")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("V", [70, 5000, 50257])
def test_an_lse_that_is_not_the_rows_own_is_taken_as_given(dtype, V):
    """As where a vocabulary is shared out: the row's part of a larger sum."""
    dt = DT[dtype]
    gen = torch.Generator(device="cuda").manual_seed(9)
    z = (2e4 + 200 * torch.randn(2, 9, V, generator=gen, device="cuda")).to(dt)
    t = torch.randint(0, V, (2, 9), generator=gen, device="cuda", dtype=torch.int32)
    d = torch.randn(2, 9, generator=gen, device="cuda")
    _, lse = P.cross_entropy_forward(z, t)
    for more in (0.5, 3.0, 100.0):
        within(P.cross_entropy_backward(d, z, t, lse + more), *gradient64(d, z, t, lse + more, dt), "dlogits")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_far_rows_among_others(dtype):
    """Rows that do not count, rows that are not numbers and near rows keep what they have beside far ones; the same bits each time."""
    dt, V = DT[dtype], 50257
    gen = torch.Generator(device="cuda").manual_seed(11)
    z = torch.randn(3, 40, V, generator=gen, device="cuda")
    z[:, ::3] += 1e6
    z = z.to(dt)
    z[:, 3, 17], z[:, 4, 5], z[:, 6] = float("nan"), float("inf"), -float("inf")
    t = torch.randint(0, V, (3, 40), generator=gen, device="cuda", dtype=torch.int32)
    t[:, 9], t[:, 12] = -1, V
    d = torch.randn(3, 40, generator=gen, device="cuda")
    _, lse = P.cross_entropy_forward(z, t)
    g = P.cross_entropy_backward(d, z, t, lse)
    assert all(bool(g[:, i].isnan().all()) for i in (3, 4, 6, 12)) and not bool(g[:, 9].any())
    rows = [0, 1, 2, 5, 7, 8, 10, 11, *range(13, 40)]
    for far in (True, False):
        r = [i for i in rows if (i % 3 == 0) == far]
        args = d[:, r], z[:, r], t[:, r]
        within(g[:, r], *(softmax_gradient64(*args, dt) if far else gradient64(*args, lse[:, r], dt)), "dlogits")
    assert torch.equal(P.cross_entropy_backward(d, z, t, lse).nan_to_num(), g.nan_to_num())
