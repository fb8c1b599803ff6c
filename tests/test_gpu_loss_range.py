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
