"""The linear operator's activations and their slopes against the bound that the C header states, 2^-21 (1 + |z|) before the result is
rounded, by the kernels of few tokens and of whole tiles.

The bound, with u = 2^-24 one rounding of a binary32 value below 1: a logistic function's argument y is off by up to 5 u of itself and its
exponential by 4 u more, so s by s (1 - s) (5 |y| + 4) u <= 2.5 u, and z s and the slope's second term stay within 4 u (1 + |z|).  erf(z / sqrt 2)
to two units is 2 u of Phi.  The rational form of erf is off by 1.5e-7, 1.3 u of Phi; its Horner steps by 4 u times t e^(-z^2 / 2) / 2 <= 1 / 2, the
reciprocal t by 3 u and the exponential by 4 u and two roundings of z^2, of which Phi(-|z|) <= 1 / 2 leaves 4 u: 7.2 u <= 8 u (1 + |z|); the
slope's z phi(z) <= 0.25 adds 2 u where 8 u |z| are left for it.  The Chebyshev form is off by 2 u of Phi(-|z|), its polynomial by 4 u and its
exponent E by 3 u |E|, of which E e^E <= 0.37 leaves 1 u: less again."""
import pytest
import torch

import paper_2504_18454_b200 as P
from _block_ref import BF, U, act64, within

pytestmark = pytest.mark.gpu
DT = {"fp32": torch.float32, "bf16": torch.bfloat16}
KINDS = [P.ACT_SILU, P.ACT_GELU, P.ACT_GELU_TANH, P.ACT_RELU]
BOUND = 2.0 ** -21


def _values(dt):
    if dt == torch.bfloat16:                               # every one up to 64, and the tiny
        z = torch.arange(0x4280, device="cuda", dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
        return torch.cat((z, -z))
    gen = torch.Generator(device="cuda").manual_seed(5)
    z = torch.rand(60000, generator=gen, device="cuda", dtype=torch.float64)
    return torch.cat((z[:40000] * 14 - 7, z[40000:50000] * 60 - 30, torch.exp(z[50000:] * 80 - 75) * (1 - 2 * (z[50000:] < 0.5).double()))).float()


def _expected(got, value, z, dt, what):
    e = BOUND * (1 + z.double().abs())
    within(got, value, e + (BF if dt == torch.bfloat16 else U) * (value.abs() + e) + 2.0 ** -126, what)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("tokens", [60000, 70000])          # by the kernel of few tokens, by the matrix kernel
def test_values(dtype, kind, tokens):
    dt = DT[dtype]
    z = _values(dt).repeat(3)[:tokens]
    one = torch.ones(1, 1, 1, device="cuda", dtype=dt)
    y, kept = P.linear_forward(z.view(1, -1, 1), one, activation=kind, save=P.SAVE_FULL)
    within(kept[0, :, 0], z.double(), 2 * U * z.double().abs(), "z")
    _expected(y[0, :, 0], act64(kind, kept[0, :, 0])[0], z, dt, "y")


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("tokens", [1, 60000])              # by the kernel of few tokens, by the pass before the matrix kernel
def test_slopes(dtype, kind, tokens):
    dt = DT[dtype]
    z = _values(dt)[:60000]
    one = torch.ones(1, 1, 1, device="cuda", dtype=dt)
    if tokens == 1:                                        # dw = dz x
        n = z.numel()
        _, slope, _ = P.linear_backward(one.expand(1, 1, n).contiguous(), one, one.expand(1, n, 1).contiguous(), z.view(1, 1, n), activation=kind)
        slope = slope[0, :, 0]
    else:                                                  # dx = dz w
        slope, _, _ = P.linear_backward(one.expand(1, z.numel(), 1).contiguous(), one.expand(1, z.numel(), 1).contiguous(), one, z.view(1, -1, 1), activation=kind)
        slope = slope[0, :, 0]
    _expected(slope, act64(kind, z)[1], z, dt, "slope")
