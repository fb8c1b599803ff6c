"""The cross entropy against its 64-bit statement: types, vocabularies from one value on, odd ones, strides, masked logits, targets
that do not count, work in place."""
import math

import pytest
import torch

import paper_2504_18454_b200 as P
from _block_ref import within
from _more_ref import loss64, loss_backward64

pytestmark = pytest.mark.gpu
DT = {"fp32": torch.float32, "bf16": torch.bfloat16}
INF = float("inf")
# K, tokens, vocabulary: few and many rows, a warp's and a CTA's, every size of a team, several parts of a row
SIZES = [(1, 1, 1), (2, 3, 2), (3, 9, 7), (1, 700, 64), (2, 33, 255), (1, 5, 1000), (2, 400, 1031), (1, 3, 8192), (1, 900, 2049), (1, 2, 50257), (2, 700, 4099),
         (1, 610, 16411), (64, 2, 40)]


def _inputs(K, M, V, dt, seed=1):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    z = (torch.randn(K, M, V, generator=gen, device="cuda") * 3).to(dt)
    t = torch.randint(0, V, (K, M), generator=gen, device="cuda", dtype=torch.int32)
    t[torch.rand(K, M, generator=gen, device="cuda") < 0.15] = -1
    return z, t, torch.randn(K, M, generator=gen, device="cuda")


def check(z, t, d, bf):
    loss, lse = P.cross_entropy_forward(z, t)
    want, want_lse = loss64(z, t)
    within(loss, *want, "loss")
    within(lse, *want_lse, "lse")
    within(P.cross_entropy_backward(d, z, t, lse), *loss_backward64(d, z, t, lse, bf), "dlogits")
    return loss, lse


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_forward_and_backward(dtype, size):
    check(*_inputs(*size, DT[dtype]), dtype == "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("V", [40, 3001])
@pytest.mark.parametrize("offsets", [(8, 8), (1, 1), (3, 8), (2, 5)])
def test_rows_anywhere_and_untouched_surroundings(dtype, V, offsets):
    """The logits and their gradients inside wider rows, starting alike and not."""
    K, M = 2, 21
    z, t, d = _inputs(K, M, V, DT[dtype], seed=3)
    box = lambda: torch.full((K, M, V + 16), 1536.0, device="cuda", dtype=DT[dtype])
    zb, gb = box(), box()
    zi, gi = zb[:, :, offsets[0]:offsets[0] + V], gb[:, :, offsets[1]:offsets[1] + V]
    zi.copy_(z)
    loss, lse = P.cross_entropy_forward(zi, t)
    within(loss, *loss64(z, t)[0], "loss")
    P.cross_entropy_backward(d, zi, t, lse, out=gi)
    within(gi, *loss_backward64(d, z, t, lse, dtype == "bf16"), "dlogits")
    for b, o in ((zb, offsets[0]), (gb, offsets[1])):
        assert bool((b[:, :, :o] == 1536).all()) and bool((b[:, :, o + V:] == 1536).all())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("V", [50257, 129])
def test_work_in_place(dtype, V):
    z, t, d = _inputs(2, 60, V, DT[dtype], seed=4)
    _, lse = P.cross_entropy_forward(z, t)
    want = P.cross_entropy_backward(d, z, t, lse)
    got = P.cross_entropy_backward(d, z, t, lse, out=z)
    assert got is z or got.data_ptr() == z.data_ptr()
    assert torch.equal(z, want)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("V", [70, 5000])
def test_masked_logits(dtype, V):
    """Most of a vocabulary masked by -infinity or the type's lowest value, in whole pieces and in parts of them."""
    z, t, d = _inputs(2, 30, V, DT[dtype], seed=5)
    keep = torch.rand(2, 30, V, device="cuda") < 0.2
    keep[:, :, V // 2:] = False
    keep[:, :5] = False
    keep.scatter_(-1, t.long().clamp_min(0)[..., None], True)
    for low in (-INF, torch.finfo(DT[dtype]).min):
        check(torch.where(keep, z, torch.tensor(low, device="cuda", dtype=z.dtype)), t, d, dtype == "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("V", [70, 5000])
def test_rows_that_are_not_numbers(dtype, V):
    z, t, d = _inputs(1, 9, V, DT[dtype], seed=6)
    t[:] = 2
    z[0, 0] = -INF                                        # nothing above -infinity
    z[0, 1, 30] = float("nan")
    z[0, 2, 31] = INF
    z[0, 3, 2] = -INF                                     # the target's own
    z[0, 4], t[0, 4] = float("nan"), -1                   # does not count
    t[0, 5] = V                                           # beyond the vocabulary
    t[0, 6] = 2 ** 31 - 1
    z[0, 7] = z[0, 7] * 0 + 1e4                           # large and equal
    loss, lse = P.cross_entropy_forward(z, t)
    g = P.cross_entropy_backward(d, z, t, lse)
    nan = [bool(v) for v in loss[0].isnan()]
    assert nan == [True, True, True, False, False, True, True, False, False], nan
    assert float(lse[0, 0]) == -INF and bool(lse[0, 1:3].isnan().all())
    assert float(loss[0, 3]) == INF and float(loss[0, 4]) == 0.0
    # log V, to the rounding of lse's parts at 10^4 (none: the difference is taken of equal values)
    assert abs(float(loss[0, 7]) - math.log(V)) < 1e-4
    assert bool(g[0, 0].isnan().all()) and bool(g[0, 1].isnan().all()) and bool(g[0, 5:7].isnan().all())
    assert bool(g[0, 3].isfinite().all()) and not bool(g[0, 4].any())
    rest = slice(8, None)                                 # (the statement indexes with its targets: those inside only)
    within(g[:, rest], *loss_backward64(d[:, rest], z[:, rest], t[:, rest], lse[:, rest], dtype == "bf16"), "dlogits")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_one_row_of_targets_for_all_workers(dtype):
    z, t, d = _inputs(3, 20, 300, DT[dtype], seed=7)
    check(z, t[:1].expand(3, 20), d, dtype == "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_a_confident_row_keeps_its_small_loss(dtype):
    """loss = log(1 + (V - 1) e^-9), far below the rounding of lse = 100: formed from the sum, not from lse - z."""
    V = 64
    z = torch.full((1, 2, V), 91.0, device="cuda", dtype=DT[dtype])
    z[..., 5] = 100.0
    loss, _ = P.cross_entropy_forward(z, torch.full((1, 2), 5, device="cuda", dtype=torch.int32))
    want = math.log1p((V - 1) * math.exp(-9.0))
    assert abs(float(loss[0, 0]) - want) < 2.0 ** -20      # the sum near 1 is rounded a few times

def test_no_tokens():
    z, t, d = _inputs(2, 0, 50, torch.bfloat16)
    loss, lse = P.cross_entropy_forward(z, t)
    assert loss.shape == lse.shape == (2, 0) and P.cross_entropy_backward(d, z, t, lse).shape == z.shape
