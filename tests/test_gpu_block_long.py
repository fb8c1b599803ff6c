"""The block operators' persistent loops where each CTA goes round several times: against the 64-bit statements, every row."""
import pytest
import torch

import paper_2504_18454_b200 as P
from _block_ref import U, act64, ffn_backward64, ffn_forward64, qk_backward64, qk_forward64, rounded, within

pytestmark = pytest.mark.gpu
DT = {"fp32": torch.float32, "bf16": torch.bfloat16}


def _qk_inputs(K, M, HQ, HK, DH, R, dt, seed=1, rows=1000):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s, m=0.0, std=1.0: (m + torch.randn(*s, generator=gen, device="cuda") * std).to(dt)
    ang = torch.rand(rows, R // 2, generator=gen, device="cuda", dtype=torch.float64) * 6.3
    pos = torch.randint(0, rows, (K, M), generator=gen, device="cuda", dtype=torch.int32)
    return (r(K, M, HQ, DH), r(K, M, HK, DH, std=3.0), r(K, DH, m=1.0, std=0.2), r(K, DH, m=1.0, std=0.2), ang.cos().float(),
            ang.sin().float(), pos, r(K, M, HQ, DH, std=0.1), r(K, M, HK, DH, std=0.1))


# K, tokens, heads_q, heads_k, head_dim, rotary_dim: two to fifty turns of a warp, the last one short; whole vectors, halves
# that cut vectors, no 16-byte boundaries; 4, 8, 16 and 32 lanes a head, one to eight slots a lane
LONG = [(1, 20011, 3, 1, 64, 64), (1, 70001, 3, 1, 64, 32), (1, 20011, 3, 1, 128, 64), (1, 20011, 3, 1, 64, 20), (1, 9001, 3, 1, 256, 256),
        (1, 20011, 3, 1, 33, 20), (1, 5003, 2, 1, 512, 512), (2, 6007, 1, 3, 512, 36), (1, 3001, 3, 1, 511, 500), (3, 9001, 5, 2, 40, 40)]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("size", LONG, ids=str)
@pytest.mark.parametrize("interleaved", [False, True])
def test_qk_over_several_turns_of_a_warp(dtype, size, interleaved):
    q, k, wq, wk, cos, sin, pos, dq, dk = _qk_inputs(*size, DT[dtype])
    bf = dtype == "bf16"
    got = P.qk_norm_rope(q, k, wq, wk, cos, sin, pos, eps=1e-5, interleaved=interleaved)
    back = P.qk_norm_rope_backward(dq, dk, q, k, wq, wk, cos, sin, pos, eps=1e-5, interleaved=interleaved)
    for i, (x, w, d) in enumerate(((q, wq, dq), (k, wk, dk))):
        within(got[i], *qk_forward64(x, w, pos, cos, sin, 1e-5, interleaved, bf), "qk"[i])
        dx, dw = qk_backward64(d, x, w, pos, cos, sin, 1e-5, interleaved, bf)
        within(back[i], *dx, "dx")
        within(back[2 + i], *dw, "dw")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("size", [s for s in LONG if s[0] == 1], ids=str)
@pytest.mark.parametrize("interleaved", [False, True])
def test_every_head_counts_once_in_the_weight_gradient(dtype, size, interleaved):
    """Whole numbers, which no sum of this length rounds: x = w = cos = 1, sin = 0, and d is 1 in one channel of a head, so
    that dw counts heads.  (Its bound against random numbers would let one head in 60000 be lost.)  bfloat16 holds whole
    numbers to 256: several calls, each with a part of the heads.  (1 / sqrt(1 + 0) may be off by two units in the last
    place: 2^-21 of the count in all.)"""
    _, M, HQ, HK, DH, R = size
    one = lambda *s, v=1.0: torch.full(s, v, device="cuda", dtype=DT[dtype])
    cos, sin = torch.ones(1, R // 2, device="cuda"), torch.zeros(1, R // 2, device="cuda")
    pos = torch.zeros(1, M, device="cuda", dtype=torch.int32)
    N = M * HQ
    parts = -(-N // (DH * 250)) if dtype == "bf16" else 1
    for part in range(parts):
        head = torch.arange(N, device="cuda")
        channel = (head // parts) % DH
        on = head % parts == part
        dq = torch.zeros(N, DH, device="cuda", dtype=DT[dtype])
        dq[head[on], channel[on]] = 1.0
        count = torch.bincount(channel[on], minlength=DH).double()
        assert dtype == "fp32" or int(count.max()) <= 256
        _, _, dw, dwk = P.qk_norm_rope_backward(dq.view(1, M, HQ, DH), one(1, M, HK, DH), one(1, M, HQ, DH), one(1, M, HK, DH), one(1, DH), one(1, DH),
                                                cos, sin, pos, eps=0.0, interleaved=interleaved)
        within(dw[0], count, 2.0 ** -21 * count if dtype == "fp32" else 0.0, "dw")
        if dtype == "fp32":
            within(dwk[0], torch.full_like(count, float(M * HK)), 2.0 ** -21 * M * HK, "dw_k")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_qk_offsets_beyond_32_bits(dtype):
    """Workers and tokens far apart in one long buffer: offsets of 2^31 elements and more, read and written."""
    K, M, H, DH, far = 2, 5, 2, 64, 2 ** 29 + 8
    q, k, wq, wk, cos, sin, pos, dq, dk = _qk_inputs(K, M, H, H, DH, DH, DT[dtype])

    def spread():
        flat = torch.empty((M - 1) * far + 4 * H * DH * K, device="cuda", dtype=DT[dtype])
        view = lambda o: flat.as_strided((K, M, H, DH), (2 * H * DH, far, DH, 1), o)
        return view(0), view(H * DH)

    a, out = spread(), spread()
    a[0].copy_(q), a[1].copy_(k)
    P.qk_norm_rope(*a, wq, wk, cos, sin, pos, out=out)
    for t, x, w in zip(out, (q, k), (wq, wk)):
        within(t, *qk_forward64(x, w, pos, cos, sin, 1e-6, False, dtype == "bf16"), "out")
    P.qk_norm_rope_backward(dq, dk, *a, wq, wk, cos, sin, pos, out=(*out, None, None))
    for t, x, w, d in zip(out, (q, k), (wq, wk), (dq, dk)):
        within(t, *qk_backward64(d, x, w, pos, cos, sin, 1e-6, False, dtype == "bf16")[0], "dx")


# K, tokens, d_model, d_ff: tiles of the gate/up, hidden, second and backward products: 162, 90, 36, 126; 54, 36, 90, 162; 240, 120, 120, 285
TILES = [(3, 1500, 264, 1100), (3, 1500, 1100, 264), (5, 1900, 520, 600)]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("size", TILES, ids=str)
@pytest.mark.parametrize("save", [P.SAVE_FULL, P.SAVE_8BIT])
def test_ffn_over_several_tiles_of_a_pair(dtype, size, save):
    K, M, D, F = size
    gen = torch.Generator(device="cuda").manual_seed(21)
    r = lambda *s, std: (torch.randn(*s, generator=gen, device="cuda") * std).to(DT[dtype])
    x, wg, wu, wd, dy = r(K, M, D, std=1.0), r(K, F, D, std=D ** -0.5), r(K, F, D, std=D ** -0.5), r(K, D, F, std=F ** -0.5), r(K, M, D, std=0.01)
    y, saved = P.ffn_forward(x, wg, wu, wd, save=save)
    want = ffn_forward64(x, wg, wu, wd, 0, dtype == "bf16")
    within(y, *want["y"], "y")
    if save == P.SAVE_FULL:
        g, u = saved
        for t, name in zip(saved, ("gate", "up")):
            within(t, want[name][0], rounded(*want[name], dtype == "bf16"), name)
    else:
        g, u = (P.act8_unpack(a, dtype=torch.float32) for a in saved)
        for t, a, name in zip((g, u), saved, ("gate", "up")):
            step = torch.exp2(a.exponent.double() - 127).repeat_interleave(32, -1)[..., :F]
            within(t, want[name][0], step / 2 + want[name][1], name)
    got = P.ffn_backward(dy, x, wg, wu, wd, saved)
    ref = ffn_backward64(dy, x, wg, wu, wd, g, u, 0, dtype == "bf16")
    for t, name in zip(got, ("dx", "dw_gate", "dw_up", "dw_down")):
        within(t, *ref[name], name)


def test_fp32_sums_are_rounded_to_nearest_along_the_way():
    """4096 terms: the tensor cores cut off what an addition does not hold, 4.4e-6 of the result's norm if nothing is done
    about it; with a rounding to nearest every 256 terms it stays below 1e-6 (half a unit in the last place is 6e-8)."""
    K, M, D, F = 1, 300, 4096, 264
    gen = torch.Generator(device="cuda").manual_seed(22)
    r = lambda *s, std: torch.randn(*s, generator=gen, device="cuda") * std
    x, wg, wu, wd = r(K, M, D, std=1.0), r(K, F, D, std=D ** -0.5), r(K, F, D, std=D ** -0.5), r(K, D, F, std=F ** -0.5)
    _, saved = P.ffn_forward(x, wg, wu, wd)
    for t, w in zip(saved, (wg, wu)):
        want = x.double() @ w.double().mT
        assert float((t.double() - want).norm() / want.norm()) < 1e-6


@pytest.mark.parametrize("kind", range(4))
def test_fp32_activations_to_a_few_roundings(kind):
    """One inner element, weights 1: g = u = x exactly.  The logistic (exponential to 2 units, sum, quotient) or erf is off by
    at most 2^-21, and act by |g| times that; the product with u and the split into three parts round twice more.  The slopes
    have the same error times the factor of their tail: |g|, for the tanh form 1.6 |g| (1 + 0.135 g^2)."""
    x = torch.cat([torch.linspace(-8, 8, 4001), torch.zeros(1)]).cuda()[None, :, None]
    one = torch.ones(1, 1, 1, device="cuda")
    y, saved = P.ffn_forward(x, one, one, one, activation=kind)
    g = x.double()
    a, slope = act64(kind, g)
    within(y, a * g, (2.0 ** -21 * (1 + g.abs()) + 2 * U * a.abs()) * g.abs().clamp_min(1), "y")
    dx, *_ = P.ffn_backward(torch.ones_like(x), torch.ones_like(x), one, torch.zeros_like(one), one, (x, torch.ones_like(x)), activation=kind)
    tail = g.abs() * (1.6 * (1 + 0.135 * g * g) if kind == 2 else 1.0)
    within(dx, slope, 2.0 ** -21 * (1 + tail), "act'")
