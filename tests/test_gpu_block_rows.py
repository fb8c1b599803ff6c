"""8-bit checkpoints (exact against a 64-bit statement) and the q/k norm with rotation (against its 64-bit statement)."""
import numpy as np
import pytest
import torch

import paper_2504_18454_b200 as P
from _block_ref import act8_numpy, qk_backward64, qk_forward64, within

pytestmark = pytest.mark.gpu
DT = {"fp32": torch.float32, "bf16": torch.bfloat16}


# ---------------------------------------------------------------------------------------------- 8-bit checkpoints

@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("shape", [(1, 1), (1, 7), (3, 31), (5, 32), (4, 33), (2, 40), (37, 257), (9, 256), (130, 72), (0, 64), (3, 1000)], ids=str)
def test_pack_and_unpack_are_exact(dtype, shape):
    gen = torch.Generator(device="cuda").manual_seed(shape[1])
    x = (torch.randn(shape, generator=gen, device="cuda") * torch.exp(4 * torch.randn(shape[0], 1, generator=gen, device="cuda"))).to(DT[dtype])
    a = P.act8_pack(x)
    q, e, v = act8_numpy(x.float().cpu().numpy())
    assert np.array_equal(a.q.cpu().numpy(), q) and np.array_equal(a.exponent.cpu().numpy(), e)
    for out in (torch.bfloat16, torch.float32):
        assert np.array_equal(P.act8_unpack(a, dtype=out).double().cpu().numpy(), v)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("cols", [64, 65])
def test_edges_of_the_number_range(dtype, cols):
    big = torch.finfo(DT[dtype]).max
    rows = [[0.0], [-0.0, 0.0], [float("inf"), 1.0], [float("-inf")], [float("nan"), 2.0], [big, -big, 1.0],
            [127.0, 126.5, 0.5, 1.5, -2.5], [127.5, 1.0, 3.0], [127.25, 1.0], [255.0, 63.0], [1e-30, 3e-31], [1e-38, 1e-39],
            [1.2e-38, 5e-39, -1e-40], [2.0 ** -120, 2.0 ** -127], [1.0, 2.0 ** -7, 2.0 ** -8, 3 * 2.0 ** -8]]
    x = torch.zeros(len(rows), cols)
    for i, r in enumerate(rows):
        x[i, :len(r)] = torch.tensor(r, dtype=torch.float64).to(torch.float32)
        x[i, 40:40 + len(r)] = x[i, :len(r)]
    x = x.to(DT[dtype]).cuda()
    a = P.act8_pack(x)
    q, e, v = act8_numpy(x.float().cpu().numpy())
    assert np.array_equal(a.exponent.cpu().numpy(), e) and np.array_equal(a.q.cpu().numpy(), q)
    got = P.act8_unpack(a, dtype=torch.float32).double().cpu().numpy()
    assert np.array_equal(got, v, equal_nan=True)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("shift", [0, 1, 8])
def test_workers_strides_and_untouched_surroundings(dtype, shift):
    K, R, Ccols = 3, 11, 96
    base = torch.randn(K, R + 1, Ccols + 32, device="cuda").to(DT[dtype])
    x = base[:, :R, shift:shift + Ccols]
    q = torch.full((K, R, Ccols + 32), 99, dtype=torch.int8, device="cuda")
    e = torch.full((K, R, 8), 99, dtype=torch.uint8, device="cuda")
    a = P.act8_pack(x, out=P.Act8(q[..., shift:shift + Ccols], e[..., 2:5], x.dtype))
    wq, we, wv = act8_numpy(x.float().reshape(K * R, Ccols).cpu().numpy())
    assert np.array_equal(a.q.reshape(K * R, Ccols).cpu().numpy(), wq)
    assert np.array_equal(a.exponent.reshape(K * R, 3).cpu().numpy(), we)
    assert bool((q[..., :shift] == 99).all()) and bool((q[..., shift + Ccols:] == 99).all())
    assert bool((e[..., :2] == 99).all()) and bool((e[..., 5:] == 99).all())
    out = torch.full_like(base, 5.0)
    P.act8_unpack(a, out=out[:, :R, shift:shift + Ccols])
    assert np.array_equal(out[:, :R, shift:shift + Ccols].double().reshape(K * R, Ccols).cpu().numpy(), wv)
    assert bool((out[:, R:] == 5).all()) and bool((out[:, :, :shift] == 5).all()) and bool((out[:, :, shift + Ccols:] == 5).all())


def test_rows_beyond_31_bits_of_elements():
    rows, cols = 70000, 32768 + 8                        # 2.3 G elements: offsets pass 31 bits
    x = torch.zeros(rows, cols, device="cuda", dtype=torch.bfloat16)
    at = [0, 1, 33333, 65535, 65536, rows - 1]
    for i in at:
        x[i, i % cols], x[i, cols - 1] = 3.0, -5.0
    a = P.act8_pack(x)
    back = P.act8_unpack(a)
    for i in at:
        assert float(back[i, i % cols]) == 3.0 and float(back[i, cols - 1]) == -5.0
    assert sum(float(back[i].float().abs().sum()) for i in at) == 8.0 * len(at)


# ---------------------------------------------------------------------------------------------- q/k norm + rotation

# K, tokens, heads_q, heads_k, head_dim, rotary_dim
QK = [(1, 1, 1, 1, 1, 0), (1, 1, 1, 1, 2, 2), (2, 3, 4, 2, 64, 64), (3, 77, 6, 2, 40, 40), (2, 33, 3, 3, 128, 64), (1, 50, 2, 1, 33, 10),
      (1, 9, 5, 0, 256, 256), (1, 9, 0, 5, 256, 32), (1, 20, 2, 2, 512, 512), (1, 20, 2, 2, 511, 500), (2, 30, 12, 12, 64, 36),
      (1, 600, 4, 4, 80, 80), (1, 10, 3, 1, 24, 8), (8, 5, 2, 1, 96, 48), (1, 7, 1, 1, 160, 160)]


def _qk_inputs(K, M, HQ, HK, DH, R, dt, seed=1):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s, m=0.0, std=1.0: (m + torch.randn(*s, generator=gen, device="cuda") * std).to(dt)
    q, k = r(K, M, HQ, DH), r(K, M, HK, DH, std=3.0)
    rows = 50
    ang = torch.rand(rows, R // 2, generator=gen, device="cuda", dtype=torch.float64) * 6.3
    pos = torch.randint(0, rows, (K, M), generator=gen, device="cuda", dtype=torch.int32)
    return q, k, r(K, DH, m=1.0, std=0.2), r(K, DH, m=1.0, std=0.2), ang.cos().float(), ang.sin().float(), pos, r(K, M, HQ, DH, std=0.1), r(K, M, HK, DH, std=0.1)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("size", QK, ids=str)
@pytest.mark.parametrize("interleaved", [False, True])
def test_qk_forward_and_backward(dtype, size, interleaved):
    q, k, wq, wk, cos, sin, pos, dq, dk = _qk_inputs(*size, DT[dtype])
    bf = dtype == "bf16"
    got = P.qk_norm_rope(q, k, wq, wk, cos, sin, pos, eps=1e-5, interleaved=interleaved)
    for t, x, w, n in zip(got, (q, k), (wq, wk), "qk"):
        within(t, *qk_forward64(x, w, pos, cos, sin, 1e-5, interleaved, bf), n)
    back = P.qk_norm_rope_backward(dq, dk, q, k, wq, wk, cos, sin, pos, eps=1e-5, interleaved=interleaved)
    for i, (d, x, w) in enumerate(((dq, q, wq), (dk, k, wk))):
        if x.shape[2] == 0:
            continue
        dx, dw = qk_backward64(d, x, w, pos, cos, sin, 1e-5, interleaved, bf)
        within(back[i], *dx, "dx")
        within(back[2 + i], *dw, "dw")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("shift", [0, 1])
def test_qk_views_of_one_projection(dtype, shift):
    K, M, HQ, HK, DH, R = 2, 21, 4, 2, 64, 64
    q, k, wq, wk, cos, sin, pos, dq, dk = _qk_inputs(K, M, HQ, HK, DH, R, DT[dtype], seed=2)
    width = (HQ + 2 * HK) * DH

    def fused():
        f = torch.full((K, M, width + 16), 1536.0, device="cuda", dtype=DT[dtype])
        v = f[:, :, shift:shift + width].unflatten(2, (HQ + 2 * HK, DH))
        return f, v[:, :, :HQ], v[:, :, HQ:HQ + HK]

    _, a, b = fused()
    a.copy_(q), b.copy_(k)
    out = fused()
    P.qk_norm_rope(a, b, wq, wk, cos, sin, pos, out=out[1:])
    for t, x, w in zip(out[1:], (q, k), (wq, wk)):
        within(t, *qk_forward64(x, w, pos, cos, sin, 1e-6, False, dtype == "bf16"), "out")
    grad = fused()
    dw = (torch.empty_like(wq), torch.empty_like(wk))
    P.qk_norm_rope_backward(dq, dk, a, b, wq, wk, cos, sin, pos, out=(*grad[1:], *dw))
    for t, d, x, w in zip(grad[1:], (dq, dk), (q, k), (wq, wk)):
        within(t, *qk_backward64(d, x, w, pos, cos, sin, 1e-6, False, dtype == "bf16")[0], "dx")
    for f in (out[0], grad[0]):
        assert bool((f[:, :, :shift] == 1536).all()) and bool((f[:, :, shift + (HQ + HK) * DH:] == 1536).all())


def test_qk_positions_outside_the_table_give_nan_rows_only():
    K, M = 1, 8
    q, k, wq, wk, cos, sin, pos, dq, dk = _qk_inputs(K, M, 2, 1, 64, 32, torch.float32, seed=3)
    pos[0, 2], pos[0, 5] = -1, 50
    oq, ok = P.qk_norm_rope(q, k, wq, wk, cos, sin, pos)
    for t in (oq, ok):
        bad = t.isnan().all(-1).all(-1)[0]
        assert bad.tolist() == [i in (2, 5) for i in range(M)]
        assert not bool(t[0, ~bad].isnan().any())
    dx, _, dw, _ = P.qk_norm_rope_backward(dq, dk, q, k, wq, wk, cos, sin, pos)
    assert bool(dw.isnan().all()) and not bool(dx[0, 0].isnan().any())


def test_qk_zero_rows_and_no_tokens():
    K, DH = 2, 64
    q, k, wq, wk, cos, sin, pos, dq, dk = _qk_inputs(K, 3, 2, 1, DH, 64, torch.float32, seed=4)
    q.zero_()
    oq, _ = P.qk_norm_rope(q, k, wq, wk, cos, sin, pos, eps=1e-6)
    assert bool((oq == 0).all())
    e = lambda t: t[:, :0]
    got = P.qk_norm_rope_backward(e(dq), e(dk), e(q), e(k), wq, wk, cos, sin, pos[:, :0],
                                  out=(None, None, torch.full_like(wq, 7), torch.full_like(wk, 7)))
    assert bool((got[2] == 0).all()) and bool((got[3] == 0).all())
    assert P.qk_norm_rope(e(q), e(k), wq, wk, cos, sin, pos[:, :0])[0].shape == (K, 0, 2, DH)


def test_qk_gradients_against_differences_and_repeatable():
    K, M, HQ, HK, DH, R = 2, 13, 3, 1, 16, 12
    q, k, wq, wk, cos, sin, pos, dq, dk = _qk_inputs(K, M, HQ, HK, DH, R, torch.float32, seed=5)
    args = [q, k, wq, wk]
    run = lambda *a: P.qk_norm_rope(*a, cos, sin, pos, interleaved=True)
    f = lambda *a: sum((o.double() * d.double()).sum() for o, d in zip(run(*a), (dq, dk)))
    grads = P.qk_norm_rope_backward(dq, dk, *args, cos, sin, pos, interleaved=True)
    again = P.qk_norm_rope_backward(dq, dk, *args, cos, sin, pos, interleaved=True)
    assert all(torch.equal(a, b) for a, b in zip(grads, again))
    gen = torch.Generator(device="cuda").manual_seed(6)
    h = 2.0 ** -6                                        # third-order term ~ h^2 / 6 of f', rounding 1e-6 / h
    for i in range(4):
        v = torch.randn(args[i].shape, generator=gen, device="cuda") * args[i].std()
        up, down = ([a + s * h * v if j == i else a for j, a in enumerate(args)] for s in (1, -1))
        numeric = float((f(*up) - f(*down)) / (2 * h))
        scale = float(grads[i].double().norm() * v.double().norm())
        assert abs(numeric - float((grads[i].double() * v.double()).sum())) <= 2e-3 * scale


def test_python_refusals():
    q, k, wq, wk, cos, sin, pos, dq, dk = _qk_inputs(1, 4, 2, 1, 16, 8, torch.float32)
    bad = [lambda: P.qk_norm_rope(q.cpu(), k, wq, wk, cos, sin, pos), lambda: P.qk_norm_rope(q, k.bfloat16(), wq, wk, cos, sin, pos),
           lambda: P.qk_norm_rope(q, k, wq[:, :8], wk, cos, sin, pos), lambda: P.qk_norm_rope(q, k, wq, wk, cos.double(), sin, pos),
           lambda: P.qk_norm_rope(q, k, wq, wk, cos, sin[:3], pos), lambda: P.qk_norm_rope(q, k, wq, wk, cos, sin, pos.long()),
           lambda: P.qk_norm_rope(q, k, wq, wk, cos, sin, pos, eps=-1.0),
           lambda: P.qk_norm_rope(q, k, wq, wk, cos, sin, pos, eps=float("nan")),
           lambda: P.qk_norm_rope(q, k, wq, wk, torch.cat([cos] * 3, 1), torch.cat([sin] * 3, 1), pos),
           lambda: P.qk_norm_rope(q, k, wq, wk, cos, sin, pos, out=(q[:, :, :1].expand_as(q), k)),
           lambda: P.act8_pack(q[0, 0].cpu()), lambda: P.act8_pack(q[0, 0].half()), lambda: P.act8_pack(q[0, 0].t()[::2]),
           lambda: P.act8_pack(q)]
    for call in bad:
        with pytest.raises(P.PalsgdError):
            call()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("cols", [24, 33, 64, 77])
@pytest.mark.parametrize("shift", range(8))
def test_act8_at_every_alignment(dtype, cols, shift):
    R = 13
    base = torch.randn(R, cols + 11, device="cuda").to(DT[dtype])
    x = base[:, shift:shift + cols]
    q = torch.full((R, cols + 9), 99, dtype=torch.int8, device="cuda")
    e = torch.empty(R, (cols + 31) // 32, dtype=torch.uint8, device="cuda")
    a = P.act8_pack(x, out=P.Act8(q[:, shift:shift + cols], e, x.dtype))
    wq, we, wv = act8_numpy(x.float().cpu().numpy())
    assert np.array_equal(a.q.cpu().numpy(), wq) and np.array_equal(a.exponent.cpu().numpy(), we)
    assert bool((q[:, :shift] == 99).all()) and bool((q[:, shift + cols:] == 99).all())
    out = torch.full_like(base, 5.0)
    P.act8_unpack(a, out=out[:, shift:shift + cols])
    assert np.array_equal(out[:, shift:shift + cols].double().cpu().numpy(), wv)
    assert bool((out[:, :shift] == 5).all()) and bool((out[:, shift + cols:] == 5).all())
