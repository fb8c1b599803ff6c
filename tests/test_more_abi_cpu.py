"""Host-side checks of the linear, layer norm and cross entropy entry points that need no GPU: layouts, refusals, workspaces."""
import ctypes as C

import pytest

import paper_2504_18454_b200 as P
from paper_2504_18454_b200 import block as B

N = C.byref
A = 0x10000000


def test_struct_layouts_match_the_header():
    assert C.sizeof(B.LinearShape) == 40 and B.LinearShape.tokens.offset == 16
    assert C.sizeof(B.NormShape) == 32 and B.NormShape.eps.offset == 24
    assert C.sizeof(B.LossShape) == 32 and B.LossShape.target_worker_stride.offset == 24
    assert P.ACT_NONE == 4


def _change(t, over):
    for name, v in over.items():
        if isinstance(v, dict):
            for f, w in v.items():
                setattr(t[name], f, w)
        else:
            t[name] = v
    return {k: (N(v) if v is not None else None) for k, v in t.items()}


def linear(back=False, K=2, prec=1, act=0, save=1, M=16, D=32, F=64, ws=None, n=0, size=True, **over):
    m = lambda i, r, c: B.Mat(A * (i + 1), r * c, c)
    t = dict(x=m(0, M, D), w=m(1, F, D), b=m(2, 1, F), r=m(3, M, F), y=m(4, M, F), z=m(5, M, F), ze=m(6, M, (F + 31) // 32), dy=m(7, M, F),
             dx=m(8, M, D), dw=m(9, F, D), db=m(10, 1, F), xe=None)
    r = _change(t, over)
    s, count = B.LinearShape(K, prec, act, save, M, D, F), C.c_size_t(n)
    pn = N(count) if size else None
    if back:
        rc = B.lib().palsgd_linear_backward(N(s), r["dy"], r["x"], r["xe"], r["w"], r["z"], r["ze"], r["dx"], r["dw"], r["db"], ws, pn, None)
    else:
        rc = B.lib().palsgd_linear_forward(N(s), r["x"], r["w"], r["b"], r["r"], r["y"], r["z"], r["ze"], ws, pn, None)
    return rc, count.value


LINEAR = [dict(K=0), dict(K=65), dict(prec=2), dict(act=5), dict(act=-1), dict(save=3), dict(save=-1), dict(act=4), dict(D=0), dict(F=0), dict(M=1 << 31),
          dict(D=1 << 31), dict(F=1 << 31), dict(x=None), dict(w=None), dict(z=None), dict(save=2, ze=None), dict(x=dict(data=None)),
          dict(w=dict(row_stride=-1)), dict(w=dict(worker_stride=-4)), dict(z=dict(row_stride=1 << 50)), dict(size=False)]


@pytest.mark.parametrize("over", LINEAR + [dict(y=None), dict(y=dict(row_stride=63)), dict(y=dict(worker_stride=0)), dict(z=dict(row_stride=0)),
                                           dict(save=2, ze=dict(worker_stride=1)), dict(b=dict(worker_stride=-1)), dict(r=dict(row_stride=-1)),
                                           dict(y=dict(data=A)), dict(y=dict(data=A * 4)), dict(z=dict(data=A * 5)), dict(b=dict(data=None))], ids=str)
def test_linear_forward_refuses_before_any_cuda_call(over):
    assert linear(**over)[0] == -1


@pytest.mark.parametrize("over", LINEAR + [dict(save=0), dict(dy=None), dict(dw=None), dict(dw=dict(row_stride=31)), dict(db=dict(worker_stride=63)),
                                           dict(dx=dict(row_stride=0)), dict(xe=B.Mat(A * 20, -1, 1)), dict(dx=dict(data=A * 8)),
                                           dict(dw=dict(data=A * 2)), dict(db=dict(data=A * 10))], ids=str)
def test_linear_backward_refuses_before_any_cuda_call(over):
    assert linear(back=True, **over)[0] == -1


@pytest.mark.parametrize("back", [False, True])
def test_linear_alignment_and_workspace(back):
    assert linear(back, x=dict(data=A + 1))[0] == -2 and linear(back, prec=0, w=dict(data=A * 2 + 2))[0] == -2
    for kw in (dict(), dict(prec=0), dict(save=2), dict(M=0), dict(M=5), dict(M=1, prec=0), dict(D=33, F=65), dict(M=700, F=8, D=4096), dict(act=4, save=0)):
        rc, need = linear(back, **kw)
        assert rc == 0 and need > 0
        assert linear(back, ws=A * 40, n=need - 1, **kw) == (-1, need)
        assert linear(back, ws=A * 40 + 128, n=need + 256, **kw)[0] == -2
        if need > 256 and kw.get("M") != 0:                # (256: a call that uses none)
            assert linear(back, ws=A, n=need, **kw)[0] == -1    # the workspace over x
    assert linear(back, b=None, r=None)[0] == 0
    assert linear(back, x=dict(worker_stride=0, row_stride=0), w=dict(worker_stride=0))[0] == 0
    assert linear(back, act=4, save=0, z=None, ze=None)[0] == 0
    if back:
        assert linear(back, dx=None)[0] == 0 and linear(back, db=None)[0] == 0
        assert linear(back, save=2, xe=B.Mat(A * 20, 16, 1))[0] == 0 and linear(back, act=4, save=0, xe=B.Mat(A * 20, 16, 1))[0] == 0


def norm(back=False, K=2, prec=1, M=16, D=64, eps=1e-5, ws=None, n=0, **over):
    m = lambda i, r, c: B.Mat(A * (i + 1), r * c, c)
    t = dict(x=m(0, M, D), r=m(1, M, D), w=m(2, 1, D), b=m(3, 1, D), y=m(4, M, D), total=m(5, M, D), mean=m(6, 1, M), rstd=m(7, 1, M), dy=m(8, M, D),
             past=m(9, M, D), dx=m(10, M, D), dw=m(11, 1, D), db=m(12, 1, D))
    r = _change(t, over)
    s, count = B.NormShape(K, prec, M, D, eps), C.c_size_t(n)
    if back:
        rc = B.lib().palsgd_layer_norm_backward(N(s), r["dy"], r["x"], r["w"], r["mean"], r["rstd"], r["past"], r["dx"], r["dw"], r["db"], ws, N(count), None)
        return rc, count.value
    return B.lib().palsgd_layer_norm_forward(N(s), r["x"], r["r"], r["w"], r["b"], r["y"], r["total"], r["mean"], r["rstd"], None), 0


NORM = [dict(K=0), dict(K=65), dict(prec=3), dict(D=0), dict(D=1 << 31), dict(M=1 << 31), dict(eps=-1.0), dict(eps=float("nan")), dict(x=None), dict(w=None),
        dict(x=dict(data=None)), dict(x=dict(row_stride=-1)), dict(mean=dict(worker_stride=-1))]


@pytest.mark.parametrize("over", NORM + [dict(b=None), dict(y=None), dict(total=None), dict(r=None), dict(y=dict(row_stride=63)), dict(mean=dict(worker_stride=15)),
                                         dict(total=dict(data=A)), dict(y=dict(data=A * 6)), dict(rstd=dict(data=A * 7))], ids=str)
def test_norm_forward_refuses_before_any_cuda_call(over):
    assert norm(**over)[0] == -1


@pytest.mark.parametrize("over", NORM + [dict(dy=None), dict(mean=None), dict(rstd=None), dict(dx=None), dict(dw=None), dict(db=None), dict(dx=dict(data=A * 9)),
                                         dict(dx=dict(row_stride=1)), dict(db=dict(data=A * 12)), dict(dw=dict(worker_stride=0))], ids=str)
def test_norm_backward_refuses_before_any_cuda_call(over):
    assert norm(True, **over)[0] == -1


def test_norm_alignment_width_and_workspace():
    for back in (False, True):
        assert norm(back, x=dict(data=A + 1))[0] == -2 and norm(back, rstd=dict(data=A * 8 + 2))[0] == -2
        assert norm(back, D=16385)[0] == -6
    for kw in (dict(), dict(M=0), dict(D=1), dict(prec=0), dict(past=None)):
        rc, need = norm(True, **kw)
        assert rc == 0 and need > 0 and norm(True, ws=A * 40, n=need - 1, **kw) == (-1, need)
    assert norm(True, ws=A * 40 + 16, n=1 << 30)[0] == -2
    assert norm(M=0)[0] == 0


def loss(back=False, K=2, prec=1, M=16, V=100, tw=16, targets=A * 20, **over):
    m = lambda i, r, c: B.Mat(A * (i + 1), r * c, c)
    r = _change(dict(z=m(0, M, V), loss=m(1, 1, M), lse=m(2, 1, M), d=m(3, 1, M), dz=m(4, M, V)), over)
    s, t = B.LossShape(K, prec, M, V, tw), C.c_void_p(targets)
    if back:
        return B.lib().palsgd_cross_entropy_backward(N(s), r["d"], r["z"], t, r["lse"], r["dz"], None)
    return B.lib().palsgd_cross_entropy_forward(N(s), r["z"], t, r["loss"], r["lse"], None)


@pytest.mark.parametrize("back", [False, True])
def test_loss_refusals(back):
    for over in (dict(K=0), dict(K=65), dict(prec=2), dict(V=0), dict(V=1 << 31), dict(M=1 << 31), dict(tw=-1), dict(targets=None), dict(z=None), dict(lse=None),
                 dict(z=dict(data=None)), dict(z=dict(row_stride=-1)), dict(lse=dict(worker_stride=-1))):
        assert loss(back, **over) == -1, over
    assert loss(back, z=dict(data=A + 1)) == -2 and loss(back, targets=A * 20 + 2) == -2 and loss(back, lse=dict(data=A * 3 + 2)) == -2
    if back:
        for over in (dict(d=None), dict(dz=None), dict(dz=dict(row_stride=99)), dict(dz=dict(data=A + 2)), dict(dz=dict(data=A * 20)), dict(dz=dict(data=A * 3)),
                     dict(dz=dict(data=A, row_stride=101, worker_stride=1616))):
            assert loss(True, **over) == -1, over
    else:
        for over in (dict(loss=None), dict(loss=dict(data=A)), dict(loss=dict(data=A * 3)), dict(loss=dict(worker_stride=15)), dict(lse=dict(data=A * 20))):
            assert loss(False, **over) == -1, over
    assert loss(back, M=0, targets=None) == 0


def test_null_shapes():
    L, n = B.lib(), C.c_size_t(0)
    assert L.palsgd_linear_forward(*[None] * 9, N(n), None) == -1
    assert L.palsgd_linear_backward(*[None] * 11, N(n), None) == -1
    assert L.palsgd_layer_norm_forward(*[None] * 10) == -1
    assert L.palsgd_layer_norm_backward(*[None] * 11, N(n), None) == -1
    assert L.palsgd_cross_entropy_forward(*[None] * 6) == -1
    assert L.palsgd_cross_entropy_backward(*[None] * 7) == -1


def test_cpu_tensors_are_refused():
    import torch
    t = torch.zeros(1, 2, 4)
    i = torch.zeros(1, 2, dtype=torch.int32)
    for call in (lambda: P.linear_forward(t, t), lambda: P.linear_backward(t, t, t), lambda: P.layer_norm_forward(t, t[0], t[0]),
                 lambda: P.layer_norm_backward(t, t, t[0], i, i), lambda: P.cross_entropy_forward(t, i), lambda: P.cross_entropy_backward(i, t, i, i)):
        with pytest.raises(P.PalsgdError):
            call()


def test_saved_forms_that_do_not_fit_are_refused():
    import torch
    t = torch.zeros(1, 2, 4)
    eight = P.Act8(t, t, torch.float32)
    with pytest.raises(P.PalsgdError, match="saved must be"):
        P.linear_forward(t, t, save=P.SAVE_FULL, saved=eight)
    with pytest.raises(P.PalsgdError, match="saved must be"):
        P.linear_forward(t, t, save=P.SAVE_8BIT, saved=t)
    with pytest.raises(P.PalsgdError, match="out must be"):
        P.linear_backward(t, t, t, out=(t,))
