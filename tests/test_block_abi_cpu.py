"""Host-side checks of the block operators' C ABI that need no GPU: exports, struct layouts, refusals before any CUDA call."""
import ctypes as C
import os
import re

import pytest

import paper_2504_18454_b200 as P
from paper_2504_18454_b200 import block as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
N = C.byref


def test_library_exports_every_declared_entry_point():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "palsgd_block.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(palsgd_[a-z_0-9]+)\s*\(", text)))
    assert {"palsgd_act8_pack", "palsgd_act8_unpack", "palsgd_ffn_forward", "palsgd_ffn_backward",
            "palsgd_qk_norm_rope_forward", "palsgd_qk_norm_rope_backward"} <= set(names)
    for n in names:
        assert hasattr(B.lib(), n), n


def test_struct_layouts_match_the_header():
    assert C.sizeof(B.Mat) == 24 and C.sizeof(B.Heads) == 32
    assert C.sizeof(B.FfnShape) == 40 and B.FfnShape.tokens.offset == 16
    assert C.sizeof(B.QkShape) == 64 and B.QkShape.table_rows.offset == 40 and B.QkShape.eps.offset == 56


A = 0x10000000


def _mats(K, M, D, F, es):
    """Plausible matrices at addresses that nothing reads; each far from the others."""
    m = lambda i, r, c: B.Mat(A * (i + 1), r * c, c)
    return dict(x=m(0, M, D), wg=m(1, F, D), wu=m(2, F, D), wd=m(3, D, F), y=m(4, M, D), gate=m(5, M, F), up=m(6, M, F),
                ge=m(7, M, (F + 31) // 32), ue=m(8, M, (F + 31) // 32), dy=m(9, M, D), dx=m(10, M, D), dwg=m(11, F, D),
                dwu=m(12, F, D), dwd=m(13, D, F))


def _ffn(back=False, K=2, prec=1, act=0, save=1, M=16, D=32, F=64, xe=None, ws=None, n=0, size=True, **over):
    s = B.FfnShape(K, prec, act, save, M, D, F)
    t = _mats(max(K, 1), M, D, F, 2)
    for name, v in over.items():
        if isinstance(v, dict):
            for f, w in v.items():
                setattr(t[name], f, w)
        else:
            t[name] = v
    r = {k: (N(v) if v is not None else None) for k, v in t.items()}
    count = C.c_size_t(n)
    pn = N(count) if size else None
    if back:
        rc = B.lib().palsgd_ffn_backward(N(s), r["dy"], r["x"], N(xe) if xe else None, r["wg"], r["wu"], r["wd"], r["gate"],
                                         r["up"], r["ge"], r["ue"], r["dx"], r["dwg"], r["dwu"], r["dwd"], ws, pn, None)
    else:
        rc = B.lib().palsgd_ffn_forward(N(s), r["x"], r["wg"], r["wu"], r["wd"], r["y"], r["gate"], r["up"], r["ge"], r["ue"],
                                        ws, pn, None)
    return rc, count.value


COMMON = [dict(K=0), dict(K=65), dict(prec=2), dict(prec=-1), dict(act=4), dict(act=-1), dict(save=3), dict(D=0), dict(F=0),
          dict(M=1 << 31), dict(D=1 << 31), dict(x=None), dict(wg=None), dict(wu=None), dict(wd=None), dict(gate=None),
          dict(up=None), dict(save=2, ge=None), dict(save=2, ue=None), dict(x=dict(data=None)), dict(wd=dict(row_stride=-1)),
          dict(wg=dict(worker_stride=-64)), dict(wu=dict(row_stride=1 << 50)), dict(size=False)]


@pytest.mark.parametrize("over", COMMON + [dict(y=None), dict(y=dict(row_stride=31)), dict(y=dict(worker_stride=0)),
                                           dict(gate=dict(worker_stride=100)), dict(up=dict(row_stride=0))], ids=str)
def test_forward_refuses_before_any_cuda_call(over):
    assert _ffn(**over)[0] == -1


@pytest.mark.parametrize("over", COMMON + [dict(save=0), dict(dy=None), dict(dwg=None), dict(dwu=None), dict(dwd=None),
                                           dict(dx=dict(row_stride=8)), dict(dwd=dict(worker_stride=1)),
                                           dict(xe=B.Mat(A, 16, 1))], ids=str)
def test_backward_refuses_before_any_cuda_call(over):
    assert _ffn(back=True, **over)[0] == -1


def test_alignment_and_workspace():
    assert _ffn(x=dict(data=A + 1))[0] == -2 and _ffn(back=True, dwg=dict(data=A + 1))[0] == -2
    assert _ffn(prec=0, wd=dict(data=A + 2))[0] == -2
    for back in (False, True):
        for kw in (dict(), dict(prec=0), dict(save=2), dict(M=0), dict(D=33, F=65)):
            rc, need = _ffn(back=back, **kw)
            assert rc == 0
            if need:
                assert _ffn(back=back, ws=A * 20, n=need - 1, **kw)[0] == -1
            assert _ffn(back=back, ws=A * 20 + 128, n=need + 256, **kw)[0] == -2
    # rows that interleave with workers are no overlap; absent save needs no matrices
    assert _ffn(y=dict(worker_stride=32, row_stride=64))[0] == 0
    assert _ffn(save=0, gate=None, up=None, ge=None, ue=None)[0] == 0
    assert _ffn(back=True, dx=None)[0] == 0


def _act8(pack=True, prec=1, K=1, rows=4, cols=40, **over):
    t = dict(x=B.Mat(A, rows * cols, cols), q=B.Mat(2 * A, rows * cols, cols), e=B.Mat(3 * A, rows * 2, 2))
    for name, v in over.items():
        if isinstance(v, dict):
            for f, w in v.items():
                setattr(t[name], f, w)
        else:
            t[name] = v
    r = {k: (N(v) if v is not None else None) for k, v in t.items()}
    if pack:
        return B.lib().palsgd_act8_pack(prec, K, rows, cols, r["x"], r["q"], r["e"], None)
    return B.lib().palsgd_act8_unpack(prec, K, rows, cols, r["q"], r["e"], r["x"], None)


@pytest.mark.parametrize("pack", [True, False])
def test_act8_refusals(pack):
    for over in (dict(K=0), dict(K=65), dict(prec=2), dict(x=None), dict(q=None), dict(e=None), dict(x=dict(data=None)),
                 dict(q=dict(row_stride=-1)), dict(rows=1 << 31), dict(cols=1 << 31)):
        assert _act8(pack, **over) == -1
    assert _act8(pack, x=dict(data=A + 1)) == -2
    assert _act8(True, q=dict(row_stride=39)) == -1 and _act8(True, K=2, e=dict(worker_stride=7)) == -1
    assert _act8(False, x=dict(row_stride=39)) == -1
    assert _act8(pack, rows=0) == 0 and _act8(pack, cols=0) == 0


def _qk(back=False, null=None, **over):
    f = dict(K=2, precision=1, tokens=5, heads_q=4, heads_k=2, head_dim=64, rotary_dim=64, interleaved=0, reserved_=0,
             table_rows=100, pos_worker_stride=5, eps=1e-6)
    f.update({k: v for k, v in over.items() if k in f})
    s = B.QkShape(**f)
    h = lambda i, n: B.Heads(A * i, 5 * n * 64, n * 64, 64)
    t = dict(q=h(1, 4), k=h(2, 2), oq=h(3, 4), ok=h(4, 2), dq=h(5, 4), dk=h(6, 2), wq=B.Mat(7 * A, 64, 0), wk=B.Mat(8 * A, 64, 0),
             dwq=B.Mat(9 * A, 64, 0), dwk=B.Mat(10 * A, 64, 0))
    for name, v in over.items():
        if name in t:
            for g, w in v.items():
                setattr(t[name], g, w)
    r = {k: (N(v) if k != null else None) for k, v in t.items()}
    tab = [C.c_void_p(None if null == n else A * (20 + i)) for i, n in enumerate(("cos", "sin", "pos"))]
    if not back:
        return B.lib().palsgd_qk_norm_rope_forward(N(s), r["q"], r["k"], r["wq"], r["wk"], *tab, r["oq"], r["ok"], None)
    n = C.c_size_t(0)
    return B.lib().palsgd_qk_norm_rope_backward(N(s), r["oq"], r["ok"], r["q"], r["k"], r["wq"], r["wk"], *tab, r["dq"],
                                                r["dk"], r["dwq"], r["dwk"], None, N(n), None)


@pytest.mark.parametrize("back", [False, True])
def test_qk_refusals(back):
    for over in (dict(K=0), dict(K=65), dict(precision=2), dict(head_dim=0), dict(rotary_dim=63), dict(rotary_dim=66),
                 dict(interleaved=2), dict(reserved_=1), dict(eps=-1.0), dict(eps=float("inf")), dict(tokens=1 << 31),
                 dict(pos_worker_stride=-1), dict(heads_q=70000), dict(null="q"), dict(null="wk"), dict(null="cos"),
                 dict(null="pos"), dict(q=dict(data=None)), dict(k=dict(token_stride=-1))):
        assert _qk(back, **over) == -1, over
    out = "dq" if back else "oq"
    assert _qk(back, **{out: dict(head_stride=63)}) == -1 and _qk(back, **{out: dict(worker_stride=0)}) == -1
    assert _qk(back, head_dim=514, rotary_dim=64) == -6
    assert _qk(back, q=dict(data=A + 1)) == -2
    if back:
        assert _qk(True, null="dwq") == -1 and _qk(True) == 0
    else:
        assert _qk(False, tokens=0) == 0


def test_null_shapes():
    L = B.lib()
    n = C.c_size_t(0)
    assert L.palsgd_ffn_forward(*[None] * 11, N(n), None) == -1
    assert L.palsgd_ffn_backward(*[None] * 16, N(n), None) == -1
    assert L.palsgd_qk_norm_rope_forward(*[None] * 11) == -1
    assert L.palsgd_qk_norm_rope_backward(*[None] * 15, N(n), None) == -1


def test_cpu_tensors_are_refused():
    import torch
    t = torch.zeros(1, 2, 4)
    with pytest.raises(P.PalsgdError):
        P.ffn_forward(t, t, t, t)
    with pytest.raises(P.PalsgdError):
        P.act8_pack(t)
    with pytest.raises(P.PalsgdError):
        P.qk_norm_rope(t[None], t[None], t, t, t, t, t)
