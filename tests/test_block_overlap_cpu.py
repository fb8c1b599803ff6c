"""Overlap of what a block operator writes with what it reads: refused by every entry point, told exactly (no GPU needed: the
calls only ask for the workspace's size, or have nothing to launch)."""
import ctypes as C
import random

import pytest

from paper_2504_18454_b200 import block as B

N = C.byref
A = 0x10000000


def ffn(t, back=False, K=2, prec=1, save=1, M=6, D=8, F=12):
    """The status of a call that asks for the workspace; t: Mats by name."""
    s, n = B.FfnShape(K, prec, 0, save, M, D, F), C.c_size_t(0)
    r = {k: N(v) for k, v in t.items()}
    g = [r.get(k) for k in ("gate", "up", "gate_e", "up_e")]
    if back:
        return B.lib().palsgd_ffn_backward(N(s), r["dy"], r["x"], None, r["wg"], r["wu"], r["wd"], *g, r.get("dx"), r["dwg"], r["dwu"], r["dwd"],
                                           None, N(n), None)
    return B.lib().palsgd_ffn_forward(N(s), r["x"], r["wg"], r["wu"], r["wd"], r["y"], *g, None, N(n), None)


def mats(M=6, D=8, F=12):
    m = lambda i, r, c: B.Mat(A * (i + 1), r * c, c)
    return dict(x=m(0, M, D), wg=m(1, F, D), wu=m(2, F, D), wd=m(3, D, F), y=m(4, M, D), gate=m(5, M, F), up=m(6, M, F), dy=m(7, M, D),
                dx=m(8, M, D), dwg=m(9, F, D), dwu=m(10, F, D), dwd=m(11, D, F))


@pytest.mark.parametrize("a,b", [("y", "x"), ("gate", "x"), ("y", "wd"), ("gate", "up"), ("y", "gate"), ("up", "wg")])
def test_forward(a, b):
    t = mats()
    assert ffn(t) == 0
    t[a].data = t[b].data + 2 * 5
    assert ffn(t) == -1


@pytest.mark.parametrize("a,b", [("dx", "dy"), ("dx", "x"), ("dwg", "dwu"), ("dwd", "wd"), ("dwu", "gate"), ("dx", "dwd")])
def test_backward(a, b):
    t = mats()
    assert ffn(t, True) == 0
    t[a].data = t[b].data
    assert ffn(t, True) == -1


def test_views_of_one_buffer_are_no_overlap():
    """Rows of an arena (one worker stride, other row strides), and columns side by side in wider rows."""
    M, D, F, K = 6, 8, 12, 2
    t, row = mats(), 3 * F * D + 5
    for i, n in enumerate(("dwg", "dwu", "dwd")):
        t[n] = B.Mat(A * 20 + 2 * i * F * D, row, D if i < 2 else F)
    wide = D + D + F + F
    for n, c in (("x", 0), ("dx", D), ("gate", 2 * D), ("up", 2 * D + F)):
        t[n] = B.Mat(A * 30 + 2 * c, M * wide, wide)
    assert ffn(t, True) == 0
    t["dx"].data -= 2
    assert ffn(t, True) == -1
    t["dx"].data += 4
    assert ffn(t, True) == -1


def test_workspace():
    t = mats()
    s, n = B.FfnShape(2, 0, 0, 1, 6, 8, 12), C.c_size_t(0)
    call = lambda ws: B.lib().palsgd_ffn_forward(N(s), N(t["x"]), N(t["wg"]), N(t["wu"]), N(t["wd"]), N(t["y"]), N(t["gate"]), N(t["up"]), None,
                                                 None, ws, N(n), None)
    assert call(None) == 0
    assert call(t["x"].data) == -1 and call(t["wd"].data - n.value // 256 * 256 + 256) == -1


def places(m, K, rows, cols, es):
    return {m.data + es * (k * m.worker_stride + r * m.row_stride) + b for k in range(K) for r in range(rows) for b in range(cols * es)}


def test_random_layouts_against_the_bytes_themselves():
    """Small matrices of random strides near each other: y and x alike in shape, gate of another width."""
    rng = random.Random(7)
    seen = [0, 0]
    for _ in range(4000):
        K, M, D, F = rng.randint(1, 3), rng.randint(1, 4), rng.randint(1, 5), rng.randint(1, 5)
        t = mats(M, D, F)
        def lay(cols, output):
            while True:
                w, r = rng.choice([0, rng.randint(1, 60)]), rng.choice([0, cols, rng.randint(1, 24)])
                m = B.Mat(A * 40 + 2 * rng.randint(0, 120), w, r)
                p = places(m, K, M, cols, 2)
                if not output or (len(p) == K * M * cols * 2 and ok_output(K, M, w, r, cols)):
                    return m, p
        pairs = rng.sample([("x", D, False), ("y", D, True), ("gate", F, True), ("up", F, True)], 2)
        if not any(o for _, _, o in pairs):
            continue
        got = []
        for name, cols, out in pairs:
            t[name], p = lay(cols, out)
            got.append(p)
        meets = bool(got[0] & got[1])
        seen[meets] += 1
        assert ffn(t, K=K, M=M, D=D, F=F) == (-1 if meets else 0), [(n, t[n].data, t[n].worker_stride, t[n].row_stride) for n, _, _ in pairs]
    assert min(seen) > 500


def ok_output(K, M, w, r, cols):
    """The condition that the library has for an output's own rows: each axis steps over the one inside it."""
    span = cols
    for n, s in sorted(((K, w if K > 1 else 0), (M, r if M > 1 else 0)), key=lambda a: a[1]):
        if n > 1:
            if s < span:
                return False
            span += s * (n - 1)
    return True


def test_checkpoints():
    """Refused before anything is launched; calls without overlap are left to the GPU tests."""
    rows, cols = 4, 40
    x, q, e = B.Mat(A, rows * cols, cols), B.Mat(2 * A, rows * cols, cols), B.Mat(3 * A, rows * 2, 2)
    for a, b in ((q, x), (e, x), (e, q)):
        kept, a.data = a.data, b.data + 8
        assert B.lib().palsgd_act8_pack(1, 1, rows, cols, N(x), N(q), N(e), None) == -1
        a.data = kept
    for a in (q, e):
        kept, a.data = a.data, x.data + 8
        assert B.lib().palsgd_act8_unpack(1, 1, rows, cols, N(q), N(e), N(x), None) == -1
        a.data = kept


def qk(back, tokens=5, **over):
    """Forward: only calls that are refused, or with no heads, may be made here."""
    s = B.QkShape(2, 1, tokens, 4, 4, 64, 64, 0, 0, 100, 5, 1e-6)
    h = lambda i: B.Heads(A * i, 5 * 4 * 64, 4 * 64, 64)
    t = dict(q=h(1), k=h(2), oq=h(3), ok=h(4), dq=h(5), dk=h(6), wq=B.Mat(7 * A, 64, 0), wk=B.Mat(8 * A, 64, 0), dwq=B.Mat(9 * A, 64, 0),
             dwk=B.Mat(10 * A, 64, 0))
    for k, v in over.items():
        t[k].data = v
    r = {k: N(v) for k, v in t.items()}
    tab = [C.c_void_p(A * (20 + i)) for i in range(3)]
    if not back:
        return B.lib().palsgd_qk_norm_rope_forward(N(s), r["q"], r["k"], r["wq"], r["wk"], *tab, r["oq"], r["ok"], None)
    return B.lib().palsgd_qk_norm_rope_backward(N(s), r["oq"], r["ok"], r["q"], r["k"], r["wq"], r["wk"], *tab, r["dq"], r["dk"], r["dwq"], r["dwk"],
                                                None, N(C.c_size_t(0)), None)


def test_heads():
    for over in (dict(oq=A + 128), dict(oq=2 * A), dict(ok=3 * A), dict(oq=7 * A), dict(oq=20 * A), dict(ok=22 * A), dict(q=5 * A, k=5 * A, oq=5 * A)):
        assert qk(False, **over) == -1, over
    for over in (dict(dq=A + 128), dict(dq=2 * A), dict(dq=4 * A), dict(dk=5 * A), dict(dwq=7 * A), dict(dwk=6 * A), dict(dwq=10 * A), dict(dk=21 * A)):
        assert qk(True, **over) == -1, over
    for over in (dict(), dict(dq=A), dict(dq=3 * A, dk=4 * A), dict(dk=2 * A)):      # in place
        assert qk(True, **over) == 0, over
