"""Host-side checks of the block operators' C ABI where there is little or nothing to do (no GPU needed)."""
import ctypes as C

import pytest

from paper_2504_18454_b200 import block as B

A = 0x10000000
N = C.byref


def qk_backward(heads_q, heads_k, tokens=5, ws=None, n=0, **over):
    """The status and the bytes asked for, with addresses that nothing reads; a side without heads has NULL pointers."""
    s = B.QkShape(2, 1, tokens, heads_q, heads_k, 64, 64, 0, 0, 100, 5, 1e-6)
    h = lambda i, n: B.Heads(A * i, 5 * n * 64, n * 64, 64) if n else None
    t = dict(q=h(1, heads_q), k=h(2, heads_k), gq=h(3, heads_q), gk=h(4, heads_k), dq=h(5, heads_q), dk=h(6, heads_k),
             wq=B.Mat(7 * A, 64, 0) if heads_q else None, wk=B.Mat(8 * A, 64, 0) if heads_k else None,
             dwq=B.Mat(9 * A, 64, 0) if heads_q else None, dwk=B.Mat(10 * A, 64, 0) if heads_k else None)
    t.update(over)
    r = {k: (N(v) if v is not None else None) for k, v in t.items()}
    count = C.c_size_t(n)
    rc = B.lib().palsgd_qk_norm_rope_backward(N(s), r["gq"], r["gk"], r["q"], r["k"], r["wq"], r["wk"], *[C.c_void_p(A * (20 + i)) for i in range(3)],
                                              r["dq"], r["dk"], r["dwq"], r["dwk"], ws, N(count), None)
    return rc, count.value


@pytest.mark.parametrize("side", ["dwq", "dwk"])
def test_a_weight_gradient_of_no_heads_is_checked_where_it_is_given(side):
    heads = (0, 2) if side == "dwq" else (2, 0)
    assert qk_backward(*heads)[0] == 0
    assert qk_backward(*heads, **{side: B.Mat(None, 64, 0)})[0] == 0
    assert qk_backward(*heads, **{side: B.Mat(A * 11, 64, 0)})[0] == 0
    assert qk_backward(*heads, **{side: B.Mat(A * 11, 63, 0)})[0] == -1
    assert qk_backward(*heads, **{side: B.Mat(A * 11, -64, 0)})[0] == -1
    assert qk_backward(*heads, **{side: B.Mat(A * 11 + 1, 64, 0)})[0] == -2


def ffn(back, tokens=0, ws=None, n=0):
    D, F = 32, 64
    s, m = B.FfnShape(2, 1, 0, 1, tokens, D, F), lambda i, r, c: B.Mat(A * i, r * c, c)
    x, wg, wu, wd, y, g, u, dwg, dwu, dwd = (N(m(i + 1, *rc)) for i, rc in enumerate(
        [(tokens, D), (F, D), (F, D), (D, F), (tokens, D), (tokens, F), (tokens, F), (F, D), (F, D), (D, F)]))
    count = C.c_size_t(n)
    if back:
        rc = B.lib().palsgd_ffn_backward(N(s), y, x, None, wg, wu, wd, g, u, None, None, None, dwg, dwu, dwd, ws, N(count), None)
    else:
        rc = B.lib().palsgd_ffn_forward(N(s), x, wg, wu, wd, y, g, u, None, None, ws, N(count), None)
    return rc, count.value


@pytest.mark.parametrize("call", [lambda **k: ffn(False, **k), lambda **k: ffn(True, **k), lambda **k: qk_backward(0, 0, **k),
                                  lambda **k: qk_backward(2, 1, tokens=0, **k)], ids=["forward", "backward", "no heads", "no tokens"])
def test_a_call_with_nothing_to_do_still_asks_for_a_workspace(call):
    """A caller who is told 0 bytes passes NULL for them, which would be taken for the question again: the weight gradients
    of a backward call would stay as they were, with status OK."""
    rc, need = call()
    assert rc == 0 and need > 0
    assert call(ws=A * 30, n=need - 1) == (-1, need)
